"""MI355X-native Mixture-of-Logits retrieval (gfx950 HIP kernels behind a C ABI).

The compute path lives in libmol.so (paper_2407_15462_amd/csrc, declared in
include/mol.h); this package is its Python binding.
"""
from . import mol
from .mol import (AdamwTensors, Learner, MolError, Problem, adamw_step, avg_embed, averaged_problem,
                  embed_grad, embed_lookup, rerank, score, score_grad, softmax_loss,
                  topk_exact, topk_per_embd)

__all__ = ["mol", "MolError", "Problem", "score", "topk_exact", "topk_per_embd", "rerank",
           "avg_embed", "averaged_problem", "embed_lookup", "embed_grad", "softmax_loss", "score_grad",
           "AdamwTensors", "adamw_step", "Learner"]
