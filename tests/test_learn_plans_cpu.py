"""What plans and learners hold on to and refuse before anything is launched (CPU only)."""
import gc
import weakref

import pytest
import torch

from paper_2407_15462_amd import mol


def test_adamw_plan_keeps_its_tensors_when_the_lists_change():
    """The descriptors hold addresses: whatever the caller does to the lists afterwards, the tensors stay."""
    f = lambda: torch.zeros(300)  # noqa: E731
    e = lambda: torch.zeros(300, dtype=torch.uint8).view(torch.float8_e4m3fn)  # noqa: E731
    s = lambda: torch.zeros(2)  # noqa: E731
    lists = dict(p=[f()], g=[f()], m=[e()], v=[e()], m_scale=[s()], v_scale=[s()])
    out = dict(p=[f()], m=[e()], v=[e()], m_scale=[s()], v_scale=[s()], copy=[f().bfloat16()])
    held = {k: weakref.ref(x[0]) for k, x in lists.items()}
    held.update({"out " + k: weakref.ref(x[0]) for k, x in out.items()})
    address = {k: r().data_ptr() for k, r in held.items()}
    plan = mol.AdamwTensors(**lists, out=out)
    for x in lists.values():
        x[0] = None
    for x in out.values():
        x.clear()
    out.clear()
    gc.collect()
    gone = [k for k, r in held.items() if r() is None]
    assert not gone, f"freed under the plan: {gone}"
    assert all(r().data_ptr() == address[k] for k, r in held.items())
    del plan
    gc.collect()
    assert all(r() is None for r in held.values())
