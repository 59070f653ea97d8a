"""BlockCache without a GPU: which buffers a call is given."""
import os

import pytest
import torch


@pytest.fixture
def A(monkeypatch):
    from paper_2409_16546_amd import binding
    if not os.path.exists(binding.LIB_PATH):
        from paper_2409_16546_amd import build
        build.build_library(verbose=False)
    monkeypatch.setattr(binding, "_ptr", lambda t: None if t is None else t.data_ptr())   # (it takes device tensors only)
    return binding


def buffers(A, *shape):
    sz = A.akb_layout_sizes(*shape)
    kinds = dict(k8=torch.uint8, v8=torch.uint8, exps=torch.int8, k_tail=shape[-1], v_tail=shape[-1], lens=torch.int32, flags=torch.int32, score=torch.float32)
    return {n: torch.zeros(getattr(sz, n) // torch.empty(0, dtype=t).element_size(), dtype=t) for n, t in kinds.items()}


def test_assigned_fields_reach_the_next_call(A):
    shape = (2, 4, 2, 64, 128, torch.float16)
    first, second = buffers(A, *shape), buffers(A, *shape)
    c = A.BlockCache(*shape, **{**first, "score": None})
    assert c.struct().score is None and c.ref()._obj is c.struct()
    for name, t in second.items():
        setattr(c, name, t)
        assert getattr(c.ref()._obj, name) == t.data_ptr(), name
        assert getattr(c.struct(), name) == t.data_ptr(), name
    c.score = None
    assert c.ref()._obj.score is None
    kept = c.ref()
    c.workspace = torch.zeros(256, dtype=torch.uint8)     # no part of the struct
    assert c.ref() is kept


def test_assigned_fields_are_checked(A):
    shape = (2, 4, 2, 64, 128, torch.float16)
    c = A.BlockCache(*shape, **buffers(A, *shape))
    c.ref()
    for name, bad in (("k8", torch.zeros(64, dtype=torch.uint8)), ("lens", torch.zeros(2, dtype=torch.int64)), ("k_tail", torch.zeros(2 * 2 * 64 * 64, dtype=torch.bfloat16)),
                      ("score", torch.zeros(5)), ("Ncap", 192), ("dtype", torch.bfloat16)):
        good = getattr(c, name)
        setattr(c, name, bad)
        with pytest.raises(AssertionError):
            c.ref()
        setattr(c, name, good)
        c.ref()
    c.Ncap = 100
    with pytest.raises(A.AkvError):
        c.ref()
