"""The workspaces of the cross entropy against the bounds that the header states (nothing here needs a GPU)."""
import math
import random

import pytest

MIB = 1 << 20


@pytest.fixture(scope="module")
def tfe():
    from paper_2607_07388_b200 import binding, build
    build.build()
    binding.lib()
    return binding


def up(x, to):
    return -(-x // to) * to


def cases():
    rng = random.Random(1)
    log = lambda lo, hi: int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    yield from [(1, 1, 8), (64, 151_936, 1024), (65, 151_936, 1024), (256, 262_144, 4096), (257, 262_144, 4096), (3840, 262_144, 1024), (4096, 151_936, 1024), (1 << 20, 151_936, 64),
                (1 << 20, 4096, 4096), (1 << 20, 151_936, 8), (32_768, 32_768, 128), (32_769, 1 << 24, 136), (1 << 24, 1 << 24, 8), (1 << 24, 1, 1 << 16), (1, 1 << 24, 1 << 16)]
    for _ in range(4000):
        yield log(1, 1 << 24), log(1, 1 << 24), 8 * log(1, 1 << 13)


def test_workspace_bounds(tfe):
    for N, V, d in cases():
        n, wide = up(N, 256), up(d, 256 if d >= 256 else 128)
        small = 16 * 256                    # every part begins on a boundary of 256 bytes
        forward = 64 * MIB + 16 * n + (2 * n * d + 12 * n if N > 256 else 0) + small
        assert 0 < tfe.tfe_xent_forward_workspace_bytes(N, V, d) <= forward, (N, V, d)
        g = max(256 * MIB, 8192 * n)
        backward = g + g // 64 + 2 * n * d + max(256 * MIB, 4 * n * wide) + 4 * min(n, V) * d + 32 * n + 5 * V + small
        assert 0 < tfe.tfe_xent_backward_workspace_bytes(N, V, d) <= backward, (N, V, d)


def test_narrow_rows_take_no_room_for_wide_ones(tfe):
    """Up to 128 columns the sums of grad_hidden take 512 bytes a row (they took 1,024)."""
    N, V = 1 << 20, 32_000
    n = N
    g = 8192 * n
    assert tfe.tfe_xent_backward_workspace_bytes(N, V, 64) <= g + g // 64 + 128 * n + 512 * n + 256 * V + 32 * n + 5 * V + 4096


@pytest.mark.parametrize("how", ["missing", "version", "function"])
def test_a_torch_that_cannot_be_asked_about_its_tensors(tfe, monkeypatch, how):
    """Said as what it is, by its own name, and not as a refusal of the tensors."""
    import ctypes as C

    import torch

    from paper_2607_07388_b200 import engine
    monkeypatch.setattr(tfe, "_describe", None)
    exchange = tfe._DlpackExchange(2 if how == "version" else 1, 0, None, None, None, None, None if how == "function" else 1, None)
    new = C.pythonapi.PyCapsule_New
    new.restype, new.argtypes = C.py_object, [C.c_void_p, C.c_char_p, C.c_void_p]
    name = b"dlpack_exchange_api"
    monkeypatch.setattr(torch.Tensor, "__dlpack_c_exchange_api__", None if how == "missing" else new(C.addressof(exchange), name, None), raising=False)
    for call in (lambda: engine.grad_norm([torch.ones(3)]), lambda: engine.clip_grad_norm([torch.ones(3)], 1.0)):
        with pytest.raises(NotImplementedError, match="DLPack"):
            call()
    assert tfe._describe is None
