"""Refusals of the calls on rows of logits: found on the host, before any device call (nothing here needs a GPU)."""
import pytest

P = 0x1000                                  # an address that is never touched


@pytest.fixture(scope="module")
def tfe():
    from paper_2607_07388_b200 import binding, build
    build.build()
    binding.lib()
    return binding


def test_distillation(tfe):
    L = tfe.lib()

    def forward(logits=P, dtype=1, N=2, V=8, ld=8, ids=P, t=P, K=4, tau=1.0, loss=P, lse=P):
        return L.tfe_distill_forward(logits, dtype, N, V, ld, ids, t, K, tau, loss, lse, None)

    def backward(logits=P, dtype=1, N=2, V=8, ld=8, ids=P, t=P, K=4, tau=1.0, lse=P, g=P, grad=2 * P, ld_grad=8):
        return L.tfe_distill_backward(logits, dtype, N, V, ld, ids, t, K, tau, lse, g, grad, ld_grad, None)

    both = [dict(dtype=2), dict(dtype=-1), dict(N=-1), dict(N=tfe.ROWS_MAX + 1), dict(V=0), dict(ld=7), dict(ld=1 << 40),
            dict(logits=None), dict(logits=P + 2), dict(dtype=0, logits=P + 1), dict(ids=None), dict(ids=P + 2), dict(t=None),
            dict(t=P + 1), dict(K=0), dict(K=tfe.DISTILL_MAX_TOP + 1), dict(tau=0.0), dict(tau=-1.0), dict(tau=float("nan")),
            dict(tau=float("inf")), dict(lse=None)]
    for kw in both + [dict(loss=None)]:
        assert forward(**kw) == tfe.TFE_ERR_INVALID_ARG, kw
    for kw in both + [dict(g=None), dict(grad=None), dict(grad=P + 32), dict(grad=P - 32), dict(grad=P, ld_grad=9), dict(ld_grad=7),
                      dict(grad=2 * P + 2)]:
        assert backward(**kw) == tfe.TFE_ERR_INVALID_ARG, kw
    assert forward(N=0, logits=None, ids=None, t=None, loss=None, lse=None) == tfe.TFE_OK
    assert backward(N=0, logits=None, ids=None, t=None, lse=None, g=None, grad=None) == tfe.TFE_OK


def test_sampling(tfe):
    import ctypes as C
    L = tfe.lib()

    def sample(logits=P, dtype=1, B=2, V=8, ld=8, params=(None, None, None, None), u=P, tokens=P, prob=None):
        prm = None if params is None else C.byref(tfe.TfeSampleParams(*params))
        return L.tfe_sample_tokens(logits, dtype, B, V, ld, prm, u, tokens, prob, None)

    for kw in (dict(dtype=2), dict(B=-1), dict(B=tfe.ROWS_MAX + 1), dict(V=0), dict(V=tfe.SAMPLE_MAX_VOCAB + 1, ld=1 << 30), dict(ld=7),
               dict(ld=1 << 40), dict(logits=None), dict(logits=P + 2), dict(u=None), dict(u=P + 1), dict(tokens=None), dict(tokens=P + 2),
               dict(prob=P + 2), dict(params=None), dict(params=(P + 1, None, None, None)), dict(params=(None, P + 2, None, None)),
               dict(params=(None, None, P + 3, None)), dict(params=(None, None, None, P + 1))):
        assert sample(**kw) == tfe.TFE_ERR_INVALID_ARG, kw
    assert sample(B=0, logits=None, u=None, tokens=None) == tfe.TFE_OK


def test_conversion_and_product_in_8_bits(tfe):
    import ctypes as C
    L = tfe.lib()

    def quantize(x=P, dtype=1, R=2, C_=8, ld=8, block_rows=1, q=P, scale=P):
        return L.tfe_quantize_fp8(x, dtype, R, C_, ld, block_rows, q, scale, None)

    for kw in (dict(dtype=2), dict(R=-1), dict(C_=0), dict(C_=tfe.FP8_MAX_COLS + 1, ld=1 << 20), dict(ld=7), dict(ld=1 << 40), dict(block_rows=0),
               dict(block_rows=64), dict(x=None), dict(x=P + 2), dict(q=None), dict(scale=None), dict(scale=P + 2),
               dict(R=(1 << 31) - 1, C_=256, ld=256)):
        assert quantize(**kw) == tfe.TFE_ERR_INVALID_ARG, kw
    assert quantize(R=0, x=None, q=None, scale=None) == tfe.TFE_OK

    def product(a=P, lda=64, sa=P, M=2, w=P, ldw=64, sw=P, N=8, K=64, out=P, dtype=1, ldo=8):
        return L.tfe_matmul_fp8(a, lda, sa, M, w, ldw, sw, N, K, out, dtype, ldo, None)

    for kw in (dict(a=None), dict(a=P + 8), dict(lda=63), dict(lda=72), dict(lda=1 << 40), dict(sa=None), dict(sa=P + 2), dict(M=-1),
               dict(M=tfe.ROWS_MAX + 1), dict(w=None), dict(w=P + 4), dict(ldw=48), dict(ldw=65), dict(sw=None), dict(sw=P + 1), dict(N=0),
               dict(N=tfe.ROWS_MAX + 1, ldo=1 << 30), dict(K=0), dict(K=65), dict(K=tfe.FP8_MAX_COLS + 1, lda=1 << 20, ldw=1 << 20),
               dict(out=None), dict(out=P + 2), dict(dtype=2), dict(dtype=-1), dict(ldo=7), dict(ldo=1 << 40)):
        assert product(**kw) == tfe.TFE_ERR_INVALID_ARG, kw
    assert product(M=0, a=None, sa=None, w=None, sw=None, out=None) == tfe.TFE_OK
    assert L.tfe_matmul_fp8_status(None, None) == tfe.TFE_ERR_INVALID_ARG
    assert L.tfe_matmul_fp8_status.argtypes[0] == C.POINTER(C.c_uint32)


def test_sizes_beyond_32_bits():
    """The library takes 32-bit sizes, and a call through ctypes cuts larger ones down without a word: the package refuses them."""
    import ctypes as C
    from types import SimpleNamespace

    import torch

    from paper_2607_07388_b200 import engine
    assert C.c_int32((1 << 32) + 5).value == 5

    def matrix(rows, cols, dtype):                  # no such memory is needed: sizes are looked at first
        return SimpleNamespace(dtype=dtype, is_cuda=True, shape=(rows, cols), dim=lambda: 2, stride=lambda: (cols, 1), data_ptr=lambda: P)

    for rows, cols in (((1 << 32) + 5, 16), (1 << 31, 16), (1, (1 << 32) + 16), (3, 1 << 31)):
        with pytest.raises(ValueError):
            engine._row_matrix(matrix(rows, cols, torch.bfloat16), "x")
        with pytest.raises(ValueError):
            engine._fp8_matrix(matrix(rows, cols, torch.float8_e4m3fn), "a")
    assert engine._row_matrix(matrix((1 << 31) - 1, 16, torch.float32), "x") == ((1 << 31) - 1, 16, 16, engine.tfe.DTYPE_F32)
    assert engine._fp8_matrix(matrix((1 << 31) - 1, 16, torch.float8_e4m3fn), "a") == ((1 << 31) - 1, 16, 16)


def test_gradient_on_its_other_operands_is_refused(tfe):
    """A gradient that would be written over the teacher's entries, the log-sum-exps or the incoming gradient."""
    L, Q = tfe.lib(), 16 * P

    def backward(ids=P, t=2 * P, lse=3 * P, g=4 * P, grad=Q, V=8):
        return L.tfe_distill_backward(5 * P, 1, 2, V, V, ids, t, 4, 1.0, lse, g, grad, V, None)

    for name, size in (("ids", 32), ("t", 32), ("lse", 8), ("g", 8)):
        for at in (Q, Q + 60, Q - size + 4):
            assert backward(**{name: at}) == tfe.TFE_ERR_INVALID_ARG, (name, at)


def test_conversion_into_rows_apart(tfe):
    L = tfe.lib()
    for ldq in (7, 0, -8, (1 << 34) + 1):
        assert L.tfe_quantize_fp8_ld(P, 1, 2, 8, 8, 1, P, ldq, P, None) == tfe.TFE_ERR_INVALID_ARG
    assert L.tfe_quantize_fp8_ld(None, 1, 0, 8, 8, 1, None, 16, None, None) == tfe.TFE_OK
