"""What the entry points between the products refuse, and what they take without a GPU call: no GPU needed, nothing is launched."""
import ctypes

import pytest
import torch

from paper_2008_13006_amd import binding as tw

# The pointers are made up: a library older than a refusal below would launch a kernel on them, so this file runs only where nothing can be launched.
pytestmark = pytest.mark.skipif(torch.cuda.device_count() > 0, reason="made-up device pointers: only on machines without a GPU")
ARG, BUF, ALIGN, UNSUPPORTED = -1, -3, -4, -6
P = 0x10000          # stands for a device pointer: checked, never read (every call below ends before a launch)


def ln(entry="tw_layernorm", X=P, ld=64, M=4, N=64, gamma=P, beta=P, eps=1e-5, Y=P, ldy=64, mean=None, rstd=None, dt=0):
    return getattr(tw._lib, entry)(X, ld, M, N, gamma, beta, eps, Y, ldy, mean, rstd, dt, None)


@pytest.mark.parametrize("entry", ["tw_layernorm", "tw_layernorm_t"])
def test_layernorm_refusals(entry):
    wide = dict(M=64, N=4) if entry == "tw_layernorm_t" else {}
    bad = [(dict(X=None), ARG), (dict(Y=None), ARG), (dict(M=-1), ARG), (dict(N=0), ARG), (dict(N=-3), ARG), (dict(ld=63), ARG), (dict(ldy=63), ARG),
           (dict(dt=2), ARG), (dict(dt=-1), ARG), (dict(eps=-1e-9), ARG), (dict(eps=float("nan")), ARG), (dict(eps=float("inf")), ARG),
           (dict(X=P + 1), ALIGN), (dict(Y=P + 1), ALIGN), (dict(gamma=P + 1), ALIGN), (dict(beta=P + 1), ALIGN), (dict(mean=P + 2), ALIGN),
           (dict(rstd=P + 1), ALIGN)]
    for kw, want in bad:
        if entry == "tw_layernorm_t" and "N" not in kw:
            kw = {**wide, **kw}
        assert ln(entry, **kw) == want, kw
    assert ln(entry, N=1 << 24, ld=1 << 24, ldy=1 << 24) == UNSUPPORTED
    assert ln(entry, M=0, X=None, Y=None) == 0
    if entry == "tw_layernorm_t":
        assert ln(entry, M=(1 << 28) + 1, N=1, ld=1 << 29, ldy=1 << 29) == UNSUPPORTED


def grad(dY=P, lddy=64, X=P, ldx=64, M=4, N=64, gamma=P, mean=P, rstd=P, dX=P, lddx=64, dgamma=None, dbeta=None, ws=P, nbytes=None, dt=0):
    if nbytes is None:
        nbytes = tw.tw_layernorm_grad_workspace(max(M, 0), max(N, 1))
    return tw._lib.tw_layernorm_grad(dY, lddy, X, ldx, M, N, gamma, mean, rstd, dX, lddx, dgamma, dbeta, ws, nbytes, dt, None)


def test_layernorm_grad_refusals():
    for kw, want in [(dict(dY=None), ARG), (dict(X=None), ARG), (dict(mean=None), ARG), (dict(rstd=None), ARG), (dict(dX=None), ARG), (dict(ws=None), ARG),
                     (dict(M=-1), ARG), (dict(N=0), ARG), (dict(dt=7), ARG), (dict(lddy=63), ARG), (dict(ldx=63), ARG), (dict(lddx=63), ARG),
                     (dict(dY=P + 1), ALIGN), (dict(X=P + 1), ALIGN), (dict(dX=P + 1), ALIGN), (dict(gamma=P + 1), ALIGN), (dict(mean=P + 2), ALIGN),
                     (dict(rstd=P + 2), ALIGN), (dict(dgamma=P + 2), ALIGN), (dict(dbeta=P + 1), ALIGN), (dict(ws=P + 8), ALIGN),
                     (dict(nbytes=tw.tw_layernorm_grad_workspace(4, 64) - 1), BUF),
                     (dict(N=1 << 24, lddy=1 << 24, ldx=1 << 24, lddx=1 << 24), UNSUPPORTED)]:
        assert grad(**kw) == want, kw
    assert grad(M=0, dY=None, X=None, mean=None, rstd=None, dX=None, ws=None, nbytes=0) == 0   # (no sums wanted: nothing to do)
    n = ctypes.c_size_t(0)
    for args, want in [((-1, 4), ARG), ((4, 0), ARG)]:
        assert tw._lib.tw_layernorm_grad_workspace(*args, ctypes.byref(n)) == want
    assert tw._lib.tw_layernorm_grad_workspace(4, 4, None) == ARG
    # room for the sums of at most 512 groups of rows and two numbers a row
    assert tw.tw_layernorm_grad_workspace(1, 5) == 4 * (2 * 5 + 2) and tw.tw_layernorm_grad_workspace(10 ** 6, 768) == 4 * (1024 * 768 + 2 * 10 ** 6)


def test_layernorm_grad_workspace_of_very_many_rows():
    rows = 2 ** 31 - 1
    assert tw.tw_layernorm_grad_workspace(rows, 8) == 4 * (512 * 2 * 8 + 2 * rows)


def attention(Q=P, ldq=128, K=P, ldk=64, V=P, ldv=64, O=P, ldo=128, M=4, seq_start=P, n_seqs=1, heads=2, kv_heads=1, d=64, scale=0.125, causal=1, dt=0):
    return tw._lib.tw_attention(Q, ldq, K, ldk, V, ldv, O, ldo, M, seq_start, n_seqs, heads, kv_heads, d, scale, causal, dt, None)


def test_attention_refusals():
    for kw, want in [(dict(Q=None), ARG), (dict(K=None), ARG), (dict(V=None), ARG), (dict(O=None), ARG), (dict(M=-1), ARG), (dict(n_seqs=-1), ARG),
                     (dict(heads=0), ARG), (dict(kv_heads=0), ARG), (dict(heads=3, kv_heads=2, ldq=192, ldo=192, ldk=128, ldv=128), ARG), (dict(d=0), ARG),
                     (dict(dt=2), ARG), (dict(scale=-1.0), ARG), (dict(scale=float("nan")), ARG), (dict(scale=float("inf")), ARG),
                     (dict(seq_start=None, n_seqs=2), ARG), (dict(ldq=120), ARG), (dict(ldk=56), ARG), (dict(ldv=56), ARG), (dict(ldo=120), ARG),
                     (dict(d=136, ldq=272, ldk=136, ldv=136, ldo=272), UNSUPPORTED), (dict(d=60), UNSUPPORTED), (dict(ldq=130), ALIGN), (dict(ldk=68), ALIGN),
                     (dict(ldv=68), ALIGN), (dict(ldo=132), ALIGN), (dict(Q=P + 8), ALIGN), (dict(K=P + 2), ALIGN), (dict(V=P + 4), ALIGN),
                     (dict(O=P + 8), ALIGN), (dict(seq_start=P + 2), ALIGN), (dict(ldk=1 << 24), UNSUPPORTED), (dict(ldv=1 << 24), UNSUPPORTED),
                     (dict(M=1 << 30), UNSUPPORTED)]:
        assert attention(**kw) == want, kw
    assert attention(M=0, Q=None, K=None, V=None, O=None) == 0
    assert attention(n_seqs=0) == 0                              # no sequence, no row


def test_attention_scale_out_of_range():
    # the kernel multiplies by scale * log2 e, which has to be finite as well
    assert attention(scale=3e38) == UNSUPPORTED
    assert attention(scale=2.3e38, M=0) == 0


def test_add_refusals():
    """The products that add a matrix: what they refuse beyond what the products without it do."""
    import numpy as np
    blob = tw.tw_pack(np.zeros((64, 96), np.uint16), np.ones((64, 96), np.uint8), 32, "f16")
    tew = tw.tw_pack_tew(np.zeros((64, 96), np.uint16), np.r_[np.ones((63, 96), np.uint8), np.zeros((1, 96), np.uint8)] * (np.arange(96) > 0).astype(np.uint8),
                         np.ones((64, 96), np.uint8), 32, "f16")
    Q = 2 * P

    def row(blob=blob, dev=P, A=P, M=4, lda=64, bias=None, act=0, R=P, ldr=96, C=Q, ldc=96, ws=P, n=256):
        return tw._lib.tw_gemm_bias_act_add(blob.ctypes.data, dev, A, M, lda, bias, act, R, ldr, C, ldc, ws, n, None)

    def col(blob=blob, dev=P, A=P, M=8, lda=8, bias=None, act=0, R=P, ldr=8, C=Q, ldc=8, ws=P, n=256):
        return tw._lib.tw_gemm_t_bias_act_add(blob.ctypes.data, dev, A, M, lda, bias, act, R, ldr, C, ldc, ws, n, None)

    def dense(A=P, lda=64, B=P, ldb=96, bias=None, act=0, R=P, ldr=96, C=Q, ldc=96, M=4, N=96, K=64, dt=0):
        return tw._lib.tw_dense_gemm_bias_act_add(A, lda, B, ldb, bias, act, R, ldr, C, ldc, M, N, K, dt, None)

    for kw, want in [(dict(R=None), ARG), (dict(ldr=95), ARG), (dict(R=P + 1), ALIGN), (dict(R=Q, ldr=104), ARG),
                     (dict(A=None), ARG), (dict(C=None), ARG), (dict(act=3), ARG), (dict(bias=P + 1), ALIGN), (dict(lda=56), ARG), (dict(lda=68), ALIGN),
                     (dict(ldc=95), ARG), (dict(M=-1), ARG), (dict(n=255), BUF), (dict(ws=P + 16), ALIGN), (dict(blob=tew, R=Q), UNSUPPORTED)]:
        assert row(**kw) == want, kw
    for kw, want in [(dict(R=None), ARG), (dict(ldr=7), ARG), (dict(ldr=12), ALIGN), (dict(R=P + 8), ALIGN), (dict(R=Q, ldr=16), ARG), (dict(A=None), ARG),
                     (dict(act=-1), ARG), (dict(ldc=12), ALIGN), (dict(lda=0), ARG), (dict(n=0), BUF), (dict(blob=tew, R=Q), UNSUPPORTED)]:
        assert col(**kw) == want, kw
    for kw, want in [(dict(R=None), ARG), (dict(ldr=88), ARG), (dict(ldr=100), ALIGN), (dict(R=P + 8), ALIGN), (dict(R=Q, ldr=104), ARG), (dict(A=None), ARG),
                     (dict(dt=2), ARG), (dict(act=9), ARG), (dict(K=0), ARG), (dict(M=-1), ARG)]:
        assert dense(**kw) == want, kw
    assert row(M=0) == 0 and col(M=0) == 0 and dense(M=0) == 0


def test_sizes_beyond_32_bits_are_not_cut():
    class Operand:                                               # what the binding looks at
        is_cuda, dtype = True, torch.float16

        def __init__(self, rows, cols, ld):
            self.shape, self.ld = (rows, cols), ld

        def get_device(self):
            return 0

        def stride(self):
            return self.ld, 1

    for rows, cols, ld in [(2 ** 32 + 4, 8, 8), (4, 8, 2 ** 32 + 8), (4, 2 ** 31 + 8, 2 ** 31 + 8)]:
        with pytest.raises(AssertionError):
            tw._matrix(Operand(rows, cols, ld), rows, cols, Operand(rows, cols, ld))
    assert tw._matrix(Operand(4, 8, 2 ** 31 - 8), 4, 8, Operand(4, 8, 8)) == 2 ** 31 - 8


def test_in_place_means_the_same_pitch():
    """A result that starts where an operand does and has another pitch would be written over rows that are still to be read."""
    assert ln(ldy=72) == ARG and ln(ld=72) == ARG
    assert ln("tw_layernorm_t", M=64, N=4, ldy=72) == ARG and ln("tw_layernorm_t", M=64, N=4, ld=128) == ARG
    other = dict(X=2 * P, dX=3 * P)
    assert grad(lddx=72) == ARG and grad(lddy=72, X=2 * P) == ARG and grad(ldx=128, dY=2 * P) == ARG
    assert grad(lddx=72, **{**other, "dX": P}) == ARG and grad(lddx=72, dY=2 * P) == ARG
    assert attention(O=P, ldo=136) == ARG and attention(Q=P, ldq=256) == ARG
    # one row has no pitch, no row nothing to write
    for call in (lambda **kw: ln(ldy=72, **kw), lambda **kw: grad(lddx=72, **kw), lambda **kw: attention(ldo=136, **kw)):
        assert call(M=1) != ARG and call(M=0) == 0
    assert ln("tw_layernorm_t", M=64, N=1, ldy=72) != ARG and ln("tw_layernorm_t", M=0, N=4, ldy=72) == 0


def test_operands_and_stream_of_another_device(monkeypatch):
    """The library launches on the current device: operands or a stream of another one are refused before it is called."""
    from types import SimpleNamespace
    import numpy as np

    class Operand:
        is_cuda = True

        def __init__(self, *shape, dtype=torch.float16):
            self.shape, self.dtype, self.device = shape, dtype, "cuda:1"

        def get_device(self):
            return 1

        def dim(self):
            return len(self.shape)

        def numel(self):
            return int(np.prod(self.shape))

        def is_contiguous(self):
            return True

        def stride(self, k=None):
            steps = (self.shape[1], 1) if len(self.shape) == 2 else (1,)
            return steps if k is None else steps[k]

        def data_ptr(self):
            return P

    x, seq, f = Operand(64, 64), Operand(2, dtype=torch.int32), Operand(64, dtype=torch.float32)
    w = SimpleNamespace(info={"K": 64, "N": 64}, torch_dtype=torch.float16, workspace_for=lambda M, stream=None: (P, 256), _blob_ptr=P, blob_dev=x)
    calls = [lambda s: tw.tw_gemm_bias_act_add(w, x, x, C=Operand(64, 64), stream=s), lambda s: tw.tw_gemm_t_bias_act_add(w, x, x, Ct=Operand(64, 64), stream=s),
             lambda s: tw.tw_dense_gemm_bias_act_add(x, x, x, C=x, stream=s), lambda s: tw.tw_layernorm(x, Y=x, stream=s), lambda s: tw.tw_layernorm_t(x, Yt=x, stream=s),
             lambda s: tw.tw_layernorm_grad(x, x, None, f, f, x, f, f, Operand(1 << 20, dtype=torch.uint8), stream=s), lambda s: tw.tw_attention(x, x, x, seq, 1, O=x, stream=s)]
    reached = []
    library = SimpleNamespace(**{name: lambda *args, name=name: reached.append(name) or 0 for name in tw.SYMBOLS})
    monkeypatch.setattr(tw, "_lib", library)
    here, there = (SimpleNamespace(cuda_stream=5, device_index=k) for k in (1, 0))
    for k, call in enumerate(calls):
        monkeypatch.setattr(tw, "_current_device", lambda: 0)
        for s in (None, here, there):
            with pytest.raises(AssertionError, match="current device"):
                call(s)
        monkeypatch.setattr(tw, "_current_device", lambda: 1)
        with pytest.raises(AssertionError, match="current device"):
            call(there)
        assert len(reached) == k
        call(here)
        assert len(reached) == k + 1
