"""Layer norm, forward and backward, through the C ABI on the GPU, against the formulas in 64 bits.

Tolerances.  A result is rounded once to 16 bits: half a step, eps/2 relative.  What is in front of that is fp32: a sum of n values
whose longest chain of additions is `depth` is off by at most depth * 2^-24 * sum|values|, and every further operation by 2^-24 of its
result.  `depth` counts the chain of the longest kernel for that size (a thread's own values, then the tree across threads)."""
import itertools

import pytest
import torch

from paper_2008_13006_amd import binding as tw

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
TYPES = {"f16": torch.float16, "bf16": torch.bfloat16}


def half_step(t):
    return torch.finfo(t).eps / 2


def depth(n):
    """Additions in a chain over n values: at most 64 of a thread's own in registers or n / 256 in a loop, ten levels of a tree."""
    return max(64, -(-n // 256)) + 10


def tiny(t):
    """Results below the type's smallest normal number are off by half of its smallest step."""
    return torch.finfo(t).smallest_normal * torch.finfo(t).eps / 2


def make(M, N, dtype, pitch=8, offset=0, gen=None, scale=1.0, shift=0.0):
    """An M x N matrix inside a larger buffer of a known pattern, pitch a multiple of `pitch`, base `offset` elements off."""
    ld = -(-N // pitch) * pitch
    buf = torch.full((M * ld + offset + 64,), 7.0, dtype=dtype, device="cuda")
    m = buf[offset:offset + M * ld].view(M, ld)[:, :N]
    if gen is not None:
        m.copy_(torch.randn((M, N), generator=gen, device="cuda") * scale + shift)
    return m, buf


def check_rest(buf, m):
    """Nothing of the buffer outside the matrix was written."""
    M, N = m.shape
    off = m.storage_offset()
    ld = m.stride(0) if M > 1 else N
    mask = torch.ones(buf.numel(), dtype=torch.bool, device="cuda")
    idx = off + torch.arange(M, device="cuda")[:, None] * ld + torch.arange(N, device="cuda")
    mask[idx.flatten()] = False
    assert bool((buf[mask] == 7.0).all()), "wrote outside the matrix"


def reference(x, gamma, beta, eps):
    x = x.double()
    mean = x.mean(1, keepdim=True)
    var = (x - mean).square().mean(1, keepdim=True)
    rstd = 1.0 / torch.sqrt(var + eps)
    g = gamma.double() if gamma is not None else torch.ones(x.shape[1], device="cuda", dtype=torch.float64)
    b = beta.double() if beta is not None else torch.zeros(x.shape[1], device="cuda", dtype=torch.float64)
    return (x - mean) * rstd * g + b, mean[:, 0], rstd[:, 0], g, b


def check_forward(y, mean, rstd, x, gamma, beta, eps):
    want, m64, r64, g, b = reference(x, gamma, beta, eps)
    x64, c = x.double(), depth(x.shape[1]) + 8
    d_mean = c * U * x64.abs().mean(1)                          # error of the mean, and with it of x - mean
    # relative error of 1 / sqrt(var + eps): half of that of var + eps, which has the chain's and what the mean's error adds
    r_var = c * U + 2 * d_mean * r64 + (d_mean * r64).square()
    d_rstd = r_var + 4 * U
    if mean is not None:
        assert bool(((mean.double() - m64).abs() <= d_mean + 1e-37).all())
        assert bool(((rstd.double() - r64).abs() <= d_rstd * r64).all())
    xh = ((x64 - m64[:, None]) * r64[:, None]).abs()
    fp32 = g.abs() * (xh * (d_rstd + 4 * U)[:, None] + (d_mean * r64)[:, None]) + 2 * U * (want.abs() + b.abs())
    bound = half_step(y.dtype) * (want.abs() + fp32) + fp32 + tiny(y.dtype)
    worst = ((y.double() - want).abs() / bound).max().item()
    assert worst <= 1.0, worst


SIZES = [(1, 1), (3, 2), (1, 7), (5, 8), (2, 64), (33, 100), (17, 128), (9, 129), (70, 256), (31, 257), (13, 511), (64, 768), (130, 1000),
         (7, 1025), (5, 1543), (4, 2048), (3, 2049), (6, 4095), (2, 5000), (3, 8200), (2, 16384), (2, 16385)]


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("M,N", SIZES)
def test_rows(M, N, dtype):
    gen = torch.Generator(device="cuda").manual_seed(M * 65537 + N)
    t = TYPES[dtype]
    x, _ = make(M, N, t, gen=gen, scale=1.5, shift=0.7)
    gamma = (1 + 0.2 * torch.randn(N, generator=gen, device="cuda")).to(t)
    beta = (0.2 * torch.randn(N, generator=gen, device="cuda")).to(t)
    for with_g, with_b, stats in ((True, True, True), (False, False, False), (True, False, True), (False, True, False)):
        y, buf = make(M, N, t)
        mean, rstd = (torch.empty(M, device="cuda") for _ in range(2)) if stats else (None, None)
        g, b = gamma if with_g else None, beta if with_b else None
        assert tw.tw_layernorm(x, g, b, 1e-5, y, mean, rstd) is y
        check_forward(y, mean, rstd, x, g, b, 1e-5)
        check_rest(buf, y)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("M,N", [(1, 1), (7, 3), (8, 64), (63, 100), (65, 256), (64, 257), (200, 512), (129, 700), (66, 768), (40, 1000), (90, 1025),
                                 (9, 2048), (70, 2049), (1, 3000)])
def test_columns(M, N, dtype):
    gen = torch.Generator(device="cuda").manual_seed(M * 65537 + N + 1)
    t = TYPES[dtype]
    xt, _ = make(N, M, t, gen=gen, scale=1.5, shift=0.7)
    gamma = (1 + 0.2 * torch.randn(N, generator=gen, device="cuda")).to(t)
    beta = (0.2 * torch.randn(N, generator=gen, device="cuda")).to(t)
    for affine in (True, False):
        yt, buf = make(N, M, t)
        mean, rstd = (torch.empty(M, device="cuda") for _ in range(2)) if affine else (None, None)
        g, b = (gamma, beta) if affine else (None, None)
        tw.tw_layernorm_t(xt, g, b, 1e-5, yt, mean, rstd)
        check_forward(yt.t(), mean, rstd, xt.t(), g, b, 1e-5)
        check_rest(buf, yt)


def check_grad(dx, dgamma, dbeta, dy, x, gamma, mean, rstd):
    M, N = x.shape
    g64 = gamma.double() if gamma is not None else torch.ones(N, device="cuda", dtype=torch.float64)
    dy64, r = dy.double(), rstd.double()[:, None]
    xh = (x.double() - mean.double()[:, None]) * r
    g = dy64 * g64
    want = r * (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True))
    c = depth(N) + 8
    fp32 = c * U * r * (g.abs() + g.abs().mean(1, keepdim=True) + xh.abs() * (g * xh).abs().mean(1, keepdim=True))
    bound = half_step(dx.dtype) * (want.abs() + fp32) + fp32 + tiny(dx.dtype)
    assert ((dx.double() - want).abs() / bound).max().item() <= 1.0
    # the rows: at most 512 parts of ceil(M / 512) or 16 rows; a part's own rows one after the other, 16 row groups, 128 parts a wave
    c = max(16, -(-M // 512)) + 16 + 128 + 8
    for got, terms in ((dgamma, dy64 * xh), (dbeta, dy64)):
        bound = c * U * terms.abs().sum(0) + 1e-37
        assert ((got.double() - terms.sum(0)).abs() / bound).max().item() <= 1.0


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("M,N", SIZES + [(300, 96), (1000, 130), (9000, 24), (17000, 8)])
def test_backward(M, N, dtype):
    gen = torch.Generator(device="cuda").manual_seed(M * 65537 + N + 2)
    t = TYPES[dtype]
    x, _ = make(M, N, t, gen=gen, scale=1.5, shift=0.7)
    dy, _ = make(M, N, t, gen=gen)
    gamma = (1 + 0.2 * torch.randn(N, generator=gen, device="cuda")).to(t)
    mean, rstd = (torch.empty(M, device="cuda") for _ in range(2))
    tw.tw_layernorm(x, None, None, 1e-5, None, mean, rstd)
    for g in (gamma, None):
        dx, buf = make(M, N, t)
        out = tw.tw_layernorm_grad(dy, x, g, mean, rstd, dx)
        check_grad(*out, dy, x, g, mean, rstd)
        check_rest(buf, dx)
        again = tw.tw_layernorm_grad(dy, x, g, mean, rstd)
        assert all(torch.equal(a, b) for a, b in zip(out, again))


@pytest.mark.parametrize("pitch,offset", [(1, 0), (8, 1), (8, 4), (3, 2)])
def test_pitches_and_alignment(pitch, offset):
    """Pitches that are no multiple of 8 and bases off 16 bytes, of each operand in turn."""
    gen = torch.Generator(device="cuda").manual_seed(5)
    t = torch.bfloat16
    for M, N, which in itertools.product((5,), (37, 300, 2500), range(3)):
        def mk(k, **kw):
            return make(M, N, t, pitch if k == which else 8, offset if k == which else 0, **kw)
        x, _ = mk(0, gen=gen)
        dy, _ = mk(1, gen=gen)
        gbuf = torch.randn(N + 8, generator=gen, device="cuda").to(t)
        gamma, beta = gbuf[offset % 8:offset % 8 + N], gbuf[:N]
        y, buf = mk(2)
        mean, rstd = (torch.empty(M, device="cuda") for _ in range(2))
        tw.tw_layernorm(x, gamma, beta, 1e-5, y, mean, rstd)
        check_forward(y, mean, rstd, x, gamma, beta, 1e-5)
        check_rest(buf, y)
        dx, buf = mk(2)
        check_grad(*tw.tw_layernorm_grad(dy, x, gamma, mean, rstd, dx), dy, x, gamma, mean, rstd)
        check_rest(buf, dx)
        xt, _ = make(N, M, t, pitch if which == 0 else 8, offset if which == 0 else 0, gen=gen)
        yt, buf = make(N, M, t, pitch if which == 2 else 8, offset if which == 2 else 0)
        tw.tw_layernorm_t(xt, gamma, beta, 1e-5, yt, mean, rstd)
        check_forward(yt.t(), mean, rstd, xt.t(), gamma, beta, 1e-5)
        check_rest(buf, yt)


@pytest.mark.parametrize("N,pitch", [(96, 8), (768, 8), (3000, 8), (100, 1)])
def test_in_place(N, pitch):
    gen = torch.Generator(device="cuda").manual_seed(N)
    t, M = torch.float16, 37
    x, _ = make(M, N, t, pitch, gen=gen)
    dy, _ = make(M, N, t, pitch, gen=gen)
    mean, rstd = (torch.empty(M, device="cuda") for _ in range(2))
    y = tw.tw_layernorm(x, None, None, 1e-5, None, mean, rstd)
    dx, dgamma, dbeta = tw.tw_layernorm_grad(dy, x, None, mean, rstd)
    for target in ("dy", "x"):
        a, b = dy.clone(memory_format=torch.preserve_format), x.clone(memory_format=torch.preserve_format)
        got = tw.tw_layernorm_grad(a, b, None, mean, rstd, a if target == "dy" else b)
        assert torch.equal(got[0], dx) and torch.equal(got[1], dgamma) and torch.equal(got[2], dbeta)
    tw.tw_layernorm(x, None, None, 1e-5, x)
    assert torch.equal(x, y)
    xt, _ = make(N, M, t, pitch, gen=gen)
    yt = tw.tw_layernorm_t(xt)
    tw.tw_layernorm_t(xt, Yt=xt)
    assert torch.equal(xt, yt)


def test_values_at_the_edge():
    """Rows that are constant, that hold the type's largest values, a mean far from zero, and rows with inf or NaN: those stay theirs."""
    for t in TYPES.values():
        N = 200
        big = torch.finfo(t).max
        x = torch.randn((8, N), device="cuda").to(t)
        x[0] = 3.0
        x[1] = 0.0
        x[2] = 1000.0 + torch.arange(N, device="cuda").to(t) % 2 * 8
        x[3, ::2], x[3, 1::2] = (big, -big) if t == torch.float16 else (2.0 ** 60, -2.0 ** 60)
        x[4, 5], x[5, 7] = float("inf"), float("nan")
        clean = [0, 1, 2, 3, 6, 7]
        ln = (tw.tw_layernorm(x), tw.tw_layernorm_t(x.t().contiguous()).t())
        for y in ln:
            assert bool((y[:2] == 0).all())
            assert bool(torch.isnan(y[4]).any()) and bool(torch.isnan(y[5]).all())
            check_forward(y[clean], None, None, x[clean], None, None, 1e-5)


def test_gradient_against_differences():
    """The derivative of sum(w * y) along a direction, by central differences of the formula in 64 bits."""
    gen = torch.Generator(device="cuda").manual_seed(11)
    M, N, t = 6, 72, torch.bfloat16
    x, w = (torch.randn((M, N), generator=gen, device="cuda").to(t) for _ in range(2))
    gamma = (1 + 0.3 * torch.randn(N, generator=gen, device="cuda")).to(t)
    beta = torch.zeros(N, dtype=t, device="cuda")
    mean, rstd = (torch.empty(M, device="cuda") for _ in range(2))
    tw.tw_layernorm(x, gamma, beta, 1e-5, None, mean, rstd)
    dx, dgamma, dbeta = tw.tw_layernorm_grad(w, x, gamma, mean, rstd)

    def loss(x_, g_, b_):
        return (w.double() * reference(x_, g_, b_, 1e-5)[0]).sum()

    h = 1e-5
    for got, which in ((dx, 0), (dgamma, 1), (dbeta, 2)):
        for k in range(3):
            args = [x.double(), gamma.double(), beta.double()]
            v = torch.randn(args[which].shape, generator=gen, device="cuda", dtype=torch.float64)
            ends = []
            for s in (1, -1):
                moved = list(args)
                moved[which] = args[which] + s * h * v
                ends.append(loss(*moved))
            num = (ends[0] - ends[1]) / (2 * h)
            ana = (got.double() * v).sum()
            # every element of dx is off by half a step of 16 bits at most; differences by h^2 and 64-bit rounding over h
            bound = (half_step(t) if which == 0 else 1e-5) * (got.double() * v).abs().sum() + 1e-5 * (1 + num.abs())
            assert (num - ana).abs() <= bound


def test_streams_and_graphs():
    """A call on another stream than the current one, and forward and backward captured into one graph, replayed on new data with
    eager work between."""
    gen = torch.Generator(device="cuda").manual_seed(3)
    M, N, t = 500, 768, torch.float16
    x, dy = (torch.randn((M, N), generator=gen, device="cuda").to(t) for _ in range(2))
    gamma, beta = torch.ones(N, dtype=t, device="cuda"), torch.zeros(N, dtype=t, device="cuda")
    y, dx = torch.empty_like(x), torch.empty_like(x)
    mean, rstd = (torch.empty(M, device="cuda") for _ in range(2))
    dgamma, dbeta = (torch.empty(N, device="cuda") for _ in range(2))

    def both(stream=None):
        tw.tw_layernorm(x, gamma, beta, 1e-5, y, mean, rstd, stream=stream)
        tw.tw_layernorm_grad(dy, x, gamma, mean, rstd, dx, dgamma, dbeta, stream=stream)

    both()
    want = [v.clone() for v in (y, dx, dgamma, dbeta)]
    side = torch.cuda.Stream()
    for v in (y, dx, dgamma, dbeta):
        v.zero_()
    side.wait_stream(torch.cuda.current_stream())
    both(side)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip((y, dx, dgamma, dbeta), want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for k in range(4):
        x.copy_(torch.randn((M, N), generator=gen, device="cuda") * (k + 1))
        graph.replay()
        torch.cuda.synchronize()
        got = [v.clone() for v in (y, dx, dgamma, dbeta)]
        both()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((y, dx, dgamma, dbeta), got))


def both_boundaries(x, gamma, beta, aligned=True):
    """(y, mean, rstd, c) row-major and from the transposed boundary, by the kernels for aligned operands or by those for any.  c: the length
    of the chain of additions in a sum, and a few operations beside it.  Columns of any alignment: a thread adds every 16th value, then 16
    threads' sums are added; aligned ones beyond 2048: every 128th, three levels of a tree, 16 sums."""
    M, N = x.shape
    for transposed in (False, True):
        src = x.t() if transposed else x
        a, _ = make(*src.shape, x.dtype, 8, 0 if aligned else 1)
        a.copy_(src)
        y, _ = make(*src.shape, x.dtype)
        mean, rstd = (torch.empty(M, device="cuda") for _ in range(2))
        (tw.tw_layernorm_t if transposed else tw.tw_layernorm)(a, gamma, beta, 1e-5, y, mean, rstd)
        c = max(depth(N), (-(-N // 128) + 3 if aligned else -(-N // 16)) + 16) if transposed else depth(N)
        yield y.t() if transposed else y, mean, rstd, c + 8


@pytest.mark.parametrize("aligned", [True, False])
@pytest.mark.parametrize("N", [7, 100, 1000, 1792, 2047, 3584, 5001, 20001])
def test_constant_rows(N, aligned):
    """Every element is its row's mean: what is left is the offset, whatever the value, its size and the number of features.  (A step of fp32 at
    60000 is 0.004, and 1 / sqrt(eps) makes 1.2 of it.)"""
    gen = torch.Generator(device="cuda").manual_seed(N)
    for t, values in ((torch.float16, (60000.0, -65504.0, 2049.0 * 16, 0.1, 1027.0)), (torch.bfloat16, (60000.0, -1e20, 129.0 * 512, 3.3))):
        x = torch.tensor(values, device="cuda").to(t)[:, None].expand(-1, N).contiguous()
        gamma = (1 + 0.2 * torch.randn(N, generator=gen, device="cuda")).to(t)
        beta = (0.5 + torch.rand(N, generator=gen, device="cuda")).to(t)
        for y, mean, rstd, c in both_boundaries(x, gamma, beta, aligned):
            assert torch.equal(y, beta.expand_as(y))
            assert torch.equal(mean, x[:, 0].float())
            # 1 / sqrt(eps) with eps in 32 bits: the root and the quotient are off by half a step each.  Up to 8192 features the sums of a constant
            # are exact (13 + 11 bits); beyond, the first mean may be off by c U |x|, and c U of that squared is left of the variance
            off = 0 if N <= 8192 else c * U * x[:, 0].double().abs()
            assert bool(((rstd.double() * 1e-5 ** 0.5 - 1).abs() <= 4 * U + 0.5 * c * U * off ** 2 / 1e-5).all())


@pytest.mark.parametrize("aligned", [True, False])
@pytest.mark.parametrize("N", [100, 1000, 1792, 3001, 20001])
def test_rows_that_hardly_vary(N, aligned):
    """A few elements one step beside a large common value: the mean's rounding to fp32 must not show in what is normalised.

    The first mean is off by c U mean|x| at most, c the length of the chain of sums.  x less that is exact (the two lie within a factor of two);
    its own mean is a sum of values of the size of mean|x - mean| + that error, and off by c U of it; the variance by c U of
    var + error^2 and twice the product of the two errors."""
    gen = torch.Generator(device="cuda").manual_seed(N)
    for t, value, step in ((torch.float16, 60000.0, 32.0), (torch.float16, -1500.0, 1.0), (torch.bfloat16, 60160.0, 256.0)):
        x = torch.full((4, N), value, device="cuda")
        for m, k in enumerate((1, 3, N // 10, N // 2)):
            x[m, torch.randperm(N, generator=gen, device="cuda")[:k]] += step
        x = x.to(t)
        want, m64, r64, _, _ = reference(x, None, None, 1e-5)
        x64 = x.double()
        off = (x64 - m64[:, None]).abs()
        for y, mean, rstd, c in both_boundaries(x, None, None, aligned):
            first = c * U * x64.abs().mean(1)
            second = c * U * (off.mean(1) + first)                      # error of x - mean, beside its own rounding
            d_rstd = 0.5 * (c + 4) * U * (1 + 2 * (first * r64).square()) + first * second * r64.square() + 4 * U
            fp32 = ((off * r64[:, None]) * (d_rstd + 4 * U)[:, None] + (second * r64)[:, None])
            bound = half_step(t) * (want.abs() + fp32) + fp32 + tiny(t)
            assert ((y.double() - want).abs() / bound).max().item() <= 1.0
            assert bool(((rstd.double() - r64).abs() <= d_rstd * r64).all())
            assert bool(((mean.double() - m64).abs() <= second + U * m64.abs()).all())


def test_rows_of_a_default_output_start_lines():
    """What tw_layernorm_t allocates has the pitch that whole lines are stored with; what it leaves is what an output of another pitch gets."""
    for M in (8, 63, 64, 200):
        xt = torch.randn((96, M), device="cuda").to(torch.float16)
        yt = tw.tw_layernorm_t(xt)
        assert yt.shape == (96, M) and yt.stride(1) == 1 and yt.stride(0) == -(-M // 64) * 64 and yt.data_ptr() % 128 == 0
        other, _ = make(96, M, torch.float16)
        assert torch.equal(tw.tw_layernorm_t(xt, Yt=other), yt)


@pytest.mark.parametrize("aligned", [True, False])
@pytest.mark.parametrize("N", [64, 1000, 2500])
def test_statistics_of_rows_that_are_not_finite(N, aligned):
    """The mean of a row with an infinity is that infinity, of one with both or with NaN it is NaN; its deviation is NaN."""
    for t in TYPES.values():
        x = torch.randn((6, N), device="cuda").to(t)
        x[0, 3], x[1, N - 1], x[2, 5] = float("inf"), float("-inf"), float("nan")
        x[3, 1], x[3, 2] = float("inf"), float("-inf")
        want = x.double().mean(1)
        for y, mean, rstd, c in both_boundaries(x, None, None, aligned):
            assert bool(((mean[:2] == want[:2].float()) & torch.isinf(mean[:2])).all()) and bool(torch.isnan(mean[2:4]).all())
            assert bool(torch.isnan(rstd[:4]).all()) and bool(torch.isfinite(rstd[4:]).all()) and bool(torch.isfinite(mean[4:]).all())
