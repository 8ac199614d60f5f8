"""Products that add a matrix behind the activation, through the C ABI on the GPU, on every kernel that a call can reach.

Small integers make every product and sum exact, so most comparisons are bit for bit.  Where values are drawn from a normal distribution
the bound of an element is: half a step of the 16-bit result; K + 8 roundings of the fp32 sum, each 2^-24 of sum|a b| (GELU's slope is
below 1.13); GELU's own error (3.3e-7 + 1.2e-7 of the value, as its test holds it to); two roundings of the sum with R."""
import numpy as np
import pytest
import torch

from paper_2008_13006_amd import workloads as W

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.fixture(scope="module")
def tw():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2008_13006_amd import binding
    return binding


def _torch_type(dtype):
    return torch.float16 if dtype == "f16" else torch.bfloat16


def _inside(rows, cols, dtype, pitch, offset=0):
    """A rows x cols matrix inside a buffer of 77s; the buffer too."""
    buf = torch.full((offset + rows * pitch + 16,), 77.0, dtype=_torch_type(dtype), device="cuda")
    return buf[offset:offset + rows * pitch].view(rows, pitch)[:, :cols], buf


def _only_inside(m, buf):
    rest = buf.clone()
    rest.as_strided(m.shape, m.stride(), m.storage_offset()).fill_(77.0)
    return bool((rest == 77.0).all())


def _case(tw, M, K, N, G, dtype, cp, keep, delta=0.0, a_dist="smallint"):
    spec = W.small_spec("add", M=M, K=K, N=N, G=G, dtype=dtype, col_prune=cp, keep=keep, a_dist=a_dist, seed_offset=3100 + M + K + N)
    w = W.generate(spec)
    mask = w.mask
    if delta > 0:
        ew = tw.tw_restore_ew(w.B, w.mask, delta, dtype)
        wt = tw.TwWeight(tw.tw_pack_tew(w.B, w.mask, ew, G, dtype))
        mask = w.mask | ew
    else:
        wt = tw.TwWeight(tw.tw_pack(w.B, w.mask, G, dtype))
    B = tw.bits_to_tensor(w.B, dtype).double() * torch.from_numpy(mask).cuda()
    A = _inside(M, K, dtype, -(-K // 8) * 8)[0]
    A.copy_(tw.bits_to_tensor(w.A, dtype))
    At = _inside(K, M, dtype, -(-M // 8) * 8)[0]
    At.copy_(A.t())
    return wt, A, At, B


def _integers(shape, dtype, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randint(-5, 6, shape, generator=gen, device="cuda").to(_torch_type(dtype))


# M, K, N, G, type, column pruning, keep, residual weights: K resident in blocks of 64 and of 32 rows, lowered blocks, narrow windows, teams of eight,
# four and two waves; spans wider than a window and with more pruned columns than are asked for ahead; K streamed, a wave per tile, sets of four,
# two and one tile, the kernel of TEW blobs; split K, its parts by either kernel; single rows, odd sizes, tiles of every width.
CASES = [
    (1, 771, 520, 128, "bf16", 0.05, ("const", 0.05), 0), (5, 24, 32, 32, "f16", 0.0, ("const", 0.5), 0), (77, 200, 300, 128, "f16", 0.07, ("upow", 0.05, 0.7), 0),
    (16384, 256, 390, 128, "f16", 0.05, ("upow", 0.1, 0.6), 0), (16384, 96, 200, 64, "bf16", 0.1, ("upow", 0.1, 0.5), 0), (17000, 256, 250, 128, "f16", 0.0, ("upow", 0.1, 0.6), 0),
    (150, 256, 384, 128, "f16", 0.05, ("upow", 0.1, 0.6), 0.01), (4321, 1040, 1234, 32, "f16", 0.03, ("upow", 0.05, 0.2), 0), (9000, 1000, 900, 64, "f16", 0.6, ("const", 0.1), 0),
    (12001, 1024, 1300, 128, "f16", 0.7, ("const", 0.1), 0), (90, 256, 1400, 128, "f16", 0.7, ("upow", 0.1, 0.6), 0), (45, 160, 900, 64, "bf16", 0.8, ("upow", 0.1, 0.3), 0),
    (37, 64, 24, 32, "f16", 0.75, ("const", 0.5), 0), (71, 333, 1001, 128, "f16", 0.33, ("upow", 0.05, 0.4), 0.01), (1000, 200, 1200, 128, "f16", 0.06, ("upow", 0.1, 0.6), 0),
    (1000, 500, 700, 64, "bf16", 0.06, ("upow", 0.01, 0.1), 0), (2600, 300, 1200, 128, "bf16", 0.06, ("upow", 0.02, 0.1), 0), (6000, 200, 500, 64, "f16", 0.1, ("upow", 0.1, 0.5), 0.01),
    (16384, 1600, 380, 64, "f16", 0.05, ("upow", 0.02, 0.15), 0), (16400, 1600, 250, 64, "f16", 0.1, ("upow", 0.02, 0.15), 0), (8192, 1700, 256, 64, "f16", 0.1, ("upow", 0.02, 0.15), 0.002),
    (4096, 1600, 128, 32, "f16", 0.0, ("upow", 0.02, 0.15), 0), (16385, 1537, 300, 128, "f16", 0.05, ("upow", 0.02, 0.2), 0), (12000, 2310, 900, 128, "f16", 0.3, ("upow", 0.01, 0.1), 0),
    (1, 2305, 128, 128, "f16", 0.04, ("const", 0.1), 0), (64, 2304, 768, 128, "f16", 0.05, ("upow", 0.02, 0.15), 0), (700, 2000, 300, 64, "bf16", 0.1, ("upow", 0.005, 0.02), 0),
    (1100, 1600, 250, 32, "f16", 0.1, ("upow", 0.02, 0.15), 0), (130, 3100, 300, 128, "f16", 0.3, ("upow", 0.002, 0.2), 0.002), (33, 1800, 1500, 64, "f16", 0.7, ("upow", 0.02, 0.2), 0),
    (20031, 200, 250, 32, "f16", 0.1, ("upow", 0.02, 0.9), 0), (30001, 776, 128, 128, "f16", 0.0, ("const", 0.1), 0), (8190, 3100, 520, 128, "f16", 0.1, ("upow", 0.001, 0.1), 0),
    (2490, 640, 2900, 64, "f16", 0.3, ("upow", 0.05, 0.3), 0),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "x".join(map(str, c[:4])) + "-" + c[4] + ("-tew" if c[7] else ""))
def test_integers_bit_for_bit(tw, case):
    M, K, N, G, dtype, cp, keep, delta = case
    wt, A, At, B = _case(tw, *case)
    print(f"[case] {case} {tw.tw_gemm_plan(wt.blob, M)} / {tw.tw_gemm_plan(wt.blob, M, transposed=True)}", flush=True)
    prod = A.double() @ B
    bias, R = _integers((N,), dtype, 1), _integers((M, N), dtype, 2)
    limit = 2048 if dtype == "f16" else 256
    for b, act in ((None, "none"), (bias, "relu")):
        want = prod if b is None else torch.clamp(prod + b.double(), min=0)
        want = want + R.double()
        assert want.abs().max() <= limit, "the case must stay exactly representable"
        # row-major: a pitch of R that is no multiple of 8 and a base off 16 bytes, C within a buffer
        Rm, _ = _inside(M, N, dtype, N + 3, 1)
        Rm.copy_(R)
        C, cbuf = _inside(M, N, dtype, N + 5, 2)
        assert tw.tw_gemm_bias_act_add(wt, A, Rm, b, act, C) is C
        torch.cuda.synchronize()
        assert torch.equal(C.double(), want) and _only_inside(C, cbuf)
        # whole lines
        C2 = torch.empty((M, -(-N // 64) * 64), dtype=A.dtype, device="cuda")[:, :N]
        tw.tw_gemm_bias_act_add(wt, A, R, b, act, C2)
        torch.cuda.synchronize()
        assert torch.equal(C2.double(), want)
        Rt, _ = _inside(N, M, dtype, -(-M // 8) * 8 + 8, 8)
        Rt.copy_(R.t())
        Ct, cbuf = _inside(N, M, dtype, -(-M // 8) * 8 + 16, 16)
        tw.tw_gemm_t_bias_act_add(wt, At, Rt, b, act, Ct)
        torch.cuda.synchronize()
        assert torch.equal(Ct.double().t(), want) and _only_inside(Ct, cbuf)
        if delta == 0:                                       # added to itself
            tw.tw_gemm_bias_act_add(wt, A, Rm, b, act, Rm)
            tw.tw_gemm_t_bias_act_add(wt, At, Rt, b, act, Rt)
            torch.cuda.synchronize()
            assert torch.equal(Rm.double(), want) and torch.equal(Rt.double().t(), want)
    assert wt.workspace.view(torch.int32)[:4].cpu().tolist() == [0, 0, 0, 0]


def test_split_k_with_a_small_workspace(tw):
    """The counters' 256 bytes only: the same call runs unsplit."""
    case = (64, 2304, 768, 128, "f16", 0.05, ("upow", 0.02, 0.15), 0)
    wt, A, At, B = _case(tw, *case)
    R = _integers((64, 768), "f16", 2)
    assert tw.tw_gemm_plan(wt.blob, 64)["k_parts"] > 1
    want = A.double() @ B + R.double()
    wt.ws_limit = 256
    C, Ct = tw.tw_gemm_bias_act_add(wt, A, R), tw.tw_gemm_t_bias_act_add(wt, At, R.t().contiguous())
    torch.cuda.synchronize()
    assert torch.equal(C.double(), want) and torch.equal(Ct.double().t(), want)


@pytest.mark.parametrize("K", [300, 1536, 1700])
def test_many_residual_weights_in_pruned_columns(tw, K):
    """TEW: more columns per tile that the pattern prunes and the residual restores than a tile adds itself; adding to C itself is refused."""
    M, N = 205, 300
    w = W.generate(W.small_spec("add_xcols", M=M, K=K, N=N, G=64, dtype="f16", col_prune=0.45, keep=("upow", 0.1, 0.4), a_dist="smallint", seed_offset=4242))
    rng = np.random.default_rng(17)
    alive = w.mask.any(axis=0)
    ew = np.zeros_like(w.mask)
    for n in np.flatnonzero(~alive)[::2]:                    # (the others stay pruned)
        ew[rng.choice(K, size=int(rng.integers(1, 12)), replace=False), n] = 1
    ew |= ((rng.random(w.mask.shape) < 0.01) & (w.mask == 0) & alive[None, :]).astype(np.uint8)
    wt = tw.TwWeight(tw.tw_pack_tew(w.B, w.mask, ew, 64, "f16"))
    A = _inside(M, K, "f16", -(-K // 8) * 8)[0]
    A.copy_(tw.bits_to_tensor(w.A, "f16"))
    At = _inside(K, M, "f16", -(-M // 8) * 8)[0]
    At.copy_(A.t())
    bias, R = _integers((N,), "f16", 1), _integers((M, N), "f16", 2)
    want = torch.clamp(A.double() @ (tw.bits_to_tensor(w.B, "f16").double() * torch.from_numpy(w.mask | ew).cuda()) + bias.double(), min=0) + R.double()
    assert want.abs().max() <= 2048
    Rt = _inside(N, M, "f16", 208)[0]
    Rt.copy_(R.t())
    C, Ct = tw.tw_gemm_bias_act_add(wt, A, R, bias, "relu"), tw.tw_gemm_t_bias_act_add(wt, At, Rt, bias, "relu")
    torch.cuda.synchronize()
    assert torch.equal(C.double(), want) and torch.equal(Ct.double().t(), want)
    for call in (lambda: tw.tw_gemm_bias_act_add(wt, A, C, bias, "relu", C), lambda: tw.tw_gemm_t_bias_act_add(wt, At, Rt, bias, "relu", Rt)):
        with pytest.raises(tw.TwError) as e:
            call()
        assert e.value.status == -6


def test_weight_without_columns(tw):
    """No surviving column: act(bias) + R, with and without a bias, and a TEW blob of residual weights alone."""
    M, K, N = 37, 64, 90
    rng = np.random.default_rng(3)
    bits = W.f32_to_bits(rng.integers(-2, 3, (K, N)).astype(np.float32), "f16")
    none = np.zeros((K, N), np.uint8)
    ew = (rng.random((K, N)) < 0.05).astype(np.uint8)
    A = _integers((M, K), "f16", 4)
    At = _inside(K, M, "f16", 40)[0]
    At.copy_(A.t())
    bias, R = _integers((N,), "f16", 5), _integers((M, N), "f16", 6)
    Rt = _inside(N, M, "f16", 40)[0]
    Rt.copy_(R.t())
    B = tw.bits_to_tensor(bits, "f16").double()
    for blob, mask in ((tw.tw_pack(bits, none, 32, "f16"), none), (tw.tw_pack_tew(bits, none, ew, 32, "f16"), ew)):
        wt = tw.TwWeight(blob)
        for b in (bias, None):
            want = A.double() @ (B * torch.from_numpy(mask).cuda())
            want = torch.clamp(want + (b.double() if b is not None else 0), min=0) + R.double()
            C, Ct = tw.tw_gemm_bias_act_add(wt, A, R, b, "relu"), tw.tw_gemm_t_bias_act_add(wt, At, Rt, b, "relu")
            torch.cuda.synchronize()
            assert torch.equal(C.double(), want) and torch.equal(Ct.double().t(), want)


REAL = [(300, 512, 640, 128, "f16", 0.05, ("upow", 0.1, 0.5), 0), (9000, 768, 768, 128, "bf16", 0.05, ("upow", 0.1, 0.5), 0), (200, 2304, 500, 64, "bf16", 0.1, ("upow", 0.05, 0.5), 0),
        (5000, 1900, 300, 128, "f16", 0.1, ("upow", 0.05, 0.5), 0), (700, 300, 333, 32, "bf16", 0.2, ("upow", 0.1, 0.5), 0.01)]


@pytest.mark.parametrize("act", ["none", "relu", "gelu"])
@pytest.mark.parametrize("case", REAL, ids=lambda c: "x".join(map(str, c[:4])) + "-" + c[4])
def test_normal_values(tw, case, act):
    """Rounded once; with R = 0 the values of tw_gemm_bias_act."""
    M, K, N, G, dtype, cp, keep, delta = case
    wt, A, At, B = _case(tw, *case, a_dist="normal")
    gen = torch.Generator(device="cuda").manual_seed(7)
    t = _torch_type(dtype)
    bias, R = (torch.randn(s, generator=gen, device="cuda").to(t) for s in ((N,), (M, N)))
    x = A.double() @ B + bias.double()
    spread = A.double().abs() @ B.abs() + bias.double().abs()
    f = {"none": lambda v: v, "relu": lambda v: v.clamp(min=0), "gelu": lambda v: v * torch.special.ndtr(v)}[act](x)
    want = f + R.double()
    fp32 = 1.13 * (K + 8) * U * spread + (3.3e-7 + 1.2e-7 * f.abs() if act == "gelu" else 0) + 2 * U * (f.abs() + R.double().abs())
    bound = torch.finfo(t).eps / 2 * (want.abs() + fp32) + fp32 + 2.0 ** -25
    C = tw.tw_gemm_bias_act_add(wt, A, R, bias, act)
    Rt = _inside(N, M, dtype, -(-M // 8) * 8)[0]
    Rt.copy_(R.t())
    Ct = tw.tw_gemm_t_bias_act_add(wt, At, Rt, bias, act)
    torch.cuda.synchronize()
    assert ((C.double() - want).abs() / bound).max().item() <= 1.0
    assert ((Ct.t().double() - want).abs() / bound).max().item() <= 1.0
    zero = torch.zeros_like(R)
    assert torch.equal(tw.tw_gemm_bias_act_add(wt, A, zero, bias, act), tw.tw_gemm_bias_act(wt, A, bias, act))
    Rt.zero_()
    assert torch.equal(tw.tw_gemm_t_bias_act_add(wt, At, Rt, bias, act), tw.tw_gemm_t_bias_act(wt, At, bias, act))


DENSE = [(1, 64, 64), (3, 70, 30), (300, 130, 260), (1500, 1000, 2000), (4000, 96, 700), (2048, 640, 520), (333, 40, 1001), (70, 9, 3), (20000, 72, 200)]


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("M,K,N", DENSE)
def test_dense(tw, M, K, N, dtype):
    """Every block height, ragged ends, R and C of their own pitches, added to itself, nothing written beside C or read behind R."""
    gen = torch.Generator(device="cuda").manual_seed(M + K + N)
    t = _torch_type(dtype)
    A = _inside(M, K, dtype, -(-K // 8) * 8)[0]
    B = _inside(K, N, dtype, -(-N // 8) * 8)[0]
    density = 1.0 if dtype == "f16" else min(1.0, 60.0 / K)
    A.copy_(torch.randint(-2, 3, (M, K), generator=gen, device="cuda") * (torch.rand((M, K), generator=gen, device="cuda") < density))
    B.copy_(torch.randint(-1, 2, (K, N), generator=gen, device="cuda"))
    bias, R = _integers((N,), dtype, 1), _integers((M, N), dtype, 2)
    prod = A.double() @ B.double()
    ld = -(-N // 8) * 8 + 8
    Rm = torch.empty(((M - 1) * ld + N,), dtype=t, device="cuda").as_strided((M, N), (ld, 1))      # ends with its last element
    for b, act in ((None, "none"), (bias, "relu"), (bias, "none")):
        want = prod if b is None else prod + b.double()
        want = (torch.clamp(want, min=0) if act == "relu" else want) + R.double()
        assert want.abs().max() <= (2048 if dtype == "f16" else 256)
        Rm.copy_(R)
        C, cbuf = _inside(M, N, dtype, -(-N // 64) * 64, 64)
        tw.tw_dense_gemm_bias_act_add(A, B, Rm, b, act, C)
        torch.cuda.synchronize()
        assert torch.equal(C.double(), want) and _only_inside(C, cbuf)
        tw.tw_dense_gemm_bias_act_add(A, B, Rm, b, act, Rm)
        torch.cuda.synchronize()
        assert torch.equal(Rm.double(), want)


def test_dense_gelu_and_rows_far_apart(tw):
    gen = torch.Generator(device="cuda").manual_seed(1)
    M, K, N = 130, 200, 72
    A, B = (torch.randn(s, generator=gen, device="cuda").half() for s in ((M, K), (K, N)))
    R = torch.randn((M, N), generator=gen, device="cuda").half()
    x = A.double() @ B.double()
    f = x * torch.special.ndtr(x)
    want = f + R.double()
    fp32 = 1.13 * (K + 8) * U * (A.double().abs() @ B.double().abs()) + 3.3e-7 + 1.2e-7 * f.abs() + 2 * U * (f.abs() + R.double().abs())
    bound = 2.0 ** -11 * (want.abs() + fp32) + fp32 + 2.0 ** -25
    C = tw.tw_dense_gemm_bias_act_add(A, B, R, None, "gelu")
    assert ((C.double() - want).abs() / bound).max().item() <= 1.0
    far = torch.empty((M, 1 << 23), dtype=torch.float16, device="cuda")
    far[:, :K] = A
    far[:, K:K + N] = R
    Cf = tw.tw_dense_gemm_bias_act_add(far[:, :K], B, far[:, K:K + N], None, "gelu")
    assert torch.equal(Cf, C)


def test_streams_and_graphs(tw):
    """On another stream, and captured (both boundaries, a split product with its second kernel) and replayed on new values."""
    case = (300, 2304, 500, 128, "f16", 0.05, ("upow", 0.05, 0.4), 0)
    wt, A, At, _ = _case(tw, *case, a_dist="normal")
    wt2 = wt.sibling()
    gen = torch.Generator(device="cuda").manual_seed(2)
    R = torch.randn((300, 500), generator=gen, device="cuda").half()
    Rt = _inside(500, 300, "f16", 304)[0]
    Rt.copy_(R.t())
    want, want_t = tw.tw_gemm_bias_act_add(wt, A, R), tw.tw_gemm_t_bias_act_add(wt, At, Rt)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    C, Ct = torch.empty_like(want), _inside(500, 300, "f16", 320)[0]
    tw.tw_gemm_bias_act_add(wt2, A, R, C=C, stream=side)
    tw.tw_gemm_t_bias_act_add(wt2, At, Rt, Ct=Ct, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    assert torch.equal(C, want) and torch.equal(Ct, want_t)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        tw.tw_gemm_bias_act_add(wt2, A, R, C=C)
        tw.tw_gemm_t_bias_act_add(wt2, At, Rt, Ct=Ct)
    for k in range(3):
        R.mul_(0.5)
        Rt.copy_(R.t())
        A.add_(0.25)
        At.copy_(A.t())
        graph.replay()
        torch.cuda.synchronize()
        got = C.clone(), Ct.clone()
        assert torch.equal(got[0], tw.tw_gemm_bias_act_add(wt, A, R)) and torch.equal(got[1], tw.tw_gemm_t_bias_act_add(wt, At, Rt))


MEMORY_CHILD = """
import sys
sys.path.insert(0, {root!r})
import torch
from paper_2008_13006_amd import binding as tw, workloads as W
modes = set()
for dtype, t in (("f16", torch.float16), ("bf16", torch.bfloat16)):
    for M, K, N in ((16384, 768, 768), (16384, 2304, 768), (8192, 4096, 1024)):
        w = W.generate(W.small_spec("memory", M=1, K=K, N=N, G=128, dtype=dtype, col_prune=0.05, keep=("upow", 0.1, 0.4), seed_offset=9500))
        weight = tw.TwWeight(tw.tw_pack(w.B, w.mask, 128, dtype))
        modes.add(tw.tw_gemm_plan(weight.blob, M)["mode"])
        a, r, c = (torch.zeros(s, dtype=t, device="cuda") for s in ((M, K), (M, N), (M, N)))
        # (what the call below needs of the library's code is loaded: that of the products without R, and of those with it by the other boundary's)
        tw.tw_gemm_bias_act(weight, a, None, "relu", c)
        at, ct = torch.zeros((K, 64), dtype=t, device="cuda"), torch.zeros((N, 64), dtype=t, device="cuda")
        tw.tw_gemm_t_bias_act_add(weight, at, ct, None, "relu", torch.empty_like(ct))
        torch.cuda.synchronize()
        before = torch.cuda.mem_get_info()[0]
        tw.tw_gemm_bias_act_add(weight, a, r, None, "relu", c)
        torch.cuda.synchronize()
        print("taken", (before - torch.cuda.mem_get_info()[0]) >> 20, "MB", dtype, M, K, N, flush=True)
print("modes", sorted(modes), flush=True)
"""


def test_first_calls_take_no_device_memory():
    """The library allocates no device memory, and neither does the runtime for its kernels: one whose registers spill has memory set aside for every
    lane of the card at its first call.  A process of its own, in which no other kernel has been run."""
    import os
    import subprocess
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    child = subprocess.run([sys.executable, "-c", MEMORY_CHILD.format(root=root)], capture_output=True, text=True, timeout=100)
    assert child.returncode == 0, child.stderr[-2000:]
    taken = [line.split() for line in child.stdout.splitlines() if line.startswith("taken")]
    assert len(taken) == 6 and "modes [0, 1, 2]" in child.stdout, child.stdout
    assert all(int(words[1]) == 0 for words in taken), child.stdout
