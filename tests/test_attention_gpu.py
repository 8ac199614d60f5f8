"""Attention over packed prompts through the C ABI on the GPU, against softmax in 64 bits, sequence by sequence.

Tolerance of an element, with p the weights and u = 2^-24: half a step of the result; half a step of every weight times |V| (they are rounded
for the product with V; in f16 a weight below the smallest normal number by half of the smallest step); the scores are fp32 sums of d products,
off by (d + 4) u scale sum|q k|, which with the exponential's own two units is the weights' relative error, twice since the sum of the
weights has it too; and sums over n keys, (n + 64) u each."""
import pytest
import torch

from paper_2008_13006_amd import binding as tw

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
TYPES = {"f16": torch.float16, "bf16": torch.bfloat16}


def starts_of(lens, before=0):
    s = [before]
    for n in lens:
        s.append(s[-1] + n)
    return s


def check(o, q, k, v, starts, heads, kv_heads, scale, causal, rows=None):
    """o against the formula for every row that belongs to a sequence (or those of `rows`)."""
    d = q.shape[1] // heads
    t = o.dtype
    eps2, small = torch.finfo(t).eps / 2, torch.finfo(t).smallest_normal * torch.finfo(t).eps / 2
    worst = 0.0
    for a, b in zip(starts[:-1], starts[1:]):
        n = b - a
        if n == 0:
            continue
        kk = k[a:b].double().view(n, kv_heads, d).permute(1, 0, 2).repeat_interleave(heads // kv_heads, 0).contiguous()
        vv = v[a:b].double().view(n, kv_heads, d).permute(1, 0, 2).repeat_interleave(heads // kv_heads, 0).contiguous()
        kt, ka = kk.transpose(1, 2).contiguous(), kk.abs().transpose(1, 2).contiguous()
        for i in range(0, n, 512):
            j = min(n, i + 512)
            qq = q[a + i:a + j].double().view(j - i, heads, d).permute(1, 0, 2).contiguous()
            s, sa = scale * (qq @ kt), scale * (qq.abs() @ ka)
            if causal:
                hidden = torch.arange(n, device="cuda") > torch.arange(i, j, device="cuda")[:, None]
                s, sa = s.masked_fill(hidden, float("-inf")), sa.masked_fill(hidden, 0.0)
            p = torch.softmax(s, -1)
            delta = (d + 8) * U * sa.amax(-1, keepdim=True) + 8 * U
            want, size = p @ vv, p @ vv.abs()
            fp32 = size * (2 * delta + 2 * (n + 64) * U + eps2)
            if t == torch.float16:
                fp32 = fp32 + n * 2.0 ** -25 * vv.abs().amax(1, keepdim=True)
            bound = eps2 * (want.abs() + fp32) + fp32 + small
            got = o[a + i:a + j].double().view(j - i, heads, d).permute(1, 0, 2)
            ratio = (got - want).abs() / bound
            if rows is not None:
                keep = torch.tensor([r in rows for r in range(a + i, a + j)], device="cuda")
                ratio = ratio[:, keep]
            if ratio.numel():
                assert not bool(torch.isnan(ratio).any())
                worst = max(worst, ratio.max().item())
    assert worst <= 1.0, worst


def make(M, heads, kv_heads, d, dtype, seed, size=1.0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    qkv = (torch.randn((M, (heads + 2 * kv_heads) * d), generator=gen, device="cuda") * size).to(TYPES[dtype])
    return qkv[:, :heads * d], qkv[:, heads * d:(heads + kv_heads) * d], qkv[:, (heads + kv_heads) * d:]


def run(q, k, v, starts, heads, kv_heads, causal, scale=None, **kw):
    s = torch.tensor(starts, dtype=torch.int32, device="cuda") if starts is not None else None
    return tw.tw_attention(q, k, v, s, heads, kv_heads, scale, causal, **kw)


LENGTHS = {
    "one token": [1],
    "single tokens": [1] * 67,
    "short": [3, 1, 7, 31, 2, 64, 5, 1, 33, 17],
    "around a tile": [63, 64, 65, 127, 128, 129, 1],
    "tiles": [128, 128, 256],
    "empty ones": [0, 0, 5, 0, 130, 0, 0, 1, 0, 90, 0],
    "long and short": [1, 700, 2, 300, 1],
}


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("name", LENGTHS)
def test_lengths(name, causal, dtype):
    starts = starts_of(LENGTHS[name])
    for heads, kv_heads, d in ((2, 2, 64), (4, 1, 128)):
        q, k, v = make(starts[-1], heads, kv_heads, d, dtype, 1)
        o = run(q, k, v, starts, heads, kv_heads, causal)
        check(o, q, k, v, starts, heads, kv_heads, d ** -0.5, causal)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("d", [8, 16, 24, 32, 40, 64, 72, 80, 96, 104, 128])
def test_widths(d, causal):
    starts = starts_of([70, 200, 9])
    for dtype in TYPES:
        q, k, v = make(starts[-1], 3, 3, d, dtype, d)
        o = run(q, k, v, starts, 3, 3, causal)
        check(o, q, k, v, starts, 3, 3, d ** -0.5, causal)


@pytest.mark.parametrize("heads,kv_heads", [(1, 1), (8, 8), (8, 1), (16, 4), (12, 12), (12, 3), (5, 5), (24, 8)])
def test_heads(heads, kv_heads):
    starts = starts_of([150, 1, 300])
    q, k, v = make(starts[-1], heads, kv_heads, 32, "bf16", heads)
    for causal in (True, False):
        o = run(q, k, v, starts, heads, kv_heads, causal)
        check(o, q, k, v, starts, heads, kv_heads, 32 ** -0.5, causal)


@pytest.mark.parametrize("causal", [True, False])
def test_long(causal):
    q, k, v = make(4200, 2, 1, 64, "f16", 9)
    check(run(q, k, v, None, 2, 1, causal), q, k, v, [0, 4200], 2, 1, 0.125, causal)


def test_rows_outside_every_sequence_are_left():
    """Tokens before the first and behind the last sequence: their rows stay, and whatever they hold reaches nobody."""
    for dtype, causal in (("f16", True), ("bf16", False)):
        starts = starts_of([40, 129], before=37)
        M = starts[-1] + 150
        q, k, v = make(M, 2, 2, 64, dtype, 4)
        outside = [r for r in range(M) if r < 37 or r >= starts[-1]]
        for x, value in ((q, float("nan")), (k, float("inf")), (v, float("nan"))):
            x[outside] = value
        o = torch.full((M, 128), 5.0, dtype=TYPES[dtype], device="cuda")
        run(q, k, v, starts, 2, 2, causal, O=o)
        assert bool((o[outside] == 5.0).all())
        check(o, q, k, v, starts, 2, 2, 0.125, causal)
        # no sequence at all
        o.fill_(5.0)
        run(q, k, v, [3], 2, 2, causal, O=o)
        run(q, k, v, [7, 7, 7], 2, 2, causal, O=o)
        assert bool((o == 5.0).all())


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("d", [64, 128])
def test_values_that_are_not_finite(dtype, d):
    """Infinities and NaN in K and V stay with the rows that see their token."""
    starts = starts_of([100, 60, 230])
    for causal in (True, False):
        q, k, v = make(starts[-1], 2, 1, d, dtype, 21)
        v[110, 3], v[130, 5], v[130, 6], v[131, 6] = float("inf"), float("nan"), float("inf"), float("-inf")
        k[120, :] = float("nan")
        v[300, :] = float("-inf")
        o = run(q, k, v, starts, 2, 1, causal).view(-1, 2, d)
        bad = [r for r in range(100, 160) if not causal or r >= 120]        # they see the NaN score
        seen = {3: [r for r in range(100, 160) if not causal or r >= 110], 5: [r for r in range(100, 160) if not causal or r >= 130],
                6: [r for r in range(100, 160) if not causal or r >= 130]}
        late = [r for r in range(160, 390) if not causal or r >= 300]
        touched = set(bad) | set(late)
        assert bool(torch.isnan(o[bad]).all())
        assert bool((o[late] == float("-inf")).all())
        for c, rows in seen.items():
            rows = [r for r in rows if r not in touched]
            touched |= set(rows)
            if rows and c == 3:
                assert bool((o[rows, :, 3] == float("inf")).all())
        vz = v.clone()
        vz[~torch.isfinite(vz)] = 0
        kz = k.clone()
        kz[120] = 0
        clean = set(range(390)) - touched
        assert bool(torch.isfinite(o[sorted(clean)]).all())
        check(o.reshape(-1, 2 * d), q, kz, vz, starts, 2, 1, d ** -0.5, causal, rows=clean)


def test_scores_of_every_size():
    """Scores far apart (one key takes everything, the running maximum moves from tile to tile), equal ones, and a scale of zero."""
    starts = starts_of([300, 77])
    for dtype in TYPES:
        q, k, v = make(starts[-1], 2, 2, 64, dtype, 8, size=4.0)
        check(run(q, k, v, starts, 2, 2, True), q, k, v, starts, 2, 2, 0.125, True)
        up = torch.linspace(0.1, 4, 377, device="cuda")[:, None].to(TYPES[dtype])
        k2 = (up * q.sign()).to(TYPES[dtype])                            # larger from key to key
        check(run(q, k2, v, starts, 2, 2, False), q, k2, v, starts, 2, 2, 0.125, False)
        check(run(q, k, v, starts, 2, 2, False, scale=0.0), q, k, v, starts, 2, 2, 0.0, False)
        check(run(q, k, v, starts, 2, 2, True, scale=0.01), q, k, v, starts, 2, 2, 0.01, True)


def test_pitches_and_in_place():
    gen = torch.Generator(device="cuda").manual_seed(2)
    t = torch.float16
    starts = starts_of([90, 111])
    bufs = [torch.randn((201, ld), generator=gen, device="cuda").to(t) for ld in (136, 72, 200, 160)]
    q, k, v = bufs[0][:, 8:136], bufs[1][:, :64], bufs[2][:, 64:128]
    o = torch.full((201, 160), 3.0, dtype=t, device="cuda")
    run(q, k, v, starts, 2, 1, True, O=o[:, 16:144])
    assert bool((o[:, :16] == 3.0).all()) and bool((o[:, 144:] == 3.0).all())
    check(o[:, 16:144], q, k, v, starts, 2, 1, 0.125, True)
    want = o[:, 16:144].clone()
    assert run(q, k, v, starts, 2, 1, True, O=q).data_ptr() == q.data_ptr()
    assert torch.equal(q, want)


def test_offsets_beyond_32_bits():
    """Rows two megabytes apart: the last ones lie more than 2^32 bytes behind the first."""
    M, ld, d = 2300, 1 << 20, 64
    big = torch.empty((M, ld), dtype=torch.bfloat16, device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(6)
    parts = [big[:, 64 * i:64 * i + 64] for i in range(4)]
    for x in parts[:3]:
        x.copy_(torch.randn((M, d), generator=gen, device="cuda"))
    starts = [0, 100, M]
    run(*parts[:3], starts, 1, 1, True, O=parts[3])
    check(parts[3], *[x.contiguous() for x in parts[:3]], starts, 1, 1, 0.125, True)


def test_many_sequences_and_repeats():
    gen = torch.Generator().manual_seed(0)
    lens = torch.randint(0, 4, (3000,), generator=gen).tolist()
    starts = starts_of(lens)
    q, k, v = make(starts[-1], 2, 2, 32, "f16", 30)
    o = run(q, k, v, starts, 2, 2, True)
    for a, b in zip(starts[:-1], starts[1:]):
        if b - a == 1:
            assert torch.equal(o[a], v[a])                               # one key: its value
    some = [0, 1, 2, 700, 701, 1500, 2998, 2999]
    for s in some:
        check(o, q, k, v, starts[s:s + 2], 2, 2, 32 ** -0.5, True)
    assert torch.equal(o, run(q, k, v, starts, 2, 2, True))


def test_lists_that_do_not_ascend_touch_nothing_outside():
    """What such a list gives is unspecified; the call ends and the matrices' surroundings stay."""
    M = 300
    q, k, v = make(M, 1, 1, 64, "f16", 3)
    buf = torch.full((M + 40, 64), 9.0, dtype=torch.float16, device="cuda")
    for starts in ([5, 3, 200, 100], [-50, 20, 10 ** 9], [2 ** 31 - 1, -2 ** 31], [300, 0]):
        run(q, k, v, starts, 1, 1, True, O=buf[20:20 + M])
        torch.cuda.synchronize()
        assert bool((buf[:20] == 9.0).all()) and bool((buf[20 + M:] == 9.0).all())


def test_streams_and_graphs():
    """Another stream than the current one, and a captured call replayed on other inputs and other lengths."""
    M, heads = 500, 4
    q, k, v = make(M, heads, 2, 64, "bf16", 40)
    seq = torch.tensor([0, 100, 500], dtype=torch.int32, device="cuda")
    o = torch.zeros((M, heads * 64), dtype=torch.bfloat16, device="cuda")
    want = tw.tw_attention(q, k, v, seq, heads, 2)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    tw.tw_attention(q, k, v, seq, heads, 2, O=o, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(o, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        tw.tw_attention(q, k, v, seq, heads, 2, O=o)
    for cut in (100, 1, 499, 250):
        seq.copy_(torch.tensor([0, cut, 500], dtype=torch.int32))
        v.mul_(0.5)
        graph.replay()
        torch.cuda.synchronize()
        got = o.clone()
        assert torch.equal(got, tw.tw_attention(q, k, v, seq, heads, 2))
        check(got, q, k, v, [0, cut, 500], heads, 2, 0.125, True)


@pytest.mark.parametrize("heads,d,lens,before,after", [(16, 80, [4100, 37, 0, 2500, 900, 1], 0, 0), (16, 72, [500] * 12, 150, 333), (5, 104, [9000, 1, 5500], 3, 0),
                                                       (8, 128, [1, 8500, 0], 0, 700), (3, 72, [20000, 12768], 0, 0)])
@pytest.mark.parametrize("causal", [True, False])
def test_many_tiles_of_different_lengths(heads, d, lens, before, after, causal):
    """More workgroups than run at once, prompts of several tiles: tiles start in the order of their numbers of keys.  Every row that belongs to a
    sequence is written, the others are left; in place gives the same bits."""
    starts = starts_of(lens, before)
    M = starts[-1] + after
    q, k, v = make(M, heads, 1, d, "bf16", 21)
    o = torch.full((M, heads * d), 7.0, dtype=torch.bfloat16, device="cuda")
    run(q, k, v, starts, heads, 1, causal, O=o)
    assert bool((o[:before] == 7.0).all()) and bool((o[starts[-1]:] == 7.0).all())
    check(o, q, k, v, starts, heads, 1, d ** -0.5, causal)
    again = q.clone()
    run(again, k, v, starts, heads, 1, causal, O=again)
    assert torch.equal(again[before:starts[-1]], o[before:starts[-1]]) and torch.equal(again[:before], q[:before])


def test_means_of_the_largest_values_stay_finite():
    """A result is a mean of values: where all are the type's largest it is that value, though the rounding of the weights may add up to half a step."""
    heads, d = 4, 64
    starts = starts_of([2, 3, 5, 9, 70, 200])
    for dtype, t in TYPES.items():
        big = 65504.0 if t == torch.float16 else 2.0 ** 100
        q, k, v = make(starts[-1], heads, heads, d, dtype, 33, size=0.7)
        v[:] = big
        v[:, ::2] = -big
        for causal in (False, True):
            o = run(q, k, v, starts, heads, heads, causal).double()
            assert bool(torch.isfinite(o).all())
            assert ((o - v.double()).abs() / big).max().item() <= torch.finfo(t).eps
        # every weight but one is 0.5 (1 + 2^-11) and a little: rounded up by nearly half a step of f16
        q2, k2 = torch.zeros_like(q), torch.zeros_like(k)
        score = torch.tensor(0.5 * (1 + 1.05 * 2.0 ** -11), dtype=torch.float64).log()
        q2[:, 0::d] = q2[:, 1::d] = 1.0
        k2[:, 0::d] = score.to(t)
        k2[:, 1::d] = (score - score.to(t).double()).to(t)
        k2[torch.tensor(starts[:-1], device="cuda")] = 0.0
        o = run(q2, k2, v, starts, heads, heads, False, scale=1.0).double()
        assert bool(torch.isfinite(o).all()) and ((o - v.double()).abs() / big).max().item() <= torch.finfo(t).eps
        v[4] = float("inf")                                      # an infinity stays one
        o = run(q, k, v, starts, heads, heads, False)
        assert bool((o[2:5] == float("inf")).all()) and bool(torch.isfinite(o[:2]).all()) and bool(torch.isfinite(o[5:]).all())


def test_scores_beyond_what_a_step_of_fp32_resolves():
    """Scores of 10^8 to 10^10, where neighbours in fp32 lie 8 to 1024 apart: the largest take everything, equally where they are equal."""
    n, d = 300, 64
    for dtype, t in TYPES.items():
        for unit in (1024.0, 8192.0, 32768.0):
            q = torch.zeros((n, d), dtype=t, device="cuda")
            k = torch.zeros_like(q)
            q[:, 0] = unit
            # scores rise in steps of unit * unit / 64; from key to key, or with the last ones alike
            k[:, 0] = unit + unit / 64 * (torch.arange(n, device="cuda") // 64).to(t)
            v = torch.randint(-8, 9, (n, d), device="cuda").to(t)
            for scale in (0.125, 1.0):
                o = tw.tw_attention(q, k, v, None, 1, 1, scale, True)
                s = (q[:, :1].double() @ k[:, :1].double().t()) * scale
                s = s.masked_fill(torch.arange(n, device="cuda") > torch.arange(n, device="cuda")[:, None], float("-inf"))
                want = torch.softmax(s, 1) @ v.double()
                # the largest weights are alike, and off by half a step as all are; the others are 0
                bound = torch.finfo(t).eps / 2 * (want.abs() + torch.softmax(s, 1) @ v.double().abs()) + 512 * U * 8 + 2.0 ** -25
                assert ((o.double() - want).abs() / bound).max().item() <= 1.0
                # the same beside a value that is not finite, which the rows before the last do not see
                v2 = v.clone()
                v2[n - 1] = float("inf")
                o2 = tw.tw_attention(q, k, v2, None, 1, 1, scale, True)[:n - 1]
                assert ((o2.double() - want[:n - 1]).abs() / bound[:n - 1]).max().item() <= 1.0
        # sums of many large products, whose order shows: whatever the largest is, a result lies among the values
        gen = torch.Generator(device="cuda").manual_seed(5)
        q, k = ((torch.randn((n, d), generator=gen, device="cuda") * 8000).to(t) for _ in range(2))
        v = 3.0 + torch.rand((n, d), generator=gen, device="cuda").to(t)
        v[n - 1] = float("inf")
        for causal in (True, False):
            o = tw.tw_attention(q, k, v, torch.tensor([0, n - 1, n], dtype=torch.int32, device="cuda"), 1, 1, 1.0, causal)[:n - 1]
            assert bool(((o >= 3.0) & (o <= 4.0)).all())


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_many_keys_of_little_weight(dtype):
    """One key outweighs each of the others by 2^25, and has nothing to give: the result is what the others give together.

    f16: the largest weight of a row is 2^7 at least, so that one below the smallest normal number is off by 2^-25 of 2^7 at most, 2^-32 of the
    largest; a normal one by half a step, and a result by half a step (and fp32 as above: (d + 8 + 2 (n + 64)) units and more, below 2^-6 of
    eps / 2 here for bf16, and below 2^-4 of the result for f16)."""
    n, d = 32768, 16
    t = TYPES[dtype]
    q = torch.zeros((n, d), dtype=t, device="cuda")
    k, v = torch.zeros_like(q), torch.ones_like(q)
    q[:, 0], k[:, 0] = 1.0, -17.5
    for where in (0, 20000, n - 1):
        k[:, 0] = -17.5
        k[where], v[:] = 0.0, 1.0
        v[where] = 0.0
        for causal in (False, True):
            o = tw.tw_attention(q, k, v, None, 1, 1, 1.0, causal).double()
            seen = torch.arange(1, n + 1, device="cuda", dtype=torch.float64) if causal else torch.full((n,), float(n), device="cuda", dtype=torch.float64)
            w = torch.exp(torch.tensor(-17.5, dtype=torch.float64)).item()
            sink = (torch.arange(n, device="cuda") >= where) if causal else torch.ones(n, dtype=torch.bool, device="cuda")
            want = torch.where(sink, (seen - 1) * w / (1 + (seen - 1) * w), 1.0)
            eps2 = torch.finfo(t).eps / 2
            fp32 = (d + 8 + 2 * (seen + 64)) * U * 2 * want
            bound = 2 * eps2 * want + fp32 + (seen * 2.0 ** -32 + 2.0 ** -25 if t == torch.float16 else 0.0)
            assert bool(((o - want[:, None]).abs() <= bound[:, None]).all())
