"""A whole encoder (or, causal, decoder prompt) layer as a chain of the library's calls: fused QKV product, attention, output product with the
residual, layer norm, the feed-forward pair with GELU and the residual, layer norm.  Row-major and on the transposed boundary (with
tw_transpose around the attention), eager and captured into one graph, with a tight bound on every stage: each is checked against its formula in
64 bits on the very inputs that it was given."""
import numpy as np
import pytest
import torch

from paper_2008_13006_amd import workloads as W
from tests.test_attention_gpu import check as check_attention
from tests.test_layernorm_gpu import check_forward, check_grad

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.fixture(scope="module")
def tw():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2008_13006_amd import binding
    return binding


class Layer:
    """Four packed weights with their biases, two layer norms, and a buffer for every result."""

    def __init__(self, tw, width, heads, dtype, M, seed, transposed=False):
        self.tw, self.width, self.heads, self.M, self.transposed = tw, width, heads, M, transposed
        self.t = torch.float16 if dtype == "f16" else torch.bfloat16
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.w, self.dense, self.bias = [], [], []
        for i, (K, N) in enumerate(((width, 3 * width), (width, width), (width, 4 * width), (4 * width, width))):
            spec = W.small_spec("layer", M=1, K=K, N=N, G=128, dtype=dtype, col_prune=0.05, keep=("upow", 0.1, 0.5), seed_offset=9300 + seed + i)
            w = W.generate(spec)
            self.w.append(tw.TwWeight(tw.tw_pack(w.B, w.mask, 128, dtype)))
            self.dense.append(tw.bits_to_tensor(w.B, dtype).double() * torch.from_numpy(w.mask).cuda())
            self.bias.append((0.1 * torch.randn(N, generator=gen, device="cuda")).to(self.t))
        self.gamma = [(1 + 0.1 * torch.randn(width, generator=gen, device="cuda")).to(self.t) for _ in range(2)]
        self.beta = [(0.1 * torch.randn(width, generator=gen, device="cuda")).to(self.t) for _ in range(2)]
        new = self._columns if transposed else self._rows
        self.x = new(width)
        self.qkv, self.mid, self.norm1, self.hidden, self.sum2, self.out = (new(n) for n in (3 * width, width, width, 4 * width, width, width))
        self.context = new(width)
        self.qkv_rows, self.context_rows = self._rows(3 * width), self._rows(width)
        self.mean, self.rstd = (torch.empty(M, device="cuda") for _ in range(2))

    def _rows(self, n):
        return torch.zeros((self.M, n), dtype=self.t, device="cuda")

    def _columns(self, n):
        return torch.zeros((n, -(-self.M // 64) * 64), dtype=self.t, device="cuda")[:, :self.M]

    def forward(self, seq_start, causal):
        tw, b, n = self.tw, self.bias, self.width
        product, add, norm = ((tw.tw_gemm_t_bias_act, tw.tw_gemm_t_bias_act_add, tw.tw_layernorm_t) if self.transposed else
                              (tw.tw_gemm_bias_act, tw.tw_gemm_bias_act_add, tw.tw_layernorm))
        product(self.w[0], self.x, b[0], "none", self.qkv)
        rows = self.qkv
        if self.transposed:
            rows = tw.tw_transpose(self.qkv, self.qkv_rows)
        context = self.context_rows if self.transposed else self.context
        tw.tw_attention(rows[:, :n], rows[:, n:2 * n], rows[:, 2 * n:], seq_start, self.heads, causal=causal, O=context)
        if self.transposed:
            tw.tw_transpose(context, self.context)
        add(self.w[1], self.context, self.x, b[1], "none", self.mid)
        norm(self.mid, self.gamma[0], self.beta[0], 1e-5, self.norm1)
        product(self.w[2], self.norm1, b[2], "gelu", self.hidden)
        add(self.w[3], self.hidden, self.norm1, b[3], "none", self.sum2)
        norm(self.sum2, self.gamma[1], self.beta[1], 1e-5, self.out, self.mean, self.rstd)
        return self.out

    def check(self, starts, causal):
        def rows(m):
            return m.t() if self.transposed else m

        def product(got, a, i, act, added):
            x = a.double() @ self.dense[i] + self.bias[i].double()
            f = x * torch.special.ndtr(x) if act == "gelu" else x
            want = f + (added.double() if added is not None else 0)
            K = a.shape[1]
            fp32 = 1.13 * (K + 8) * U * (a.double().abs() @ self.dense[i].abs() + self.bias[i].double().abs()) + 2 * U * want.abs()
            fp32 = fp32 + ((K + 8) * U * added.double().abs() if added is not None else 0) + (3.3e-7 + 1.2e-7 * f.abs() if act == "gelu" else 0)
            bound = torch.finfo(self.t).eps / 2 * (want.abs() + fp32) + fp32 + 2.0 ** -25
            assert ((got.double() - want).abs() / bound).max().item() <= 1.0, i

        n = self.width
        x, qkv, context, mid, norm1, hidden, sum2, out = (rows(m) for m in (self.x, self.qkv, self.context, self.mid, self.norm1, self.hidden, self.sum2, self.out))
        product(qkv, x, 0, "none", None)
        check_attention(context.contiguous(), qkv[:, :n].contiguous(), qkv[:, n:2 * n].contiguous(), qkv[:, 2 * n:].contiguous(), starts, self.heads, self.heads,
                        (n // self.heads) ** -0.5, causal)
        product(mid, context, 1, "none", x)
        check_forward(norm1, None, None, mid, self.gamma[0], self.beta[0], 1e-5)
        product(hidden, norm1, 2, "gelu", None)
        product(sum2, hidden, 3, "none", norm1)
        check_forward(out, self.mean, self.rstd, sum2, self.gamma[1], self.beta[1], 1e-5)


@pytest.mark.parametrize("transposed", [False, True], ids=["rows", "columns"])
@pytest.mark.parametrize("dtype,width,heads,lens,causal", [
    ("f16", 256, 4, [1], True), ("bf16", 256, 2, [37, 1, 200, 90], True), ("f16", 768, 12, [128] * 4, False), ("bf16", 512, 8, [900, 3, 333], False)])
def test_layer(tw, dtype, width, heads, lens, causal, transposed):
    M = sum(lens)
    layer = Layer(tw, width, heads, dtype, M, seed=width + M, transposed=transposed)
    starts = np.concatenate([[0], np.cumsum(lens)]).tolist()
    seq = torch.tensor(starts, dtype=torch.int32, device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(M)
    layer.x.copy_(torch.randn(layer.x.shape, generator=gen, device="cuda"))
    layer.forward(seq, causal)
    torch.cuda.synchronize()
    layer.check(starts, causal)


def test_layer_in_a_graph(tw):
    """Captured once, replayed on other activations and other sequence lengths, eager work in between: the bits of the eager chain."""
    for transposed in (False, True):
        layer = Layer(tw, 256, 4, "bf16", 300, seed=5, transposed=transposed)
        seq = torch.tensor([0, 100, 300], dtype=torch.int32, device="cuda")
        gen = torch.Generator(device="cuda").manual_seed(1)
        layer.forward(seq, True)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            layer.forward(seq, True)
        for cut in (100, 17, 299):
            layer.x.copy_(torch.randn(layer.x.shape, generator=gen, device="cuda"))
            seq.copy_(torch.tensor([0, cut, 300], dtype=torch.int32))
            graph.replay()
            torch.cuda.synchronize()
            got = layer.out.clone()
            layer.check([0, cut, 300], True)
            layer.forward(seq, True)
            torch.cuda.synchronize()
            assert torch.equal(got, layer.out)


def test_norm_of_a_step(tw):
    """Forward with its statistics kept, then the backward pass on them, in one graph, replayed on new values."""
    gen = torch.Generator(device="cuda").manual_seed(2)
    M, N = 700, 512
    layer = Layer(tw, N, 8, "bf16", M, seed=3)
    dy = torch.zeros((M, N), dtype=torch.bfloat16, device="cuda")
    dx = torch.zeros_like(dy)
    dgamma, dbeta = (torch.zeros(N, device="cuda") for _ in range(2))
    workspace = torch.empty(tw.tw_layernorm_grad_workspace(M, N), dtype=torch.uint8, device="cuda")

    def step():
        tw.tw_gemm_bias_act_add(layer.w[3], layer.hidden, layer.x, layer.bias[3], "none", layer.sum2)
        tw.tw_layernorm(layer.sum2, layer.gamma[1], layer.beta[1], 1e-5, layer.out, layer.mean, layer.rstd)
        tw.tw_layernorm_grad(dy, layer.sum2, layer.gamma[1], layer.mean, layer.rstd, dx, dgamma, dbeta, workspace)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(3):
        for m in (layer.hidden, layer.x, dy):
            m.copy_(torch.randn(m.shape, generator=gen, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        check_forward(layer.out, layer.mean, layer.rstd, layer.sum2, layer.gamma[1], layer.beta[1], 1e-5)
        check_grad(dx, dgamma, dbeta, dy, layer.sum2, layer.gamma[1], layer.mean, layer.rstd)


CALLS = {
    "gemm": lambda tw, o, w, s: tw.tw_gemm(w, o["a"], stream=s),
    "gemm_t": lambda tw, o, w, s: tw.tw_gemm_t(w, o["at"], stream=s),
    "gemm_bias_act": lambda tw, o, w, s: tw.tw_gemm_bias_act(w, o["a"], act="relu", stream=s),
    "transpose": lambda tw, o, w, s: tw.tw_transpose(o["a"], stream=s),
    "dense": lambda tw, o, w, s: tw.tw_dense_gemm(o["a"], o["b"], stream=s),
    "dense_bias_act": lambda tw, o, w, s: tw.tw_dense_gemm_bias_act(o["a"], o["b"], stream=s),
    "gemm_add": lambda tw, o, w, s: tw.tw_gemm_bias_act_add(w, o["a"], o["r"], stream=s),
    "gemm_t_add": lambda tw, o, w, s: tw.tw_gemm_t_bias_act_add(w, o["at"], o["rt"], stream=s),
    "dense_add": lambda tw, o, w, s: tw.tw_dense_gemm_bias_act_add(o["a"], o["b"], o["r"], stream=s),
    "layernorm": lambda tw, o, w, s: tw.tw_layernorm(o["r"], stream=s),
    "layernorm_t": lambda tw, o, w, s: tw.tw_layernorm_t(o["rt"], stream=s),
    "layernorm_grad": lambda tw, o, w, s: tw.tw_layernorm_grad(o["r"], o["r"], None, o["mean"], o["rstd"], stream=s),
    "attention": lambda tw, o, w, s: tw.tw_attention(o["r"][:, :64], o["r"][:, 64:128], o["r"][:, 128:192], None, 1, stream=s),
}


@pytest.mark.parametrize("name", CALLS)
def test_what_a_call_allocates_belongs_to_its_stream(tw, name):
    """With `stream`, outputs that are not given and a workspace that grows come from that stream's memory, not from the current one's,
    whose last user may still be running; what comes back is what the call on the current stream gives."""
    t, M, K, N = torch.float16, 64, 2048, 256
    gen = torch.Generator(device="cuda").manual_seed(8)
    spec = W.small_spec("streams", M=1, K=K, N=N, G=64, dtype="f16", col_prune=0.05, keep=("upow", 0.1, 0.5), seed_offset=9400)
    w = W.generate(spec)
    blob = tw.tw_pack(w.B, w.mask, 64, "f16")
    assert tw.tw_gemm_workspace(blob, M) > 256                   # (K is split: the products let their workspaces grow)
    o = {k: torch.randn(s, generator=gen, device="cuda").to(t) for k, s in (("a", (M, K)), ("r", (M, N)), ("b", (K, N)))}
    o.update(at=o["a"].t().contiguous(), rt=o["r"].t().contiguous(), mean=torch.zeros(M, device="cuda"), rstd=torch.ones(M, device="cuda"))

    def stream_of(x):
        at = x.data_ptr()
        return next(seg["stream"] for seg in torch.cuda.memory_snapshot() if seg["address"] <= at < seg["address"] + seg["total_size"])

    want = CALLS[name](tw, o, tw.TwWeight(blob), None)
    fresh = tw.TwWeight(blob)
    held = fresh.workspace
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = CALLS[name](tw, o, fresh, side)
    torch.cuda.current_stream().wait_stream(side)
    for x, y in zip(got, want) if isinstance(got, tuple) else [(got, want)]:
        assert stream_of(x) == side.cuda_stream and torch.equal(x, y)
    assert fresh.workspace is held or stream_of(fresh.workspace) == side.cuda_stream
    side.synchronize()


@pytest.mark.parametrize("name", CALLS)
def test_raw_handles_stand_for_streams(tw, name):
    """Whatever has a `cuda_stream`: outputs that are not given come from that stream's memory as well."""
    class Handle:
        def __init__(self, stream):
            self.cuda_stream = stream.cuda_stream

    t, M, K, N = torch.float16, 64, 512, 256
    gen = torch.Generator(device="cuda").manual_seed(9)
    w = W.generate(W.small_spec("handles", M=1, K=K, N=N, G=64, dtype="f16", col_prune=0.05, keep=("upow", 0.1, 0.5), seed_offset=9450))
    weight = tw.TwWeight(tw.tw_pack(w.B, w.mask, 64, "f16"))
    o = {k: torch.randn(s, generator=gen, device="cuda").to(t) for k, s in (("a", (M, K)), ("r", (M, N)), ("b", (K, N)))}
    o.update(at=o["a"].t().contiguous(), rt=o["r"].t().contiguous(), mean=torch.zeros(M, device="cuda"), rstd=torch.ones(M, device="cuda"))
    want = CALLS[name](tw, o, weight, None)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = CALLS[name](tw, o, weight, Handle(side))
    torch.cuda.current_stream().wait_stream(side)
    for x, y in zip(got, want) if isinstance(got, tuple) else [(got, want)]:
        assert torch.equal(x, y)
    side.synchronize()
