"""What lies between the tile-wise products of a Transformer layer: products that add a residual, layer norm, attention.

A case is one call on one MI355X.  `run` makes it twofold: in its plain form (elementary torch operations in 32 bits, rounded once
at the end), or as a user's program calls this package.

Fields of a case
  op      "add" (row-major product with bias, activation and residual, weight pruned to tiles), "add_t" (both matrices transposed),
          "add_dense" (an unpruned weight), "ln" and "ln_t" (layer norm over rows, over columns), "ln_grad" (its backward pass),
          "attention" (packed sequences)
  M       tokens
  dtype   16-bit storage type
  K, N    of a product: inputs and outputs of the weight; G: tile granularity; sparsity: zeros / (K*N), pruned columns included;
          col_prune: share of columns pruned altogether; skew: "spread" (tiles keep between 0.4 and 1.6 times the mean) or "zipf"
          (a few tiles keep most rows); bias, act: the rest of the epilogue
  N       of layer norm: features; affine: with weight and offset; stats: the call leaves mean and 1/deviation for a backward pass
  heads, kv_heads, d, causal, seqs, spread   of attention: heads of Q, of K and V, their width, number of sequences; spread: lengths are
          spread over the logarithm of a wide range (else all alike), drawn from `lens_seed`
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

_PRODUCT = dict(G=128, sparsity=0.75, col_prune=0.05, skew="spread", bias=True, act="none", dtype="f16")
_ATTENTION = dict(op="attention", spread=True, lens_seed=1, dtype="f16", causal=True)


def listed():
    return [
        # one token through the attention output's product: the latency of a call
        {**_PRODUCT, "name": "add_row_1x768x768", "op": "add", "M": 1, "K": 768, "N": 768},
        # the same product on a full batch (128 sequences of 128 tokens)
        {**_PRODUCT, "name": "add_16384x768x768", "op": "add", "M": 16384, "K": 768, "N": 768},
        # second feed-forward product of a large layer on the transposed layout, skewed tiles
        {**_PRODUCT, "name": "add_t_8192x4096x1024", "op": "add_t", "M": 8192, "K": 4096, "N": 1024, "sparsity": 0.875, "col_prune": 0.10,
         "skew": "zipf", "dtype": "bf16"},
        # a layer that was left unpruned, nothing a multiple of anything, activation in front of the residual
        {**_PRODUCT, "name": "add_dense_4321x1000x1234", "op": "add_dense", "M": 4321, "K": 1000, "N": 1234, "act": "gelu", "dtype": "bf16"},
        # a serving batch behind the residual
        {"name": "ln_512x768", "op": "ln", "M": 512, "N": 768, "dtype": "f16", "affine": True, "stats": False},
        # a full batch on the transposed layout
        {"name": "ln_t_16384x768", "op": "ln_t", "M": 16384, "N": 768, "dtype": "f16", "affine": True, "stats": False},
        # forward pass of a training step: statistics stay for the backward pass
        {"name": "ln_16384x4096", "op": "ln", "M": 16384, "N": 4096, "dtype": "bf16", "affine": True, "stats": True},
        # backward pass of a full batch, gradient of the weight included
        {"name": "ln_grad_16384x768", "op": "ln_grad", "M": 16384, "N": 768, "dtype": "bf16", "affine": True},
        # the same for sizes that are a multiple of nothing
        {"name": "ln_grad_4321x1234", "op": "ln_grad", "M": 4321, "N": 1234, "dtype": "f16", "affine": True},
        # an encoder's full batch: every token sees its whole sequence
        {**_ATTENTION, "name": "attention_128x128", "M": 16384, "seqs": 128, "spread": False, "heads": 12, "kv_heads": 12, "d": 64,
         "causal": False},
        # prompts of a serving step packed into one batch, from one token to thousands, grouped heads
        {**_ATTENTION, "name": "attention_packed_12000", "M": 12000, "seqs": 24, "heads": 16, "kv_heads": 4, "d": 128, "dtype": "bf16"},
        # one long prompt
        {**_ATTENTION, "name": "attention_1x8192", "M": 8192, "seqs": 1, "heads": 16, "kv_heads": 4, "d": 128, "dtype": "bf16"},
    ]


def _log_int(rng, lo, hi):
    """An integer spread over the logarithm of [lo, hi]; half of them multiples of 64 (where that is in range)."""
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    if v >= 64 and rng.random() < 0.5:
        v = (v + 32) // 64 * 64
    return max(lo, min(hi, v))


def draw(rng):
    op = rng.choice(["add", "add_t", "add_dense", "ln", "ln_t", "ln_grad", "attention", "attention"])
    dtype = rng.choice(["f16", "bf16"])
    if op == "attention":
        d = rng.choice([32, 64, 64, 80, 96, 128, 128])
        kv = rng.choice([1, 2, 4, 8, 12])
        heads = kv * rng.choice([1, 1, 2, 4])
        M = _log_int(rng, 1, min(16384, int(math.sqrt(2.0e10 / (heads * d)))))
        return {**_ATTENTION, "M": M, "seqs": min(M, _log_int(rng, 1, 64)), "spread": rng.random() < 0.7, "lens_seed": rng.randint(1, 10 ** 6),
                "heads": heads, "kv_heads": kv, "d": d, "causal": rng.random() < 0.6, "dtype": dtype}
    if op in ("ln", "ln_t", "ln_grad"):
        N = _log_int(rng, 64, 8192)
        case = {"op": op, "M": _log_int(rng, 1, min(32768, (16384 * 4096) // N)), "N": N, "dtype": dtype, "affine": rng.random() < 0.8}
        if op != "ln_grad":
            case["stats"] = rng.random() < 0.5
        return case
    K, N = _log_int(rng, 128, 4608), _log_int(rng, 128, 4096)
    sparsity = round(rng.uniform(0.5, 0.9), 3)
    M = _log_int(rng, 1, int(min(16384, 4.0e10 / (2.0 * K * N), 2 ** 26 / (K + 2 * N))))
    return {**_PRODUCT, "op": op, "M": M, "K": K, "N": N, "G": rng.choice([32, 64, 128, 128]), "sparsity": sparsity,
            "col_prune": round(rng.uniform(0.0, 0.10), 3), "skew": rng.choice(["spread", "zipf"]), "bias": rng.random() < 0.7,
            "act": rng.choice(["none", "none", "relu", "gelu"]), "dtype": dtype}


# ------------------------------------------------------------------------------------------------ inputs
def _type(case):
    return torch.float16 if case["dtype"] == "f16" else torch.bfloat16


def _pitched(rows, cols, dtype, pitch):
    return torch.empty((rows, -(-cols // pitch) * pitch), dtype=dtype, device="cuda")[:, :cols]


def _randn(rows, cols, dtype, gen, scale=1.0, pitch=8):
    """rows x cols on the GPU, N(0, scale), the row pitch a multiple of `pitch` elements."""
    out = _pitched(rows, cols, dtype, pitch)
    out.copy_(torch.randn((rows, cols), generator=gen, device="cuda") * scale)
    return out


def _tile_mask(w, case, gen):
    """Columns of least L1 norm pruned first, the rest regrouped G at a time, every tile keeps its strongest rows."""
    K, N, G = case["K"], case["N"], case["G"]
    a = w.float().abs()
    n_kept = N - int(math.floor(case["col_prune"] * N + 0.5))
    kept = torch.sort(torch.argsort(a.sum(0), descending=True, stable=True)[:n_kept]).values
    T = -(-n_kept // G)
    scores = torch.zeros((K, T * G), device="cuda")
    scores[:, :n_kept] = a[:, kept]
    rank = torch.argsort(torch.argsort(scores.view(K, T, G).sum(2), dim=0, descending=True, stable=True), dim=0)
    u = torch.randperm(T, generator=gen, device="cuda").float() / max(1, T - 1)
    share = 0.4 + 1.2 * u if case["skew"] == "spread" else 0.25 + 3.0 * torch.exp(-4.0 * u)
    density = (1.0 - case["sparsity"]) * N / n_kept
    rows = torch.clamp((share * density / share.mean() * K + 0.5).long(), 1, K)
    tile_of = torch.arange(n_kept, device="cuda") // G
    mask = torch.zeros((K, N), dtype=torch.bool, device="cuda")
    mask[:, kept] = (rank < rows)[:, tile_of]
    return mask


def _lengths(case):
    """Lengths of the packed sequences: they add up to M, none is empty."""
    M, n = case["M"], case["seqs"]
    if not case["spread"]:
        return [M // n + (i < M % n) for i in range(n)]
    rng = random.Random(case["lens_seed"])
    w = [math.exp(rng.uniform(0.0, math.log(100.0))) for _ in range(n)]
    lens = [1 + int((M - n) * v / sum(w)) for v in w]
    lens[lens.index(max(lens))] += M - sum(lens)
    return lens


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    op, M, dt = case["op"], case["M"], _type(case)
    st = {"case": case}
    if op == "attention":
        H, Hk, d = case["heads"], case["kv_heads"], case["d"]
        qkv = _randn(M, (H + 2 * Hk) * d, dt, gen)                  # as a fused product leaves them
        st["q"], st["k"], st["v"] = qkv[:, :H * d], qkv[:, H * d:(H + Hk) * d], qkv[:, (H + Hk) * d:]
        lens = torch.tensor(_lengths(case))
        st["seq_start"] = torch.cat([torch.zeros(1, dtype=torch.int64), lens.cumsum(0)]).to(torch.int32).cuda()
        st["longest"] = int(lens.max())
        st["out"] = _pitched(M, H * d, dt, 8)
        return st
    N = case["N"]
    if op in ("ln", "ln_t", "ln_grad"):
        # features of different size, a few of them large; tokens of different mean
        x = torch.randn((M, N), generator=gen, device="cuda")
        x *= torch.exp(0.5 * torch.randn(N, generator=gen, device="cuda"))
        x += 0.3 * torch.randn(N, generator=gen, device="cuda") + 0.2 * torch.randn((M, 1), generator=gen, device="cuda")
        if op == "ln_t":
            st["x"] = _pitched(N, M, dt, 64)
            st["x"].copy_(x.t())
            st["out"] = _pitched(N, M, dt, 64)
        else:
            st["x"] = _pitched(M, N, dt, 8)
            st["x"].copy_(x)
            st["out"] = _pitched(M, N, dt, 8)
        st["gamma"] = st["beta"] = None
        if case["affine"]:
            st["gamma"] = (1.0 + 0.1 * torch.randn(N, generator=gen, device="cuda")).to(dt)
            st["beta"] = (0.1 * torch.randn(N, generator=gen, device="cuda")).to(dt)
        if op == "ln_grad":
            st["dy"] = _randn(M, N, dt, gen)
            x = st["x"].double()
            mean = x.mean(1)
            st["mean"], st["rstd"] = mean.float(), torch.rsqrt((x - mean[:, None]).square().mean(1) + 1e-5).float()
            st["dgamma"], st["dbeta"] = (torch.empty(N, device="cuda") for _ in range(2))
        elif case["stats"]:
            st["mean"], st["rstd"] = (torch.empty(M, device="cuda") for _ in range(2))
        else:
            st["mean"] = st["rstd"] = None
        return st
    K = case["K"]
    w = _randn(K, N, dt, gen, 0.02)
    st["bias"] = _randn(1, N, dt, gen, 0.1)[0] if case["bias"] else None
    st["act"] = case["act"]
    if op == "add_t":
        st["a"], st["r"], st["out"] = _randn(K, M, dt, gen, pitch=64), _randn(N, M, dt, gen, pitch=64), _pitched(N, M, dt, 64)
    else:
        st["a"], st["r"], st["out"] = _randn(M, K, dt, gen), _randn(M, N, dt, gen), _pitched(M, N, dt, 8)
    if op != "add_dense":
        mask = _tile_mask(w, case, gen)
        w = w * mask
        if own:
            from paper_2008_13006_amd import binding as tw
            bits = w.contiguous().view(torch.int16).cpu().numpy().view(np.uint16)
            w = tw.TwWeight(tw.tw_pack(bits, mask.cpu().numpy().view(np.uint8), case["G"], case["dtype"]))
    st["w"] = w
    return st


# ------------------------------------------------------------------------------------------------ one pass
def _own_run(st):
    from paper_2008_13006_amd import binding as tw
    op = st["case"]["op"]
    if op == "add":
        return tw.tw_gemm_bias_act_add(st["w"], st["a"], st["r"], st["bias"], st["act"], st["out"])
    if op == "add_t":
        return tw.tw_gemm_t_bias_act_add(st["w"], st["a"], st["r"], st["bias"], st["act"], st["out"])
    if op == "add_dense":
        return tw.tw_dense_gemm_bias_act_add(st["a"], st["w"], st["r"], st["bias"], st["act"], st["out"])
    if op == "ln_grad":
        return tw.tw_layernorm_grad(st["dy"], st["x"], st["gamma"], st["mean"], st["rstd"], st["out"], st["dgamma"], st["dbeta"])
    if op == "attention":
        c = st["case"]
        return tw.tw_attention(st["q"], st["k"], st["v"], st["seq_start"], c["heads"], c["kv_heads"], causal=c["causal"], O=st["out"])
    norm = tw.tw_layernorm_t if op == "ln_t" else tw.tw_layernorm
    y = norm(st["x"], st["gamma"], st["beta"], 1e-5, st["out"], st["mean"], st["rstd"])
    return y if st["mean"] is None else (y, st["mean"], st["rstd"])


def _activate(x, act):
    if act == "relu":
        return torch.clamp(x, min=0.0)
    return 0.5 * x * (1.0 + torch.erf(x * math.sqrt(0.5))) if act == "gelu" else x


def _plain_add(st):
    w, dt = st["w"].float(), st["a"].dtype
    if st["case"]["op"] == "add_t":
        x = w.t() @ st["a"].float()
        if st["bias"] is not None:
            x += st["bias"].float()[:, None]
    else:
        x = st["a"].float() @ w
        if st["bias"] is not None:
            x += st["bias"].float()
    return (_activate(x, st["act"]) + st["r"].float()).to(dt)


def _plain_ln(st):
    dim = 0 if st["case"]["op"] == "ln_t" else 1
    x = st["x"].float()
    mean = x.mean(dim, keepdim=True)
    x = x - mean
    rstd = torch.rsqrt(x.square().mean(dim, keepdim=True) + 1e-5)
    y = x * rstd
    if st["gamma"] is not None:
        g, b = st["gamma"].float(), st["beta"].float()
        y = y * g[:, None] + b[:, None] if dim == 0 else y * g + b
    y = y.to(st["x"].dtype)
    return y if st["mean"] is None else (y, mean.flatten(), rstd.flatten())


def _plain_ln_grad(st):
    dy, rstd = st["dy"].float(), st["rstd"][:, None]
    xh = (st["x"].float() - st["mean"][:, None]) * rstd
    g = dy * st["gamma"].float() if st["gamma"] is not None else dy
    dx = rstd * (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True))
    return dx.to(st["x"].dtype), (dy * xh).sum(0), dy.sum(0)


def _plain_attention(st):
    """All sequences padded to the longest."""
    c = st["case"]
    M, H, Hk, d, L = c["M"], c["heads"], c["kv_heads"], c["d"], st["longest"]
    start = st["seq_start"].long()
    lens = start[1:] - start[:-1]
    pos = torch.arange(L, device="cuda")
    at = torch.clamp(start[:-1, None] + pos, max=M - 1)                                       # [B, L]
    B = at.shape[0]
    q = st["q"][at].float().view(B, L, Hk, H // Hk, d).permute(0, 2, 3, 1, 4).reshape(B * Hk, H // Hk * L, d)
    k = st["k"][at].float().view(B, L, Hk, d).permute(0, 2, 3, 1).reshape(B * Hk, d, L).contiguous()
    v = st["v"][at].float().view(B, L, Hk, d).permute(0, 2, 1, 3).reshape(B * Hk, L, d).contiguous()
    s = torch.bmm(q * d ** -0.5, k).view(B, H, L, L)
    seen = (pos < lens[:, None])[:, None, :]
    if c["causal"]:
        seen = seen & (pos <= pos[:, None])
    s = s.masked_fill(~seen[:, None].expand(B, 1, L, L), float("-inf"))
    s = torch.exp(s - s.amax(-1, keepdim=True))
    s = s / s.sum(-1, keepdim=True)
    o = torch.bmm(s.view(B * Hk, H // Hk * L, L), v).view(B, H, L, d).permute(0, 2, 1, 3).reshape(B * L, H * d)
    row = torch.arange(M, device="cuda")
    seq = torch.searchsorted(start[1:].contiguous(), row, right=True)
    return o[seq * L + row - start[seq]].to(st["q"].dtype)


def run(state):
    if own:
        return _own_run(state)
    op = state["case"]["op"]
    if op == "attention":
        return _plain_attention(state)
    if op == "ln_grad":
        return _plain_ln_grad(state)
    return _plain_ln(state) if op in ("ln", "ln_t") else _plain_add(state)


# ------------------------------------------------------------------------------------------------ in 64 bits
def exact(case, seed):
    st = prepare(case, seed)
    f = {k: v.double() for k, v in st.items() if isinstance(v, torch.Tensor) and v.is_floating_point()}
    op = case["op"]
    if op == "attention":
        H, Hk, d = case["heads"], case["kv_heads"], case["d"]
        out = torch.empty((case["M"], H, d), dtype=torch.float64, device="cuda")
        s0 = 0
        for n in _lengths(case):
            rows = slice(s0, s0 + n)
            q = f["q"][rows].reshape(n, H, d).transpose(0, 1).contiguous()
            k = f["k"][rows].reshape(n, Hk, d).transpose(0, 1).repeat_interleave(H // Hk, 0)
            v = f["v"][rows].reshape(n, Hk, d).transpose(0, 1).repeat_interleave(H // Hk, 0).contiguous()
            kt = k.transpose(1, 2).contiguous()
            for i in range(0, n, 1024):
                s = torch.matmul(q[:, i:i + 1024].contiguous(), kt) / math.sqrt(d)
                if case["causal"]:
                    s += torch.full(s.shape[1:], -math.inf, dtype=torch.float64, device="cuda").triu(i + 1)
                p = torch.softmax(s, -1)
                out[s0 + i:s0 + i + q[:, i:i + 1024].shape[1]] = torch.matmul(p, v).transpose(0, 1)
            s0 += n
        return out.reshape(case["M"], H * d)
    if op in ("ln", "ln_t"):
        x = f["x"].t() if op == "ln_t" else f["x"]
        var, mean = torch.var_mean(x, dim=1, unbiased=False)
        y = (x - mean[:, None]) / torch.sqrt(var + 1e-5)[:, None]
        if case["affine"]:
            y = y * f["gamma"] + f["beta"]
        y = y.t() if op == "ln_t" else y
        return (y, mean, 1.0 / torch.sqrt(var + 1e-5)) if case["stats"] else y
    if op == "ln_grad":
        z = (f["x"] - f["mean"][:, None]) * f["rstd"][:, None]
        g = f["dy"] * f["gamma"] if case["affine"] else f["dy"]
        N = case["N"]
        dx = f["rstd"][:, None] / N * (N * g - g.sum(1)[:, None] - z * (g * z).sum(1)[:, None])
        return dx, torch.sum(z * f["dy"], 0), f["dy"].sum(0)
    a, w = (f["a"].t() if op == "add_t" else f["a"]), f["w"]
    x = torch.matmul(a.contiguous(), w)
    if case["bias"]:
        x = x + f["bias"]
    if case["act"] == "gelu":
        x = x * torch.special.ndtr(x)
    elif case["act"] == "relu":
        x = torch.where(x > 0, x, torch.zeros_like(x))
    x = x.t() if op == "add_t" else x
    return x + f["r"]


def work(case):
    """Inputs read once, outputs written once; of a pruned weight the kept values."""
    M, N = case["M"], case.get("N", 0)
    if case["op"] == "attention":
        H, Hk, d = case["heads"], case["kv_heads"], case["d"]
        pairs = sum(n * (n + 1) / 2 if case["causal"] else n * n for n in _lengths(case))
        return {"bytes": 2.0 * M * d * (2 * H + 2 * Hk) + 4.0 * (case["seqs"] + 1), "flops": 4.0 * pairs * H * d}
    if case["op"] in ("ln", "ln_t"):
        return {"bytes": 4.0 * M * N + (4.0 * N if case["affine"] else 0.0) + (8.0 * M if case["stats"] else 0.0), "flops": 8.0 * M * N}
    if case["op"] == "ln_grad":
        return {"bytes": 6.0 * M * N + 8.0 * M + 8.0 * N + (2.0 * N if case["affine"] else 0.0), "flops": 13.0 * M * N}
    K = case["K"]
    density = 1.0 if case["op"] == "add_dense" else 1.0 - case["sparsity"]
    return {"bytes": 2.0 * M * (K + 2 * N) + 2.0 * density * K * N + (2.0 * N if case["bias"] else 0.0), "flops": 2.0 * M * K * N * density}
