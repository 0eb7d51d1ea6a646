"""The serving operators of the MoE layer that this framework is measured on: their
plain forms in elementary torch operations, and the calls that a user makes of them.

Kinds of case (field "kind"):

  few    a whole layer for 1 to 64 tokens: router, top-K, the picked experts, the
         shared expert and the weighted sum, with bf16 or 8-bit expert weights
  proj   a dense product in 8-bit integers, one scale per token and one per output
         channel; the tokens are bf16 and are quantised within the call
  ffn    the grouped expert FFN in 8-bit integers on dispatched rows: both products,
         and the quantisation of their inputs

8-bit rows: scale = max|row| / 127 and code = 127 value / max|row| rounded to the
nearest integer, ties to even.  Weights hold their channel's contraction in one row.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda"
BF16, F32, F64, I8 = torch.bfloat16, torch.float32, torch.float64, torch.int8

# No drawn case holds more expert weights (elements of W1) or gathers more of them
# (routed rows x one expert's elements) than this, nor computes more.
MAX_WEIGHTS, MAX_GATHER, MAX_FLOPS = 1.9e9, 1.2e9, 4.3e12


def _few(name, S, D, E, K, F, Fs=0, score="softmax", weights="bf16"):
    return dict(name=name, kind="few", S=S, D=D, E=E, K=K, F=F, Fs=Fs, score=score, weights=weights)


def _ffn(name, R, D, E, F, skew=0.0):
    return dict(name=name, kind="ffn", R=R, D=D, E=E, F=F, skew=skew)


def listed():
    return [
        # one sequence's decode step through the 64-expert top-6 layer: latency, and 6 experts' weights
        _few("few_1_e64", 1, 2048, 64, 6, 1024),
        # a decode step of 64 sequences through the same layer: every expert is read, for about six rows each
        _few("few_64_e64", 64, 2048, 64, 6, 1024),
        # the production layer's decode step for 8 sequences: sigmoid router, 192 experts top-7, shared expert
        _few("few_8_prod_e192", 8, 2688, 192, 7, 3520, Fs=3520, score="sigmoid"),
        # 16 sequences through the fewer-but-wider 256-expert layer held in 8 bits
        _few("few_16_e256_i8", 16, 2048, 256, 8, 2688, weights="i8"),
        # three drafted tokens through 512 narrow experts top-22 in 8 bits, dispatch width 672
        _few("few_3_e512_i8", 3, 672, 512, 22, 1856, weights="i8"),
        # a handful of tokens into the latent width
        dict(name="proj_5", kind="proj", M=5, D=2688, N=672),
        # a prompt that no tile divides, into the other latent width
        dict(name="proj_4095", kind="proj", M=4095, D=2688, N=768),
        # prefill through the 4,096 -> 1,024 down projection
        dict(name="proj_16384", kind="proj", M=16384, D=4096, N=1024),
        # the smallest layer's experts: launches and latency only
        _ffn("ffn_tiny", 1024, 256, 8, 512),
        # an odd number of rows, Zipf loads, some of the 128 experts with few rows or none
        _ffn("ffn_3001_zipf", 3001, 2048, 128, 1024, skew=1.1),
        # prefill of the 64-expert top-6 layer
        _ffn("ffn_e64", 49152, 2048, 64, 1024),
        # one of eight expert-parallel GPUs of the 192-expert layer, all 114,688 rows
        _ffn("ffn_ep24", 114688, 2688, 24, 3520),
    ]


# ---------------------------------------------------------------------------
# draws
# ---------------------------------------------------------------------------

def _log(rng, lo, hi, step=1):
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return int(min(max(round(v / step), -(-lo // step)), hi // step)) * step


def draw(rng):
    kind = rng.choice(["few", "few", "few", "proj", "ffn", "ffn"])
    D = _log(rng, 256, 2688, 16)
    F = _log(rng, 512, 3712, 16)
    if kind == "few":
        E = _log(rng, 8, 512)
        c = _few("", _log(rng, 1, 64), D, E, min(_log(rng, 2, 22), E), F, weights=rng.choice(["bf16", "i8"]))
        if rng.random() < 0.4:
            c.update(score="sigmoid", Fs=rng.choice([0, F, _log(rng, 512, 3712, 16)]))
        while c["E"] * D * F > MAX_WEIGHTS:
            c["E"] -= max(1, c["E"] // 8)
            c["K"] = min(c["K"], c["E"])
        while c["S"] > 1 and c["S"] * (c["K"] * F + c["Fs"]) * D > MAX_GATHER:
            c["S"] = c["S"] * 3 // 4
    elif kind == "proj":
        c = dict(kind=kind, M=_log(rng, 1, 16384), D=_log(rng, 256, 4096, 16), N=_log(rng, 256, 4096, 16))
        while work(c)["flops"] > MAX_FLOPS / 16:
            c["M"] = c["M"] * 3 // 4
    else:
        c = _ffn("", _log(rng, 64, 114688), D, _log(rng, 8, 128), F, skew=rng.choice([0.0, 0.0, 0.7]))
        if c["skew"]:
            c["R"] = min(c["R"], 16384)
        while work(c)["flops"] > MAX_FLOPS:
            c["R"] = c["R"] * 3 // 4
    c.pop("name", None)
    return c


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    return g


def _normal(g, shape, std, dtype):
    return (torch.randn(shape, generator=g, device=DEV, dtype=F32) * std).to(dtype)


def _weights(g, E, a, b, kind):
    """E weights of a inputs and b outputs ~ N(0, 1/a): ([E, a, b] bf16, None), or in 8
    bits ([E, b, a] codes, [E, b] scales of the bf16 values' output channels)."""
    if kind == "bf16":
        out, scale = torch.empty((E, a, b), dtype=BF16, device=DEV), None
    else:
        out = torch.empty((E, b, a), dtype=I8, device=DEV)
        scale = torch.empty((E, b), dtype=F32, device=DEV)
    for i in range(0, E, 8):
        w = _normal(g, (min(8, E - i), a, b), a ** -0.5, BF16)
        if kind == "bf16":
            out[i:i + 8] = w
        else:
            w = w.float()
            top = w.abs().amax(1)
            scale[i:i + 8] = top / 127
            out[i:i + 8] = (w * (127 / top)[:, None, :]).round_().clamp_(-127, 127).to(I8).transpose(1, 2)
    return out, scale


def _segments(g, R, E, skew):
    """Expert segment bounds of R rows: even multinomial loads, or Zipf-like ones."""
    w = torch.ones(E, device=DEV, dtype=F64)
    if skew:
        w = (torch.randperm(E, generator=g, device=DEV) + 1.0).double() ** -skew
    n = torch.bincount(torch.multinomial(w, R, replacement=True, generator=g), minlength=E)
    off = torch.zeros(E + 1, dtype=torch.int64, device=DEV)
    off[1:] = n.cumsum(0)
    return off.to(torch.int32), int(n.max())


def _scores(x, Wr, bias, sel_bias, score):
    """(logits, selection scores) in 64 bits."""
    logits = x.double() @ Wr.double() + bias.double()
    return logits, logits.sigmoid() + sel_bias.double() if score == "sigmoid" else logits


def prepare(case, seed):
    c, g = case, _gen(seed)
    D = c["D"]
    st = dict(case=dict(c))
    if c["kind"] == "few":
        S, E, F, Fs = c["S"], c["E"], c["F"], c["Fs"]
        st["Wr"] = _normal(g, (D, E), D ** -0.5, F32)
        st["bias"] = _normal(g, (E,), 0.3, F32)
        st["sel_bias"] = _normal(g, (E,), 0.05 if c["score"] == "sigmoid" else 0.0, F32)
        # whole-number outputs do not hang on the last bit of a score: of four times the
        # tokens, the first whose best K + 1 scores lie apart
        pool = _normal(g, (4 * S, D), 1.0, BF16)
        best = _scores(pool, st["Wr"], st["bias"], st["sel_bias"], c["score"])[1].sort(1, descending=True).values
        tied = (best[:, :-1] - best[:, 1:])[:, :c["K"]].amin(1) < 1e-5
        st["x"] = pool[torch.sort(tied.int(), dim=0, stable=True).indices[:S]].contiguous()
        st["W1"], st["s1"] = _weights(g, E, D, F, c["weights"])
        st["W2"], st["s2"] = _weights(g, E, F, D, c["weights"])
        if Fs:
            st["Ws1"], st["ss1"] = _weights(g, 1, D, Fs, c["weights"])
            st["Ws2"], st["ss2"] = _weights(g, 1, Fs, D, c["weights"])
    elif c["kind"] == "proj":
        W, s = _weights(g, 1, D, c["N"], "i8")
        st.update(x=_normal(g, (c["M"], D), 1.0, BF16), W=W[0], s=s[0])
    else:
        st["offsets"], st["longest"] = _segments(g, c["R"], c["E"], c["skew"])
        st["x"] = _normal(g, (c["R"], D), 1.0, BF16)
        st["W1"], st["s1"] = _weights(g, c["E"], D, c["F"], "i8")
        st["W2"], st["s2"] = _weights(g, c["E"], c["F"], D, "i8")
    st["plan"] = {}
    return st


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------

def run(st):
    if own:
        return {"few": _own_few, "proj": _own_proj, "ffn": _own_ffn}[st["case"]["kind"]](st["case"], st)
    return {"few": _plain_few, "proj": _plain_proj, "ffn": _plain_ffn}[st["case"]["kind"]](st["case"], st)


def _own_few(c, st):
    from paper_2608_28511_amd import layer

    if "layer" not in st["plan"]:   # the model's layer, built once around its weights
        sig = c["score"] == "sigmoid"
        shared = {k: (st[k] if st[k] is None else st[k][0]) for k in ("Ws1", "Ws2", "ss1", "ss2") if k in st}
        st["plan"]["layer"] = layer.LayerFew(c["S"], st["Wr"], st["W1"], st["W2"], c["K"], bias=st["bias"],
                                             sel_bias=st["sel_bias"] if sig else None, score=c["score"],
                                             s1=st["s1"], s2=st["s2"], **shared)
    return st["plan"]["layer"](st["x"])


def _own_proj(c, st):
    from paper_2608_28511_amd import layer

    return layer.latent_proj_i8(st["x"], st["W"], st["s"])


def _own_ffn(c, st):
    from paper_2608_28511_amd import layer

    return layer.grouped_ffn_i8(st["x"], st["offsets"], st["W1"], st["s1"], st["W2"], st["s2"])


def _rows_i8(x):
    """(codes as fp32, scales) of the rows of x; codes in 64 bits, since many lie half way between two integers."""
    top = x.abs().amax(-1, keepdim=True)
    q = (x.double() * 127 / top.double().clamp_min(1e-300)).round().float()
    return q, top / 127


def _relu2(u):
    return u.clamp_min(0) ** 2


def _plain_few(c, st):
    x, S, K = st["x"].float(), c["S"], c["K"]
    logits, sel = _scores(x, st["Wr"], st["bias"], st["sel_bias"], c["score"])
    idx = torch.sort(sel, dim=1, descending=True, stable=True).indices[:, :K]
    picked = logits.gather(1, idx)
    z = picked.sigmoid() if c["score"] == "sigmoid" else (picked - picked.amax(1, keepdim=True)).exp()
    p = (z / z.sum(1, keepdim=True)).float()
    e = idx.reshape(-1)
    if c["weights"] == "bf16":
        h = _relu2(torch.bmm(x.repeat_interleave(K, 0)[:, None], st["W1"][e].float()))
        y = torch.bmm(h, st["W2"][e].float())[:, 0]
        ys = _relu2(x @ st["Ws1"][0].float()) @ st["Ws2"][0].float() if c["Fs"] else 0.0
    else:
        q, sx = _rows_i8(x)
        u = torch.bmm(st["W1"][e].float(), q.repeat_interleave(K, 0)[..., None])[..., 0]
        hq, sh = _rows_i8(_relu2(u * sx.repeat_interleave(K, 0) * st["s1"][e]).to(BF16).float())
        y = torch.bmm(st["W2"][e].float(), hq[..., None])[..., 0] * sh * st["s2"][e]
        ys = 0.0
        if c["Fs"]:
            hq, sh = _rows_i8(_relu2(q @ st["Ws1"][0].float().T * sx * st["ss1"]).to(BF16).float())
            ys = hq @ st["Ws2"][0].float().T * sh * st["ss2"]
    y = (y.view(S, K, -1) * p[..., None]).sum(1) + ys
    return dict(y=y.to(BF16), topk_idx=idx.to(torch.int32), topk_prob=p)


def _plain_proj(c, st):
    q, sx = _rows_i8(st["x"].float())
    return (q @ st["W"].float().T * sx * st["s"]).to(BF16)


def _plain_ffn(c, st):
    # every expert's rows side by side, as many as the longest segment holds
    off, E = st["offsets"].long(), c["E"]
    at = off[:-1, None] + torch.arange(st["longest"], device=off.device)
    inside = at < off[1:, None]
    q, sx = _rows_i8(st["x"].float())
    rows = at.clamp_max(c["R"] - 1)
    u = torch.bmm(q[rows], st["W1"].float().transpose(1, 2)) * sx[rows] * st["s1"][:, None]
    hq, sh = _rows_i8(_relu2(u).to(BF16).float())
    y = torch.bmm(hq, st["W2"].float().transpose(1, 2)) * sh * st["s2"][:, None]
    return y[inside].to(BF16)


# ---------------------------------------------------------------------------
# the same in 64 bits
# ---------------------------------------------------------------------------

def _ints(x):
    """8-bit rows of a 64-bit matrix: (integers, scales)."""
    m = x.abs().max(dim=1).values
    n = torch.where(m > 0, m, torch.ones_like(m))
    return torch.round(127.0 * x / n[:, None]), m / 127.0


def _ffn64(x, W1, s1, W2, s2):
    """One expert on 64-bit rows: bf16 weights [in, out], or 8-bit ones [out, in] with scales."""
    if s1 is None:
        return torch.relu(x @ W1.double()).square() @ W2.double()
    q, s = _ints(x)
    u = (q @ W1.double().t()) * s[:, None] * s1.double()
    q, s = _ints(torch.relu(u).square().to(BF16).double())
    return (q @ W2.double().t()) * s[:, None] * s2.double()


def exact(case, seed):
    c, st = case, prepare(case, seed)
    x = st["x"].double()
    if c["kind"] == "proj":
        q, s = _ints(x)
        return (q @ st["W"].double().t()) * s[:, None] * st["s"].double()
    if c["kind"] == "ffn":
        y = torch.zeros_like(x)
        off = st["offsets"].tolist()
        for e in range(c["E"]):
            if off[e + 1] > off[e]:
                seg = slice(off[e], off[e + 1])
                y[seg] = _ffn64(x[seg], st["W1"][e], st["s1"][e], st["W2"][e], st["s2"][e])
        return y
    logits = x @ st["Wr"].double() + st["bias"].double()
    if c["score"] == "sigmoid":
        act = 1 / (1 + torch.exp(-logits))
        idx = torch.topk(act + st["sel_bias"].double(), c["K"], dim=1).indices
    else:
        act = torch.exp(logits - logits.max(dim=1, keepdim=True).values)
        idx = torch.topk(logits, c["K"], dim=1).indices
    gate = torch.take_along_dim(act, idx, 1)
    gate = gate / gate.sum(1, keepdim=True)
    y = torch.zeros_like(x)
    pair = (lambda k, e: None if st[k] is None else st[k][e])
    for e in sorted(set(idx.reshape(-1).tolist())):
        t, k = torch.nonzero(idx == e, as_tuple=True)
        y[t] += gate[t, k, None] * _ffn64(x[t], st["W1"][e], pair("s1", e), st["W2"][e], pair("s2", e))
    if c["Fs"]:
        y += _ffn64(x, st["Ws1"][0], pair("ss1", 0), st["Ws2"][0], pair("ss2", 0))
    return dict(y=y, topk_idx=None, topk_prob=gate)


# ---------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------

def work(case):
    c, D = case, case["D"]
    if c["kind"] == "few":
        S, E, K, F, Fs = c["S"], c["E"], c["K"], c["F"], c["Fs"]
        used = E * (1 - (1 - K / E) ** S)   # experts that receive a row, under even routing
        w = 2 if c["weights"] == "bf16" else 1
        scales = 0 if w == 2 else 4 * (used * (F + D) + (Fs + D if Fs else 0))
        return dict(bytes=4 * D * S + 4 * D * E + 8 * S * K + 2 * w * D * (used * F + Fs) + scales,
                    flops=2 * S * D * (E + 2 * K * F + 2 * Fs))
    if c["kind"] == "proj":
        M, N = c["M"], c["N"]
        return dict(bytes=2 * M * (D + N) + D * N + 4 * N, flops=2 * M * D * N)
    R, E, F = c["R"], c["E"], c["F"]
    used = min(E, R)
    return dict(bytes=4 * R * D + used * (2 * D * F + 4 * (D + F)) + 4 * (E + 1), flops=4 * R * D * F)
