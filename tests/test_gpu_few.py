"""moe_layer_few against the layer's definition in 64 bits.

Logits are sums of D exact products in fp32: chains of 16, two joins, ceil(D / 64)
partial sums and the bias, so each is within (19 + ceil(D / 64)) 2^-24 of the sum of its
terms' magnitudes; tau is a token's largest such error.  Picks may differ from 64 bits by
2 tau, weights by 2 tau + 2^-20 of their value (the exponential and the division).
bf16 weights: y's bound is elementwise.  Each expert's term carries the errors of
serving_oracle.ffn_bound and its weight's; K + 1 terms are summed in fp32 and rounded once
to bf16.
8-bit weights: the codes and integer sums are those of moe_grouped_ffn_i8, whose y_disp is
rounded to bf16 once more.
"""
import numpy as np
import pytest
import torch

from oracle import moe_oracle as O
from oracle import serving_oracle as V
from paper_2608_28511_amd import _lib as L
from paper_2608_28511_amd import layer

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16 = torch.bfloat16


def np64(t):
    return t.detach().cpu().double().numpy()


class Model:
    """Weights of one layer; the experts' bf16 values are kept beside their 8-bit form."""

    def __init__(self, D, E, K, F, Fs=0, score="softmax", weights="bf16", seed=0, bias_std=0.3):
        g = torch.Generator(device=DEV).manual_seed(seed)
        n = lambda shape, std: torch.randn(shape, generator=g, device=DEV) * std  # noqa: E731
        self.D, self.E, self.K, self.F, self.Fs, self.score, self.weights = D, E, K, F, Fs, score, weights
        self.Wr = n((D, E), D ** -0.5)
        self.bias = n((E,), bias_std)
        self.sel = n((E,), 0.05) if score == "sigmoid" else None
        self.W1, self.W2 = n((E, D, F), D ** -0.5).to(BF16), n((E, F, D), F ** -0.5).to(BF16)
        self.kw = dict(bias=self.bias, sel_bias=self.sel, score=score)
        if Fs:
            self.Ws1, self.Ws2 = n((D, Fs), D ** -0.5).to(BF16), n((Fs, D), Fs ** -0.5).to(BF16)
        if weights == "i8":
            self.w1, self.s1 = layer.quant_weights_i8(self.W1)
            self.w2, self.s2 = layer.quant_weights_i8(self.W2)
            self.kw.update(s1=self.s1, s2=self.s2)
            if Fs:
                self.ws1, self.ss1 = layer.quant_weights_i8(self.Ws1)
                self.ws2, self.ss2 = layer.quant_weights_i8(self.Ws2)
                self.kw.update(Ws1=self.ws1, Ws2=self.ws2, ss1=self.ss1, ss2=self.ss2)
        else:
            self.w1, self.w2 = self.W1, self.W2
            if Fs:
                self.kw.update(Ws1=self.Ws1, Ws2=self.Ws2)

    def layer(self, S):
        return layer.LayerFew(S, self.Wr, self.w1, self.w2, self.K, **self.kw)

    def tokens(self, S, seed=1):
        g = torch.Generator(device=DEV).manual_seed(seed)
        return torch.randn((S, self.D), generator=g, device=DEV).to(BF16)

    def picks(self, x):
        """(selection scores, weights of given picks) in 64 bits."""
        logits = np64(x) @ np64(self.Wr) + np64(self.bias)
        if self.score == "sigmoid":
            act = 1 / (1 + np.exp(-logits))
            return act + np64(self.sel), act
        return logits, np.exp(logits - logits.max(1, keepdims=True))


def check_picks(m, x, idx, prob):
    """The weights of the picks in 64 bits, and their relative error's bound per token."""
    sel, act = m.picks(x)
    S, K = idx.shape
    mag = np.abs(np64(x)) @ np.abs(np64(m.Wr)) + np.where(np.isfinite(np64(m.bias)), np.abs(np64(m.bias)), 0)
    tau = (19 + -(-m.D // 64)) * 2.0 ** -24 * mag.max(1)
    assert ((idx >= 0) & (idx < m.E)).all()
    got = np.take_along_axis(sel, idx, 1)
    for t in range(S):
        assert len(set(idx[t])) == K
        assert np.all(got[t][:-1] >= got[t][1:] - 2 * tau[t] - 2.0 ** -22)
        rest = np.delete(sel[t], idx[t])
        assert rest.size == 0 or got[t].min() >= rest.max() - 2 * tau[t] - 2.0 ** -22
    w = np.take_along_axis(act, idx, 1)
    ref = w / w.sum(1, keepdims=True)
    eps = (2 * tau + 2.0 ** -20)[:, None]
    assert np.all(np.abs(prob - ref) <= eps * ref)
    return ref, eps


def check_bf16(m, x, out):
    idx, y = out["topk_idx"].cpu().numpy().astype(int), np64(out["y"])
    p, eps = check_picks(m, x, idx, np64(out["topk_prob"]))
    xs = np64(x)
    ref, tol = np.zeros_like(xs), np.zeros_like(xs)
    for e in sorted(set(idx.ravel())):
        t, k = np.nonzero(idx == e)
        v, b = V.ffn_bound(xs[t], np64(m.W1[e]), np64(m.W2[e]))
        w = p[t, k][:, None]
        ref[t] += w * v
        tol[t] += w * (b + (eps[t] + (m.K + 1) * 2.0 ** -24) * (np.abs(v) + b))
    if m.Fs:
        v, b = V.ffn_bound(xs, np64(m.Ws1), np64(m.Ws2))
        ref += v
        tol += b + (m.K + 1) * 2.0 ** -24 * (np.abs(v) + b)
    assert np.all(np.abs(y - ref) <= tol + 2.0 ** -8 * (np.abs(ref) + tol))


def check_i8(m, x, out):
    """Against moe_grouped_ffn_i8 on the same picks."""
    idx = out["topk_idx"].long()
    S, K = idx.shape
    p, eps = (torch.tensor(a, device=DEV) for a in check_picks(m, x, idx.cpu().numpy(), np64(out["topk_prob"])))
    order = torch.sort(idx.reshape(-1), stable=True).indices
    off = torch.zeros(m.E + 1, dtype=torch.int32, device=DEV)
    off[1:] = torch.bincount(idx.reshape(-1), minlength=m.E).cumsum(0)
    yd = layer.grouped_ffn_i8(x[order // K].contiguous(), off, m.w1, m.s1, m.w2, m.s2).double()
    rows = torch.empty_like(yd)
    rows[order] = yd
    terms = rows.view(S, K, -1) * p[..., None]
    ref, mag = terms.sum(1), terms.abs().sum(1)
    if m.Fs:
        off = torch.tensor([0, S], dtype=torch.int32, device=DEV)
        s = layer.grouped_ffn_i8(x, off, m.ws1[None], m.ss1[None], m.ws2[None], m.ss2[None]).double()
        ref, mag = ref + s, mag + s.abs()
    tol = mag * (2.0 ** -8 + eps + (K + 4) * 2.0 ** -24) + ref.abs() * 2.0 ** -8
    assert bool(((out["y"].double() - ref).abs() <= tol * (1 + 2.0 ** -7)).all())


SHAPES = [   # S, D, E, K, F, Fs, score
    (1, 16, 1, 1, 16, 0, "softmax"), (2, 64, 8, 8, 48, 0, "softmax"), (3, 272, 65, 5, 176, 0, "sigmoid"),
    (1, 2048, 64, 6, 1024, 0, "softmax"), (5, 672, 512, 22, 336, 0, "softmax"), (7, 336, 24, 3, 528, 400, "sigmoid"),
    (17, 1040, 16, 2, 272, 0, "softmax"), (33, 128, 4, 2, 1040, 64, "softmax"), (64, 256, 3, 2, 512, 256, "sigmoid"),
    (64, 512, 1, 1, 80, 0, "softmax"), (64, 144, 1024, 32, 32, 0, "softmax"), (49, 64, 130, 32, 96, 16, "sigmoid")]


@pytest.mark.parametrize("weights", ["bf16", "i8"])
@pytest.mark.parametrize("S, D, E, K, F, Fs, score", SHAPES)
def test_layer_few(S, D, E, K, F, Fs, score, weights):
    m = Model(D, E, K, F, Fs, score, weights, seed=S + E)
    x = m.tokens(S)
    out = m.layer(S)(x)
    (check_i8 if weights == "i8" else check_bf16)(m, x, out)


@pytest.mark.parametrize("D, F", [(8, 8), (24, 1000), (2696, 72)])
def test_sizes_of_bf16_alone(D, F):
    m = Model(D, 6, 2, F, Fs=40, seed=D)
    x = m.tokens(9)
    check_bf16(m, x, m.layer(9)(x))


@pytest.mark.parametrize("S", [12, 20])
@pytest.mark.parametrize("weights, D, F", [("bf16", 2048, 1024), ("bf16", 1040, 2048), ("i8", 2048, 1024),
                                           ("i8", 1040, 2048)])
def test_weights_past_the_last_level_cache(weights, D, F, S):
    """Weights over 256 MB are read another way, where their rows start on cache lines."""
    m = Model(D, 80, 8, F, seed=11, weights=weights)
    x = m.tokens(S)
    (check_i8 if weights == "i8" else check_bf16)(m, x, m.layer(S)(x))
    if D == 2048:   # the same weights off the cache lines: the same sums
        ref = {k: v.clone() for k, v in m.layer(S)(x).items()}
        for name in ("w1", "w2"):
            w = getattr(m, name)
            buf = torch.empty(w.numel() + 64, dtype=w.dtype, device=DEV)
            off = 16 // w.element_size()
            buf[off:off + w.numel()] = w.reshape(-1)
            setattr(m, name, buf[off:off + w.numel()].view(w.shape))
        for k, v in m.layer(S)(x).items():
            assert torch.equal(v, ref[k]), k


@pytest.mark.parametrize("S", [32, 48])
def test_wide_slabs_past_the_last_level_cache(S):
    """8-bit weights over 256 MB, and several rows an expert."""
    m = Model(2048, 80, 10, 1024, seed=12, weights="i8")
    x = m.tokens(S)
    check_i8(m, x, m.layer(S)(x))


@pytest.mark.parametrize("weights", ["bf16", "i8"])
def test_experts_past_4_gib(weights):
    """The last experts of a large layer give what they give as a small layer's."""
    D, F, E = 2048, 2080, 1024 if weights == "i8" else 520
    i8 = weights == "i8"
    g = torch.Generator(device=DEV).manual_seed(13)
    few = 4
    shapes = [(F, D), (D, F)] if i8 else [(D, F), (F, D)]
    small = [torch.randint(-127, 128, (few,) + s, generator=g, device=DEV).to(torch.int8 if i8 else BF16)
             for s in shapes]
    large = [torch.zeros((E,) + s, dtype=small[0].dtype, device=DEV) for s in shapes]
    for a, b in zip(large, small):
        a[-few:] = b
    past = (E - few) * F * D * large[0].element_size() > 2 ** 32
    assert past
    x = torch.randn((2, D), generator=g, device=DEV).to(BF16)
    sc = torch.rand((few, D), generator=g, device=DEV) if i8 else None

    def run(W, E):
        bias = torch.full((E,), float("-inf"), device=DEV)
        bias[-few:] = torch.arange(few, device=DEV).float()
        kw = dict(s1=torch.ones((E, F), device=DEV), s2=torch.zeros((E, D), device=DEV)) if i8 else {}
        if i8:
            kw["s2"][-few:] = sc
        return layer.LayerFew(2, torch.zeros((D, E), device=DEV), *W, 2, bias=bias, **kw)(x)

    a, b = run(large, E), run(small, few)
    assert torch.equal(a["topk_idx"], b["topk_idx"] + (E - few)) and torch.equal(a["topk_prob"], b["topk_prob"])
    assert torch.equal(a["y"], b["y"]) and bool((a["y"] != 0).any())


@pytest.mark.parametrize("weights", ["bf16", "i8"])
def test_a_layer_fed_with_its_own_output(weights):
    m = Model(272, 12, 3, 176, 64, weights=weights, seed=14)
    lf = m.layer(5)
    x = m.tokens(5)
    once = lf(x)["y"].clone()
    ref = {k: v.clone() for k, v in lf(once).items()}
    for k, v in lf(lf(x)["y"]).items():
        assert torch.equal(v, ref[k]), k


@pytest.mark.parametrize("weights", ["bf16", "i8"])
def test_fewer_tokens_than_the_layer_holds(weights):
    m = Model(144, 12, 3, 176, 64, "sigmoid", weights, seed=3)
    lf = m.layer(20)
    x = m.tokens(20)
    full = {k: v.clone() for k, v in lf(x).items()}
    for n in (0, 1, 2, 15, 16, 19):
        for v in lf.out.values():
            v.fill_(-3)
        out = lf(x[:n])
        assert out["y"].shape == (n, 144)
        assert bool((lf.out["y"][n:] == -3).all()) and bool((lf.out["topk_idx"][n:] == -3).all())
        assert torch.equal(out["topk_idx"], full["topk_idx"][:n])
        (check_i8 if weights == "i8" else check_bf16)(m, x[:n], out) if n else None


def test_ties_and_masked_experts():
    m = Model(64, 96, 4, 32, seed=4)
    m.Wr[:, 40] = m.Wr[:, 7]
    m.bias[40] = m.bias[7] = 9.0          # 7 and 40 tie at the top
    x = m.tokens(6)
    out = m.layer(6)(x)
    assert bool((out["topk_idx"][:, 0] == 7).all()) and bool((out["topk_idx"][:, 1] == 40).all())
    assert torch.equal(out["topk_prob"][:, 0], out["topk_prob"][:, 1])
    # all but K - 1 experts masked: the last pick is the lowest masked one, with weight 0
    m.bias.fill_(float("-inf"))
    m.bias[[3, 50, 95]] = 0.0
    out = m.layer(6)(x)
    idx = out["topk_idx"].cpu().numpy()
    assert (np.sort(idx[:, :3], 1) == [3, 50, 95]).all() and (idx[:, 3] == 0).all()
    assert bool((out["topk_prob"][:, 3] == 0).all())
    # zero tokens: every expert scores its bias
    m.bias.zero_()
    out = m.layer(6)(torch.zeros_like(x))
    assert (out["topk_idx"].cpu().numpy() == [0, 1, 2, 3]).all() and bool((out["y"] == 0).all())
    assert bool((out["topk_prob"] == 0.25).all())


@pytest.mark.parametrize("weights", ["bf16", "i8"])
def test_a_token_that_is_not_finite_stays_alone(weights):
    m = Model(64, 8, 2, 48, seed=5, weights=weights)
    lf = m.layer(8)
    x = m.tokens(8)
    clean = {k: v.clone() for k, v in lf(x).items()}
    x2 = x.clone()
    x2[3, 9] = float("inf")
    out = lf(x2)
    keep = torch.arange(8, device=DEV) != 3
    assert not bool(torch.isfinite(out["y"][3]).all())
    assert torch.equal(out["y"][keep], clean["y"][keep]) and torch.equal(out["topk_idx"][keep], clean["topk_idx"][keep])


@pytest.mark.parametrize("weights", ["bf16", "i8"])
def test_repeats_graphs_streams_and_two_layers(weights):
    m = Model(528, 20, 4, 272, 144, "sigmoid", weights, seed=6)
    xs = [m.tokens(11, s) for s in range(3)]
    lf = m.layer(11)
    ref = [{k: v.clone() for k, v in lf(x).items()} for x in xs]
    for x, r in zip(xs, ref):
        for k, v in lf(x).items():
            assert torch.equal(v, r[k]), k
    # two objects of the same weights at once, on two streams
    other = m.layer(11)
    torch.cuda.synchronize()
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(3):
        with torch.cuda.stream(a):
            oa = lf(xs[0])
        with torch.cuda.stream(b):
            ob = other(xs[1])
        torch.cuda.synchronize()
        assert torch.equal(oa["y"], ref[0]["y"]) and torch.equal(ob["y"], ref[1]["y"])
    # captured, replayed on new values with eager calls between
    buf = xs[0].clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = lf(buf)
    for x, r in zip(xs, ref):
        buf.copy_(x)
        for v in out.values():
            v.fill_(-5)
        graph.replay()
        torch.cuda.synchronize()
        for k, v in out.items():
            assert torch.equal(v, r[k]), k
        lf(xs[2])
        torch.cuda.synchronize()


def test_follows_the_training_layer():
    """The same weights and tokens through LayerFwd: the same picks, outputs within both paths' bf16 roundings."""
    m = Model(256, 16, 4, 512, seed=7)
    x = m.tokens(64)
    out = m.layer(64)(x)
    fwd = layer.LayerFwd(64, 256, 16, 4, 512)(x, m.Wr, m.W1, m.W2, bias=m.bias)
    assert torch.equal(out["topk_idx"], fwd["topk_idx"])
    a, b = out["y"].double(), fwd["y"].double()
    assert float((a - b).norm() / b.norm()) <= 2 * 2.0 ** -8    # three roundings of rms below 2^-9 on one side, two on the other
    check_bf16(m, x, out)


def test_serving_a_model_in_8_bits():
    """The path as a server runs it: weights quantised once, a prompt through the grouped
    FFN, then decode steps through the few-token layer; both agree on the last token."""
    m = Model(256, 16, 4, 512, seed=8, weights="i8")
    x = m.tokens(300)
    r = layer.route(layer.router_logits(x, m.Wr, m.bias), m.K)
    xd, p = layer.dispatch(x, r["topk_prob"], r["inv_perm"], m.K)
    yd = layer.grouped_ffn_i8(xd, r["offsets"], m.w1, m.s1, m.w2, m.s2)
    y = layer.combine(yd, p, r["inv_perm"], 300, m.K)
    lf = m.layer(4)
    for t in (0, 37, 296):
        out = lf(x[t:t + 4])
        assert torch.equal(out["topk_idx"], r["topk_idx"][t:t + 4])
        d = (out["y"].double() - y[t:t + 4].double()).norm() / y[t:t + 4].double().norm()
        assert float(d) <= 2 * 2.0 ** -8


def test_refusals_on_the_device():
    m = Model(32, 8, 2, 48)
    lf = m.layer(4)
    with pytest.raises(ValueError):
        lf(m.tokens(5))
    with pytest.raises(ValueError):
        lf(torch.zeros(4, 64, dtype=BF16, device=DEV))
    with pytest.raises(TypeError):
        lf(torch.zeros(4, 32, device=DEV))
    with pytest.raises(ValueError):
        lf(torch.zeros(32, 4, dtype=BF16, device=DEV).t())
    with pytest.raises(ValueError):
        m.layer(65)
    with pytest.raises(ValueError):
        layer.LayerFew(4, m.Wr, m.W1, m.W2, 2, sel_bias=m.bias, score="softmax")


def parts_bound(x, W1, W2):
    """(y, b) of one bf16 expert as serving_oracle.ffn_bound gives them, with h within 2^-16 and an fp32 rounding
    of itself and sums of its two parts."""
    x, W1, W2 = (np.asarray(a, np.float64) for a in (x, W1, W2))
    D, F = W1.shape
    u = np.maximum(x @ W1, 0.0)
    du = D * 2.0 ** -24 * (np.abs(x) @ np.abs(W1))
    h = u * u
    dh = 2 * u * du + du * du + (2.0 ** -16 + 2.0 ** -23) * (u + du) ** 2
    return h @ W2, dh @ np.abs(W2) + 2 * F * 2.0 ** -24 * ((h + dh) @ np.abs(W2))


@pytest.mark.parametrize("S, D, E, K, F, Fs, score", SHAPES)
def test_hidden_values_keep_more_than_bf16(S, D, E, K, F, Fs, score, monkeypatch):
    """With bf16 weights, y is one rounding to bf16 away from the fp32 layer's."""
    monkeypatch.setattr(V, "ffn_bound", parts_bound)
    m = Model(D, E, K, F, Fs, score, seed=S + E + 1)
    x = m.tokens(S)
    check_bf16(m, x, m.layer(S)(x))


def test_hidden_values_at_the_end_of_the_range():
    """Hidden values past the largest bf16 are finite where fp32 holds them; past fp32 they are infinite."""
    D = F = 16
    W1, W2 = torch.zeros((1, D, F), device=DEV), torch.zeros((1, F, D), device=DEV)
    W1[0, 0, 0] = W1[0, 1, 0] = W1[0, 3, 1] = 1.0
    W2[0, 0, 0], W2[0, 1, 1] = 2.0 ** -100, 1.0
    x = torch.zeros((2, D), device=DEV)
    x[0, 0], x[0, 1] = 2.0 ** 64, -2.0 ** 52      # h = 2^128 (1 - 2^-11 + 2^-24): fp32 holds it, bf16 rounds it up
    x[1, 3] = 2.0 ** 64                           # h = 2^128
    y = layer.LayerFew(2, torch.zeros((D, 1), device=DEV), W1.to(BF16), W2.to(BF16), 1)(x.to(BF16))["y"]
    assert float(y[0, 0]) == 2.0 ** 28 and not bool(y[0, 1:].any())
    assert float(y[1, 1]) == float("inf")


@pytest.mark.parametrize("S", [8, 32, 64])
@pytest.mark.parametrize("weights", ["bf16", "i8"])
def test_shared_expert_past_the_last_level_cache(weights, S):
    """Routed weights over 256 MB beside a shared expert whose own need not start on cache
    lines; experts that most tokens pick, so that 16, 32 and 64 rows stage their weights."""
    m = Model(2048, 80, 10, 1024, 1040, "sigmoid", weights, seed=15, bias_std=2.0)
    x = m.tokens(S)
    out = m.layer(S)(x)
    most = int(torch.bincount(out["topk_idx"].reshape(-1).long(), minlength=80).max())
    assert most > {8: 0, 32: 16, 64: 32}[S]
    (check_i8 if weights == "i8" else check_bf16)(m, x, out)


@pytest.mark.parametrize("weights", ["bf16", "i8"])
def test_rows_of_an_experts_weights_off_the_cache_lines(weights):
    """Rows that start on cache lines in one product and between them in the other (8 bits)."""
    m = Model(2048, 80, 10, 1088, 1040, weights=weights, seed=16, bias_std=2.0)
    x = m.tokens(48)
    (check_i8 if weights == "i8" else check_bf16)(m, x, m.layer(48)(x))


@pytest.mark.parametrize("weights", ["bf16", "i8"])
def test_output_over_the_tokens_it_came_from(weights):
    """y may be written over x, whole or shifted by rows."""
    m = Model(272, 12, 3, 176, 64, weights=weights, seed=17)
    lf = m.layer(6)
    x = m.tokens(6)
    first = lf(x)["y"].clone()
    for rows in (slice(1, 6), slice(2, 4), slice(0, 6)):
        ref = {k: v.clone() for k, v in m.layer(6)(first[rows].clone()).items()}
        lf(x)
        for k, v in lf(lf.out["y"][rows]).items():
            assert torch.equal(v, ref[k]), (rows, k)


@pytest.mark.parametrize("S, D, F, E, K, Fs", [(24, 1024, 1024, 16, 8, 0), (32, 1040, 1072, 24, 9, 80), (40, 1040, 1072, 24, 8, 80),
                                               (64, 1024, 1040, 17, 16, 0), (32, 2048, 2688, 26, 10, 0),
                                               (48, 2048, 2688, 26, 10, 144)])
def test_wide_slabs_of_many_rows_an_expert(S, D, F, E, K, Fs):
    """8-bit weights, twelve rows an expert or more, within and past the last-level cache."""
    assert S * K >= 12 * E
    m = Model(D, E, K, F, Fs, weights="i8", seed=S + E)
    x = m.tokens(S)
    check_i8(m, x, m.layer(S)(x))


def test_infinite_weights():
    """They give infinities, and NaN only where a hidden value is 0 or infinities of both signs meet."""
    D, F = 32, 24
    m = Model(D, 1, 1, F, seed=18)
    x = m.tokens(20)
    m.W1[0, :, 0] = 0.0                                            # h = 0
    x[:, 0], m.W1[0, :, 1] = 1.0, 0.0
    m.W1[0, 0, 1], m.W1[0, 0, 2] = 1.0, 0.75                       # h = 1: one part holds it
    for f, d, sign in ((0, 0, 1), (1, 1, 1), (2, 2, -1), (3, 3, 1), (1, 4, 1), (2, 4, -1)):
        m.W2[0, f, d] = sign * float("inf")
    y = np64(m.layer(20)(x)["y"])
    with np.errstate(invalid="ignore"):
        h = np.maximum(np64(x) @ np64(m.W1[0]), 0.0) ** 2
        terms = h[:, :, None] * np64(m.W2[0])
        ref = terms.sum(1)
    odd = ~np.isfinite(ref)
    assert np.isnan(ref[:, 0]).all() and (ref[:, 1] == np.inf).all() and (h[:, 3] > 2.0 ** -20).any()
    clear = (h[:, 3] == 0) | (h[:, 3] > 2.0 ** -20)                # elsewhere its sign hangs on a rounding
    assert np.array_equal(y[clear][odd[clear]], ref[clear][odd[clear]], equal_nan=True)
    assert np.isfinite(y[clear][~odd[clear]]).all()


@pytest.mark.parametrize("e", [-100, -110, -118, -122, -126])
def test_small_hidden_values(e):
    """Hidden values down to the smallest normal number: their second parts are subnormal."""
    D = F = 16
    W1, W2 = torch.zeros((1, D, F), device=DEV), torch.zeros((1, F, D), device=DEV)
    W1[0, 0, 0] = W1[0, 1, 0] = 1.0
    W2[0, 0, 0] = 2.0 ** 100
    x = torch.zeros((3, D), device=DEV)
    x[0, 0], x[0, 1] = 2.0 ** (e // 2), 2.0 ** (e // 2 - 9)       # h = 2^e (1 + 2^-9)^2
    x[1, 0] = 2.0 ** (e // 2)                                     # h = 2^e
    x[2, 0], x[2, 1] = 2.0 ** (e // 2), 2.0 ** (e // 2 - 3)       # h = 2^e (1 + 2^-2 + 2^-6), a bf16 value
    y = layer.LayerFew(3, torch.zeros((D, 1), device=DEV), W1.to(BF16), W2.to(BF16), 1)(x.to(BF16))["y"].double()
    # 1 + 2^-8 + 2^-18 is 2^-18 from the middle of the bf16 values 1 and 1 + 2^-7, and h is held to 2^-16: either is right
    assert float(y[0, 0]) in (2.0 ** (e + 100), 2.0 ** (e + 100) * (1 + 2.0 ** -7))
    assert float(y[1, 0]) == 2.0 ** (e + 100) and float(y[2, 0]) == 2.0 ** (e + 100) * (1 + 2.0 ** -2 + 2.0 ** -6)


@pytest.mark.parametrize("weights", ["bf16", "i8"])
@pytest.mark.parametrize("S, D, E, K, F, Fs", [(1, 64, 5, 2, 48, 0), (9, 272, 40, 7, 176, 80), (30, 144, 64, 12, 336, 16),
                                               (64, 528, 24, 8, 112, 272)])
def test_writes_its_buffers_only(S, D, E, K, F, Fs, weights):
    """A call without exported picks and without biases, in a workspace of just the size it asks
    for, among guard bytes; the workspace holds anything before."""
    m = Model(D, E, K, F, Fs, weights=weights, seed=19)
    x = m.tokens(S)
    kw = {k: v for k, v in m.kw.items() if k not in ("bias", "sel_bias", "score")}
    ref = {k: v.clone() for k, v in layer.LayerFew(S, m.Wr, m.w1, m.w2, K, **kw)(x).items()}
    mode = L.WEIGHTS_I8 if weights == "i8" else L.WEIGHTS_BF16
    n = L.moe_layer_few_workspace_bytes(L.layer_few_args(S, D, E, K, F, Fs, weights=mode))
    for fill in (0xFF, 0x00, 0x7F):
        ws = torch.full((n + 512,), fill, dtype=torch.uint8, device=DEV)
        y = torch.full((S + 2, D), -3.0, dtype=BF16, device=DEV)
        L.moe_layer_few(L.layer_few_args(S, D, E, K, F, Fs, weights=mode, ws=ws[256:256 + n], x=x, Wr=m.Wr, W1=m.w1,
                                         W2=m.w2, y=y[1:-1], **kw))
        assert torch.equal(y[1:-1], ref["y"])
        assert bool((y[0] == -3).all()) and bool((y[-1] == -3).all())
        assert bool((ws[:256] == fill).all()) and bool((ws[256 + n:] == fill).all())
