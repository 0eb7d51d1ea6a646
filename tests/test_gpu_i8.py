"""8-bit rows, weights and products on the GPU against their definition in 64 bits.

Codes and scales are exact.  A product's sum is exact too; what is left is one
rounding of the sum to fp32, two fp32 multiplications (2^-24 each) and the one to
bf16 (2^-8), so |C - ref| <= |ref| (2^-8 + 2^-21) holds with room for their product.
"""
import numpy as np
import pytest
import torch

from gpu_helpers import check_guarded, guarded
from oracle import serving_oracle as V
from oracle.moe_oracle import round_bf16
from paper_2608_28511_amd import _lib as L
from paper_2608_28511_amd import layer

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16 = torch.bfloat16
ROUND = 2.0 ** -8 + 2.0 ** -21


def np64(t):
    return t.detach().cpu().double().numpy()


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def randn(g, *shape, std=1.0):
    return (torch.randn(shape, generator=g, device=DEV) * std).to(BF16)


def codes(g, *shape):
    return torch.randint(-127, 128, shape, generator=g, device=DEV, dtype=torch.int32).to(torch.int8)


def offsets_of(counts):
    return torch.tensor(np.concatenate([[0], np.cumsum(counts)]), dtype=torch.int32, device=DEV)


def same_quant(x, q, s):
    rq, rs = V.quant_rows(np64(x))
    assert np.array_equal(q.cpu().numpy().astype(np.float64), rq)
    assert np.array_equal(s.cpu().numpy(), rs, equal_nan=True)


@pytest.mark.parametrize("R, D", [(0, 16), (1, 16), (3, 48), (5, 512), (129, 2688), (7, 4096), (7, 4112), (2, 65536),
                                  (70001, 32)])
def test_quant_rows(R, D):
    x = randn(gen(R + D), R, D)
    if R > 2:
        x[R // 2] = 0
    q, s = layer.quant_rows_i8(x)
    same_quant(x, q, s)


@pytest.mark.parametrize("D", [64, 8192])
def test_quant_rows_borders(D):
    """Ties, the ends of bf16's range, subnormals, rows that are not finite."""
    x = randn(gen(1), 16, D)
    lo = torch.tensor(2.0 ** -133, dtype=torch.float64).to(BF16)
    big = torch.finfo(BF16).max
    x[0] = torch.arange(D, device=DEV).remainder(255).sub(127).div(2).to(BF16)   # multiples of 1/2
    x[0, 0] = 127
    x[1] = x[1].clamp(-1, 1)
    x[1, 0:8] = torch.tensor([1.0, 0.5, -0.5, 0.25, -1.0, 0.75, 0.125, -0.125])   # amax / 2 is a tie
    x[2] = lo
    x[3] = (torch.randint(0, 128, (D,), generator=gen(2), device=DEV) * 2.0 ** -126 / 128).to(BF16)   # subnormals
    x[4] = big
    x[5, ::3] = big
    x[6] = float("inf")
    x[7, D - 1] = float("-inf")
    x[8, 3] = float("nan")
    x[9] = -0.0
    x[10, 1:] = lo
    x[11, 5] = 2.0 ** 120
    q, s = layer.quant_rows_i8(x)
    same_quant(x, q, s)


def test_quant_rows_writes_its_rows_only():
    x = randn(gen(3), 37, 272)
    q = torch.full((41, 272), 99, dtype=torch.int8, device=DEV)
    buf, s = guarded((37,), torch.float32, DEV)
    L.moe_quant_rows_i8(x, 37, 272, q[2:39], s)
    assert bool((q[:2] == 99).all()) and bool((q[39:] == 99).all())
    check_guarded(buf, 2, "scale")
    same_quant(x, q[2:39], s)


@pytest.mark.parametrize("E, Kd, N", [(1, 16, 8), (3, 48, 72), (2, 272, 64), (5, 1040, 136)])
def test_quant_weights(E, Kd, N):
    W = randn(gen(E + N), E, Kd, N)
    W[0, :, 1] = 0
    W[-1, Kd // 2, 0] = float("inf")
    Wq, s = layer.quant_weights_i8(W)
    rq, rs = V.quant_weights(np64(W))
    assert np.array_equal(Wq.cpu().numpy().astype(np.float64), rq)
    assert np.array_equal(s.cpu().numpy(), rs, equal_nan=True)


def test_quant_weights_dense():
    W = randn(gen(9), 96, 40)
    Wq, s = layer.quant_weights_i8(W)
    W3, s3 = layer.quant_weights_i8(W[None])
    assert Wq.shape == (40, 96) and s.shape == (40,) and torch.equal(Wq, W3[0]) and torch.equal(s, s3[0])


# Segment lengths around the tile heights, none, one row; sizes that end inside a
# tile and inside a step; calls of one round of narrow tiles, of several rounds of
# 128-row tiles, and long ones on the 256-row tile.
GEMMS = [([0, 1, 0, 127, 128, 129, 300, 2], 48, 72), ([5], 16, 8), ([1, 1, 1], 2688, 264),
         ([40] * 60, 272, 1024), ([0, 2500, 0, 3001], 144, 2056), ([6000, 5500], 1040, 1032)]


@pytest.mark.parametrize("epilogue", [0, 1])
@pytest.mark.parametrize("counts, Kd, N", GEMMS)
def test_grouped_gemm_i8(counts, Kd, N, epilogue):
    g = gen(Kd + N)
    E, R = len(counts), sum(counts)
    A, W = codes(g, R, Kd), codes(g, E, N, Kd)
    sa = torch.rand(R, generator=g, device=DEV) + 0.5
    sw = torch.rand(E, N, generator=g, device=DEV) + 0.5
    off = offsets_of(counts)
    sched = layer.grouped_schedule(off, E, R)
    buf, C = guarded((R, N), BF16, DEV)
    layer.grouped_gemm_i8(A, sa, sched, W, sw, epilogue, out=C)
    check_guarded(buf, 2, "C")
    for e in range(E):
        a, b = int(off[e]), int(off[e + 1])
        if a == b:
            continue
        ref = (A[a:b].double() @ W[e].double().T) * sa[a:b, None].double() * sw[e].double()
        # the square doubles the relative error before its own rounding
        if epilogue:
            ref = ref.clamp_min(0) ** 2
        assert bool(((C[a:b].double() - ref).abs() <= ref.abs() * ROUND).all()), e


@pytest.mark.parametrize("M, Kd, N", [(0, 16, 8), (1, 16, 8), (5, 2688, 672), (16, 4096, 40), (17, 336, 1024),
                                      (32, 4096, 72), (31, 4080, 8), (32, 4112, 24), (33, 272, 104), (127, 48, 264),
                                      (129, 1040, 72), (4100, 336, 1024), (9000, 2064, 1288)])
def test_latent_proj_i8(M, Kd, N):
    g = gen(M + N)
    A, W = randn(g, M, Kd), randn(g, Kd, N, std=Kd ** -0.5)
    if M > 4:
        A[M // 2] = 0
        A[1, 7] = float("nan")
    Wq, sw = layer.quant_weights_i8(W)
    C = layer.latent_proj_i8(A, Wq, sw)
    q, sx = layer.quant_rows_i8(A)
    ref = (q.double() @ Wq.double().T) * sx.double()[:, None] * sw.double()
    bad = torch.isnan(ref)
    assert torch.equal(torch.isnan(C), bad)     # the row that is not finite, and it alone
    assert bool(((C.double() - ref).abs() <= ref.abs() * ROUND)[~bad].all())
    # and through grouped_gemm_i8 without a schedule
    assert torch.equal(layer.grouped_gemm_i8(q, sx, None, Wq[None], sw[None], 0).view(torch.int16), C.view(torch.int16))


# Up to a round of workgroups of 16, 32 and 64 columns of 32 rows, and past it.
@pytest.mark.parametrize("M, Kd, N", [(200, 2688, 672), (300, 2688, 680), (700, 2688, 672), (740, 2688, 672),
                                      (384, 4096, 664), (250, 4080, 1024), (8192, 256, 24), (4096, 272, 56),
                                      (4097, 1040, 40), (257, 240, 1000), (100, 1024, 4096), (30, 512, 16384)])
def test_latent_proj_i8_of_some_rows(M, Kd, N):
    test_latent_proj_i8(M, Kd, N)


def ffn_inputs(counts, D, F, seed):
    g = gen(seed)
    E, R = len(counts), sum(counts)
    W1q, s1 = layer.quant_weights_i8(randn(g, E, D, F, std=D ** -0.5))
    W2q, s2 = layer.quant_weights_i8(randn(g, E, F, D, std=F ** -0.5))
    return randn(g, R, D), offsets_of(counts), W1q, s1, W2q, s2


FEW_ROWS = [[0] * 30 + [129] + [1] * 5 + [33, 0, 64, 0, 0, 2], [16] * 7 + [17] + [0] * 9 + [32, 5, 8],
            [0] * 90 + [700], [1] * 300, [12] * 5, [96, 31, 0, 0, 0, 97, 1, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0]]


@pytest.mark.parametrize("epilogue", [0, 1])
@pytest.mark.parametrize("Kd, N", [(16, 8), (272, 104), (1040, 40), (2048, 72)])
@pytest.mark.parametrize("counts", FEW_ROWS)
def test_experts_of_few_rows(counts, Kd, N, epilogue):
    """Few rows an expert on average, some with many: other kernels than for more."""
    assert sum(counts) <= 12 * len(counts)
    test_grouped_gemm_i8(counts, Kd, N, epilogue)


@pytest.mark.parametrize("D, F", [(2048, 1024), (1040, 2064)])
def test_experts_of_few_rows_past_the_last_level_cache(D, F):
    """Their weights over 256 MB are read another way, where their rows start on cache lines.  The same rows
    among as many more as take them to the tiles of larger calls give the same."""
    E = 80
    counts = [(7 * e) % 23 for e in range(E)]
    x, offsets, W1q, s1, W2q, s2 = ffn_inputs(counts, D, F, 31)
    y = layer.grouped_ffn_i8(x, offsets, W1q, s1, W2q, s2)
    more = torch.cat([x, randn(gen(32), 2000, D)])
    off = torch.cat([offsets[:-1], offsets[-1:] + 2000])
    z = layer.grouped_ffn_i8(more, off, W1q, s1, W2q, s2)
    assert sum(counts) <= 12 * E and 20 * E < len(more)
    assert torch.equal(y, z[:len(x)])


@pytest.mark.parametrize("D, F", [(1040, 1096), (2048, 1024)])
def test_experts_of_some_rows_and_large_weights(D, F):
    """13 to 20 rows an expert on average, weights of 64 to 128 and past 128 MB; against the tiles of larger calls."""
    for E, per in ((64, 14), (80, 19)):
        counts = [(11 * e) % (2 * per) for e in range(E)]
        x, offsets, W1q, s1, W2q, s2 = ffn_inputs(counts, D, F // 16 * 16, 41)
        assert 12 * E < sum(counts) <= 20 * E and E * D * F > 2 ** 26
        more = torch.cat([x, randn(gen(42), 20 * E, D)])
        off = torch.cat([offsets[:-1], offsets[-1:] + 20 * E])
        y = layer.grouped_ffn_i8(x, offsets, W1q, s1, W2q, s2)
        assert torch.equal(y, layer.grouped_ffn_i8(more, off, W1q, s1, W2q, s2)[:len(x)])


def test_few_rows_leave_the_rows_behind_them():
    counts = [3, 0, 33, 1]
    x, offsets, W1q, s1, W2q, s2 = ffn_inputs(counts, 48, 80, 33)
    R, q = 45, layer.quant_rows_i8(torch.cat([x, x[:8]]))
    C = torch.full((R, 80), -7.0, dtype=BF16, device=DEV)
    layer.grouped_gemm_i8(*q, layer.grouped_schedule(offsets, 4, R), W1q, s1, 1, out=C)
    assert bool((C[37:] == -7).all()) and not bool((C[:37] == -7).any())


FFNS = [([1], 16, 16), ([0, 1, 0, 0], 48, 80), ([3, 0, 200, 129, 1], 272, 336), ([700, 2, 0, 1500], 512, 1040),
        ([0, 4000, 3500, 0], 2064, 1024)]


@pytest.mark.parametrize("counts, D, F", FFNS)
def test_grouped_ffn_i8_is_its_steps(counts, D, F):
    x, off, W1q, s1, W2q, s2 = ffn_inputs(counts, D, F, 5)
    R, E = x.shape[0], len(counts)
    y = layer.grouped_ffn_i8(x, off, W1q, s1, W2q, s2)
    sched = layer.grouped_schedule(off, E, R)
    q, sx = layer.quant_rows_i8(x)
    h = layer.grouped_gemm_i8(q, sx, sched, W1q, s1, 1)
    hq, sh = layer.quant_rows_i8(h)
    assert torch.equal(y, layer.grouped_gemm_i8(hq, sh, sched, W2q, s2, 0))
    assert torch.equal(y, layer.grouped_ffn_i8(x, off, W1q, s1, W2q, s2))
    # each step against 64 bits
    for e in range(E):
        a, b = int(off[e]), int(off[e + 1])
        if a == b:
            continue
        u = (q[a:b].double() @ W1q[e].double().T) * sx[a:b, None].double() * s1[e].double()
        ref = u.clamp_min(0) ** 2
        assert bool(((h[a:b].double() - ref).abs() <= ref * ROUND).all())
        ref = (hq[a:b].double() @ W2q[e].double().T) * sh[a:b, None].double() * s2[e].double()
        assert bool(((y[a:b].double() - ref).abs() <= ref.abs() * ROUND).all())
    same_quant(x, q, sx)
    same_quant(h, hq, sh)


def test_grouped_ffn_i8_exact_hidden():
    """Small integers: every value up to h is exact on both sides, so y is the oracle's
    up to its own roundings."""
    rng = np.random.default_rng(3)
    D, F, E, R = 64, 96, 2, 150
    x = rng.integers(-3, 4, (R, D)).astype(np.float64)
    x[:, 0] = 127                                        # scale 1
    W1 = rng.integers(-1, 2, (E, F, D)).astype(np.float64)
    W1[:, :, 0] = 0                                      # |u| <= 63 * 3, u^2 < 2^16
    W2 = rng.integers(-127, 128, (E, D, F)).astype(np.float64)
    s1, s2 = np.full((E, F), 0.5, np.float32), np.full((E, D), 0.25, np.float32)
    counts = [90, 60]
    t = lambda a, d: torch.tensor(a, device=DEV).to(d)  # noqa: E731
    y = layer.grouped_ffn_i8(t(x, BF16), offsets_of(counts), t(W1, torch.int8), t(s1, torch.float32),
                             t(W2, torch.int8), t(s2, torch.float32))
    at = 0
    for e, n in enumerate(counts):
        _, ref = V.ffn_i8(x[at:at + n], W1[e], s1[e], W2[e], s2[e])
        assert np.all(np.abs(np64(y[at:at + n]) - ref) <= np.abs(ref) * ROUND)
        at += n
    assert np.array_equal(round_bf16(np64(y)), np64(y))


def test_rows_past_4_gib():
    """The last rows of a call give what they give alone."""
    R, D, N = 530_003, 8192, 16
    g = torch.Generator(device=DEV).manual_seed(21)
    tail = torch.randn((300, D), generator=g, device=DEV).to(BF16)
    x = torch.zeros((R, D), dtype=BF16, device=DEV)
    x[-300:] = tail
    q, scale = layer.quant_rows_i8(x)
    qt, st = layer.quant_rows_i8(tail)
    past = q.numel() > 2 ** 32
    assert past and torch.equal(q[-300:], qt) and torch.equal(scale[-300:], st)
    assert not bool(scale[:-300].any())
    W = torch.randn((2, D, N), generator=g, device=DEV).to(BF16)
    Wq, ws = layer.quant_weights_i8(W)
    off = torch.tensor([0, R - 150, R], dtype=torch.int32, device=DEV)
    y = layer.grouped_gemm_i8(q, scale, layer.grouped_schedule(off, 2, R), Wq, ws, 0)
    for e, part in ((0, slice(0, 150)), (1, slice(150, 300))):
        ref = layer.grouped_gemm_i8(qt[part].contiguous(), st[part].contiguous(), None, Wq[e:e + 1], ws[e:e + 1], 0)
        assert torch.equal(y[R - 300:][part], ref)
    assert not bool(y[:-300].any())
    assert torch.equal(layer.latent_proj_i8(x, Wq[0], ws[0])[-300:], layer.latent_proj_i8(tail, Wq[0], ws[0]))


def test_rows_that_are_not_finite_stay_alone():
    x, off, W1q, s1, W2q, s2 = ffn_inputs([100, 0, 57], 64, 128, 6)
    clean = layer.grouped_ffn_i8(x, off, W1q, s1, W2q, s2)
    x2 = x.clone()
    x2[3, 5], x2[120, 0] = float("nan"), float("inf")
    y = layer.grouped_ffn_i8(x2, off, W1q, s1, W2q, s2)
    bad = torch.zeros(157, dtype=torch.bool, device=DEV)
    bad[3] = bad[120] = True
    assert bool(torch.isnan(y[bad]).all()) and torch.equal(y[~bad], clean[~bad])


def test_captured_and_on_another_stream():
    x, off, W1q, s1, W2q, s2 = ffn_inputs([33, 0, 290, 5], 272, 176, 7)
    Wq, sw = layer.quant_weights_i8(randn(gen(8), 272, 40))
    xs = x.clone()
    eager = [(layer.grouped_ffn_i8(v, off, W1q, s1, W2q, s2).clone(), layer.latent_proj_i8(v, Wq, sw).clone())
             for v in (x, -x, 2 * x)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        a, b = layer.grouped_ffn_i8(xs, off, W1q, s1, W2q, s2), layer.latent_proj_i8(xs, Wq, sw)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(a, eager[0][0]) and torch.equal(b, eager[0][1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a, b = layer.grouped_ffn_i8(xs, off, W1q, s1, W2q, s2), layer.latent_proj_i8(xs, Wq, sw)
    for v, (ra, rb) in zip((x, -x, 2 * x), eager):
        xs.copy_(v)
        a.fill_(float("nan"))
        b.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(a, ra) and torch.equal(b, rb)
        layer.grouped_ffn_i8(x, off, W1q, s1, W2q, s2)   # eager work between the replays


def test_refusals_on_the_device():
    x, off, W1q, s1, W2q, s2 = ffn_inputs([4], 32, 48, 8)
    with pytest.raises(ValueError):
        layer.grouped_ffn_i8(x[:, :16], off, W1q, s1, W2q, s2)
    with pytest.raises(ValueError):
        layer.grouped_ffn_i8(x.t().contiguous().t(), off, W1q, s1, W2q, s2)     # not contiguous
    with pytest.raises(TypeError):
        layer.grouped_ffn_i8(x.float(), off, W1q, s1, W2q, s2)
    with pytest.raises(L.MoeError):
        layer.quant_rows_i8(torch.zeros(2, 24, dtype=BF16, device=DEV))


@pytest.mark.parametrize("E, Kd, N", [(64, 272, 104), (100, 1040, 40), (256, 128, 72)])
def test_one_expert_with_every_row(E, Kd, N):
    """The largest calls that are taken for few rows an expert, all of them with one."""
    counts = [0] * E
    counts[E // 3] = 20 * E
    test_grouped_gemm_i8(counts, Kd, N, 1)
