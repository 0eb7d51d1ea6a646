"""The serving oracle on values worked out by hand (CPU)."""
import numpy as np

from oracle import serving_oracle as V


def test_quant_rows_by_hand():
    x = np.array([[127.0, -127.0, 63.5, 0.5, 1.5, -0.5, -1.5, 0.0],
                  [2.0, 1.0, -1.0, 0.25, -2.0, 0.0, 0.0, 0.0],
                  [0.0] * 8, [np.inf] + [1.0] * 7, [np.nan] + [1.0] * 7])
    q, s = V.quant_rows(x)
    assert q[0].tolist() == [127, -127, 64, 0, 2, 0, -2, 0]      # ties to even
    assert q[1].tolist() == [127, 64, -64, 16, -127, 0, 0, 0]    # 63.5 -> 64, 15.875 -> 16
    assert not q[2:].any() and s[0] == 1 and s[1] == np.float32(2 / 127) and s[2] == 0
    assert np.isnan(s[3:]).all()


def test_a_quotient_is_a_tie_or_far_from_one():
    """What the kernel's rounding rests on: for bf16 values x and a (|x| <= a), 127 x / a
    is half way between integers or at least 2^-17 of itself away from that."""
    m = np.arange(128, 256, dtype=np.int64)
    worst = 1.0
    for shift in range(9):               # x = xm 2^-shift, a = am: smaller quotients round to zero
        num, den = 127 * m[:, None], m[None, :] << shift
        n = num // den                   # the tie below or above is n + 1/2
        off = np.abs(2 * num - (2 * n + 1) * den)    # |127 x / a - (n + 1/2)| 2 a
        keep = (num <= 127 * den) & (2 * num >= den) & (off > 0)
        worst = min(worst, (off / (2 * num))[keep].min())
    assert worst >= 2.0 ** -17, worst


def test_product_and_ffn_by_hand():
    W1 = np.array([[[1.0, -1.0], [2.0, 0.5]]])      # [1, Kd = 2, N = 2]
    q, s = V.quant_weights(W1)
    assert q.tolist() == [[[64, 127], [-127, 64]]] and s[0, 0] == np.float32(2 / 127)
    x = np.array([[127.0, 0.0]])
    W = np.array([[2.0, 4.0], [1.0, -3.0]])
    one = np.ones(2, np.float32)
    h, y = V.ffn_i8(x, W, one, W, one)
    # u = (254, 127); h = bf16(64516, 16129) = (64512, 16128); codes 127, 31.75 -> 32
    assert h.tolist() == [[64512.0, 16128.0]]
    sh = np.float64(np.float32(64512 / 127))
    assert y.tolist() == [[(2 * 127 + 4 * 32) * sh, (127 - 3 * 32) * sh]]
