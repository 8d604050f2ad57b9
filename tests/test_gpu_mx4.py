"""The MX4 operators on the GPU against plain forms in 64 bits."""
import numpy as np
import pytest
import torch

from oracle import mx4_oracle as X
from oracle import ot_oracle as O
from paper_2406_18832_amd import ot

pytestmark = pytest.mark.gpu

# One fp16 rounding of Y: half a unit, 2^-11 of the value (2^-25 below the
# normal range).  The sum in fp32: products are exact (two levels of 2 bits and
# powers of two), so only additions round, each by at most 2^-24 of a partial sum
# that stays below S = sum |x w| + |b'|.  K channels and the bias take at most K
# additions whatever their order; the matrix unit may truncate rather than round,
# which doubles the step.
def y_tolerance(y, mags, K):
    return np.maximum(np.abs(y) * 2.0 ** -11, 2.0 ** -25) + (K + 1) * 2.0 ** -23 * mags


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def host(t):
    return t.cpu().numpy()


def draw_activations(r, M, K):
    x = r.standard_normal((M, K)).astype(np.float32)
    x[:, r.integers(0, K, max(1, K // 100))] *= 50
    z = r.uniform(-3, 3, K).astype(np.float32)
    inv_s = np.float32(1) / r.uniform(0.1, 2, K).astype(np.float32)
    return x.astype(np.float16), z, inv_s


# rows, channels: one row and one block; ragged tails of a K tile and of a wave's
# 512 channels; rows in groups of 1, 2 and 8 per wave
SHAPES = [(1, 32), (1, 64), (3, 96), (5, 256), (7, 288), (2, 512), (9, 544), (33, 768), (64, 1056),
          (130, 4128), (700, 2016), (2100, 2080)]


@pytest.mark.parametrize("M,K", SHAPES)
@pytest.mark.parametrize("sym", [True, False])
def test_quantize_codes_and_scales(M, K, sym):
    r = np.random.default_rng([M, K, sym])
    x, z, inv_s = draw_activations(r, M, K)
    x[r.integers(0, M), :32] = 0  # an empty block (without symmetrization)
    a = (z, inv_s) if sym else (None, None)
    c, e = X.to_mx4(X.activations(x, *a))
    # what a call must not leave: stale scales past K
    Xc, Xe = torch.full((M, K // 2), 0x5A, dtype=torch.uint8, device="cuda"), \
        torch.full(((K + 255) // 256, M, 8), 0x5A, dtype=torch.uint8, device="cuda")
    ot.ot_quantize_act_mx4(dev(x), *(None if v is None else dev(v) for v in a), Xc, Xe)
    assert np.array_equal(host(Xe), e)
    assert np.array_equal(host(Xc), c)
    assert np.array_equal(host(ot.dequantize_mx4(Xc, Xe)), X.values(c, e).astype(np.float32))


def test_quantize_every_level_tie_and_neighbour():
    """Every level, halfway point and its fp32 neighbours, over exponents from
    the smallest fp16 subnormal to the largest value, with both signs."""
    t = np.concatenate([X.LEVELS, X.HALFWAY, np.nextafter(X.HALFWAY.astype(np.float32), 0),
                        np.nextafter(X.HALFWAY.astype(np.float32), 9), [7.0, 7.75, 6.5, 5.5]])
    t = np.concatenate([t, -t]).astype(np.float32)
    rows = []
    for e in range(-120, 121, 5):
        for lead in (4.0, 6.0, 7.9):
            for i in range(0, t.size, 31):
                row = np.zeros(32, dtype=np.float32)
                row[0] = lead
                part = t[i:i + 31]
                row[1:1 + part.size] = part
                rows.append(np.ldexp(row, e))
    v = np.stack(rows)
    M, K = v.shape
    # x = 0 and z = -v put the values there: fp32(0 - z) * 1 (a +0 for v = -0)
    c, s = X.to_mx4(X.activations(np.zeros((M, K), np.float16), -v, np.ones((M, K), np.float32)))
    z = dev(-v.reshape(-1))
    x = torch.zeros((1, M * K), dtype=torch.float16, device="cuda")
    Xc, Xe = ot.quantize_act_mx4(x, z, torch.ones(M * K, device="cuda"))
    assert np.array_equal(host(Xc).reshape(M, K // 2), c)
    got = host(Xe).transpose(1, 0, 2).reshape(-1)[:M]
    assert np.array_equal(got, s[0, :, 0])


def test_quantize_non_finite_blocks():
    """A NaN or an infinity, of the input or of the symmetrization, makes its
    block NaN and no other."""
    x = np.ones((3, 96), dtype=np.float16)
    x[0, 5], x[1, 40], x[2, 95] = np.nan, np.inf, -np.inf
    inv_s = np.ones(96, dtype=np.float32)
    inv_s[33] = 3e38
    x[2, 33] = 60000
    Xc, Xe = ot.quantize_act_mx4(dev(x), dev(np.zeros(96, np.float32)), dev(inv_s))
    v = host(ot.dequantize_mx4(Xc, Xe))
    bad = np.isnan(v).reshape(3, 3, 32)
    assert np.array_equal(bad.all(2), bad.any(2))
    assert np.array_equal(bad.any(2), [[1, 0, 0], [0, 1, 0], [0, 1, 1]])
    c, e = X.to_mx4(X.activations(x, np.zeros(96, np.float32), inv_s))
    assert np.array_equal(host(Xe), e) and np.array_equal(host(Xc), c)


@pytest.mark.parametrize("M,K", [(1, 32), (2, 64), (5, 288), (8, 5120), (3, 9248), (1030, 1056),
                                 (40, 20512), (2, 50176), (2100, 17408 + 1024)])
def test_ln_quantize(M, K):
    r = np.random.default_rng([M, K, 3])
    h = (r.standard_normal((M, K)) * r.uniform(0.5, 2, K) + r.standard_normal(K)).astype(np.float16)
    if M > 1:
        h[1] -= h[1].mean(dtype=np.float64).astype(np.float16)
        h[0, ::2], h[0, 1::2] = 1.0, -1.0  # a mean of exactly 0
    gamma = r.uniform(0.5, 1.5, K).astype(np.float16)
    beta = (r.standard_normal(K) * 0.2).astype(np.float16)
    z = (r.standard_normal(K) * 0.2).astype(np.float32)
    inv_s = r.uniform(0.5, 2, K).astype(np.float32)
    rows = slice(None) if M <= 64 else np.r_[0:8, M - 8:M]
    f = np.float32
    mean, var = O.layernorm_stats(h[rows])
    rstd = 1 / np.sqrt(var + float(f(1e-5)))
    n = (h[rows].astype(f) - mean.astype(f)[:, None]) * rstd.astype(f)[:, None]
    v = (n * gamma.astype(f) + (beta.astype(f) - z)) * inv_s
    c, e = X.to_mx4(v)
    Xc, Xe = torch.full((M, K // 2), 0x5A, dtype=torch.uint8, device="cuda"), \
        torch.full(((K + 255) // 256, M, 8), 0x5A, dtype=torch.uint8, device="cuda")
    ot.ot_ln_quantize_act_mx4(*map(dev, (h, gamma, beta)), 1e-5, dev(z), dev(inv_s), Xc, Xe)
    assert np.array_equal(host(Xe)[:, rows], e)
    assert np.array_equal(host(Xc)[rows], c)


@pytest.mark.parametrize("N,K", [(1, 32), (2, 96), (5, 256), (31, 544), (33, 2048), (70, 2080),
                                 (256, 4128), (6, 20480)])
@pytest.mark.parametrize("how", ["all", "no z", "no s", "no bias", "none"])
def test_fold(N, K, how):
    r = np.random.default_rng([N, K])
    W = (r.standard_normal((N, K)) * 0.02).astype(np.float16)
    W[0, :32] = 0
    b = None if how in ("no bias", "none") else r.standard_normal(N).astype(np.float16)
    z = None if how in ("no z", "none") else r.uniform(-3, 3, K).astype(np.float32)
    s = None if how in ("no s", "none") else r.uniform(0.01, 20, K).astype(np.float32)
    c, e, bias = X.fold(W, b, z, s)
    Wc, We, bp = ot.fold_weights_mx4(dev(W), *(None if v is None else dev(v) for v in (b, z, s)))
    assert np.array_equal(host(We), e) and np.array_equal(host(Wc), c)
    # a float64 sum of K exact products, then one rounding to fp32 (2^-24)
    mags = np.abs(W.astype(np.float64)) @ np.abs(z.astype(np.float64)) if z is not None else 0.0
    assert np.all(np.abs(host(bp) - bias) <= 2.0 ** -24 * np.abs(bias) * 1.01 + 2.0 ** -52 * K * mags)
    assert np.array_equal(host(ot.pack_weights_mx4(Wc, We)), X.pack(c, e))


@pytest.mark.parametrize("where", ["weight", "product", "bias"])
def test_fold_refuses_non_finite(where):
    W = torch.full((5, 64), 0.5, dtype=torch.float16, device="cuda")
    b = torch.zeros(5, dtype=torch.float16, device="cuda")
    s = torch.ones(64, device="cuda")
    if where == "weight":
        W[3, 63] = float("nan")
    elif where == "product":
        W[4, 0], s[0] = 60000.0, 1e36
    else:
        b[2] = float("inf")
    with pytest.raises(ot.OTError) as err:
        ot.fold_weights_mx4(W, b, None, s)
    assert err.value.code == ot.OT_ENONFINITE


def draw_mx4(r, rows, K, spread=3):
    """Random codes and scales (blocks of different magnitudes, some empty)."""
    c = r.integers(0, 256, (rows, K // 2), dtype=np.uint8)
    tiles = -(-K // 256)
    e = np.zeros((tiles, rows, 8), dtype=np.uint8)
    for i in range(K // 32):
        e[i // 8, :, i % 8] = r.integers(124 - spread, 124 + spread, rows)
    if rows > 2:
        c[rows // 2] = 0
    return c, e


LINEARS = [(1, 1, 32), (1, 33, 64), (2, 16, 96), (16, 768, 768), (17, 100, 288), (5, 4100, 5120),
           (32, 65, 2080), (33, 200, 1056), (64, 513, 4128), (8, 64, 36864),
           (65, 1, 32), (65, 70, 96), (100, 130, 288), (131, 615, 4128), (128, 128, 256),
           (129, 257, 512), (300, 1000, 1056), (513, 2050, 544), (1000, 3000, 800),
           (2048, 4096, 2048),
           # 32 rows to a workgroup: more than 16 x 256 channels
           (1, 4128, 4352), (16, 4100, 5120), (17, 4100, 288), (32, 4097, 2304), (40, 4100, 544),
           (64, 4099, 2080), (40, 8300, 96), (64, 8193, 800),
           # each tile's own sizes, ragged (TILES)
           (4000, 8000, 320), (2000, 12250, 96), (1100, 7700, 160), (500, 5100, 1056),
           (128, 9000, 96), (2830, 5637, 288), (906, 8330, 800), (1628, 1167, 64), (264, 6535, 64),
           (1035, 7173, 64), (407, 8425, 64), (69, 8347, 64)]

TILES = {(2000, 12250, 96): "256x128", (906, 8330, 800): "192x256", (1035, 7173, 64): "256x256",
         (2830, 5637, 288): "192x128", (264, 6535, 64): "128x128", (1628, 1167, 64): "64x128",
         (69, 8347, 64): "128x64", (300, 1000, 1056): "64x64"}


def test_each_tile_has_its_sizes():
    for sizes, tile in TILES.items():
        assert sizes in LINEARS and ot.ot_qlinear_mx4_plan(*sizes) == "tiles " + tile


@pytest.mark.parametrize("M,N,K", LINEARS)
def test_linear(M, N, K):
    r = np.random.default_rng([M, N, K])
    xc, xe = draw_mx4(r, M, K)
    wc, we = draw_mx4(r, N, K)
    bias = r.standard_normal(N).astype(np.float32)
    y, mags = X.linear(X.values(xc, xe), X.values(wc, we), bias)
    Wp = ot.pack_weights_mx4(dev(wc), dev(we))
    Y = torch.full((M, N), float("nan"), dtype=torch.float16, device="cuda")
    ot.ot_qlinear_mx4(dev(xc), dev(xe), Wp, N, dev(bias), Y,
                      ot.qlinear_mx4_workspace_for(M, N, K))
    assert np.all(np.abs(host(Y).astype(np.float64) - y) <= y_tolerance(y, mags, K))


def draw_moe(r, M, H, F, E, act):
    F1 = 2 * F if act == "swiglu" else F
    x = draw_mx4(r, M, H, 1)
    logits = (r.standard_normal((M, E)) * 2).astype(np.float16)
    w1, w2 = draw_mx4(r, E * F1, H, 1), draw_mx4(r, E * H, F, 1)
    b1, b2 = (r.standard_normal((E, n)).astype(np.float32) for n in (F1, H))
    return x, logits, w1, b1, w2, b2


def run_moe(x, logits, k, w1, b1, w2, b2, F, act):
    return ot.moe_mx4(dev(x[0]), dev(x[1]), dev(logits), k, ot.pack_weights_mx4(*map(dev, w1)),
                      None if b1 is None else dev(b1), ot.pack_weights_mx4(*map(dev, w2)),
                      None if b2 is None else dev(b2), F, act)


# draw_mx4(spread 1) gives scales of 2^-4 and 2^-3, so fc1's products are multiples
# of 2^-10 and its sums below 2^24 of those units: exact in fp32 in any order.  Then
# g takes one rounding (the bias), and silu(gate) * up a few of fp32 and those of
# exp.  A hidden value that close to a halfway point may take the other code: a step
# of at most 2 scales.  The tolerance lets every such value move by its whole step.
def moe_expected(x, logits, k, w1, b1, w2, b2, F, act):
    H, E = x[0].shape[1] * 2, logits.shape[1]
    xv = X.values(*x)
    w1v, w2v = X.values(*w1).reshape(E, -1, H), X.values(*w2).reshape(E, H, F)
    y, hidden = X.moe(xv, logits, k, w1v, b1, w2v, b2, act)
    tol = np.maximum(np.abs(y) * 2.0 ** -11, 2.0 ** -25)
    for (m, j), h in hidden.items():
        e = X.top_k(logits[m:m + 1], k)[0, j]
        assert (np.abs(w1v[e]) @ np.abs(xv[m])).max() < 2.0 ** 14
        g = w1v[e] @ xv[m] + (b1[e] if b1 is not None else 0)
        g_err = 2.0 ** -24 * np.abs(g)
        if act == "relu":
            err = g_err
        else:
            err = 1.1 * g_err[:F] * np.abs(g[F:]) + np.abs(g[:F]) * g_err[F:] + 2.0 ** -20 * np.abs(h)
        scale = np.ldexp(1.0, X.scale_bytes(h.astype(np.float32).reshape(-1, 32)).astype(int) - 127)
        scale = np.repeat(scale, 32)
        t = np.abs(h) / scale
        near = np.abs(t[:, None] - X.HALFWAY).min(1) * scale <= err + 2.0 ** -24 * np.abs(h)
        step = np.where(near, 2 * scale, 0.0)
        q = np.abs(X.values(*X.to_mx4(h[None].astype(np.float32)))[0])
        tol[m] += np.abs(w2v[e]) @ step + (F * k + 8) * 2.0 ** -23 * (
            np.abs(w2v[e]) @ q + (np.abs(b2[e]) if b2 is not None else 0))
    return y, tol


MOES = [(1, 32, 32, 1, 1), (1, 256, 512, 8, 2), (2, 96, 288, 4, 2), (3, 544, 96, 70, 8),
        (16, 512, 256, 4, 4), (17, 288, 544, 3, 2), (33, 256, 96, 2, 2), (64, 64, 32, 1, 1),
        (64, 512, 352, 32, 4), (64, 96, 64, 256, 16), (40, 2048, 1408, 5, 1)]


@pytest.mark.parametrize("M,H,F,E,k", MOES)
@pytest.mark.parametrize("act", ["relu", "swiglu"])
def test_moe(M, H, F, E, k, act):
    r = np.random.default_rng([M, H, F, E, k])
    x, logits, w1, b1, w2, b2 = draw_moe(r, M, H, F, E, act)
    y, tol = moe_expected(x, logits, k, w1, b1, w2, b2, F, act)
    assert np.median(tol) <= 0.05 * np.sqrt(np.mean(y * y))  # the bound says something
    got = host(run_moe(x, logits, k, w1, b1, w2, b2, F, act)).astype(np.float64)
    assert np.all(np.abs(got - y) <= tol)


@pytest.mark.parametrize("by_choice", [True, False])
def test_moe_ties_and_logits_that_choose_nothing(by_choice):
    """Equal logits (also 0 and -0) go to the lower expert; -inf and NaN are not
    chosen; a token with nothing else gets zeros; +inf takes all the weight."""
    M, H, F, E, k = (3, 64, 64, 40, 3) if by_choice else (8, 64, 64, 9, 3)
    r = np.random.default_rng(11)
    x, logits, w1, b1, w2, b2 = draw_moe(r, M, H, F, E, "relu")
    logits[0] = 1.0
    logits[0, 1] = 0.5
    logits[1] = -np.inf
    logits[1, E - 1] = -7.0
    logits[2] = np.nan
    if not by_choice:
        logits[3, ::2], logits[3, 1::2] = -0.0, 0.0
        logits[4] = -np.inf
        logits[5, 2:4] = np.inf
        logits[6] = np.nan
        logits[6, 4] = -65504
    y, tol = moe_expected(x, logits, k, w1, b1, w2, b2, F, "relu")
    got = host(run_moe(x, logits, k, w1, b1, w2, b2, F, "relu")).astype(np.float64)
    assert np.all(np.abs(got - y) <= tol)
    assert not got[2].any() and got[1].any()


def test_moe_without_biases_and_twice():
    r = np.random.default_rng(5)
    args = draw_moe(r, 6, 288, 160, 8, "swiglu")
    x, logits, w1, _, w2, _ = args
    y, tol = moe_expected(x, logits, 2, w1, None, w2, None, 160, "swiglu")
    a = run_moe(x, logits, 2, w1, None, w2, None, 160, "swiglu")
    assert np.all(np.abs(host(a).astype(np.float64) - y) <= tol)
    assert torch.equal(a, run_moe(x, logits, 2, w1, None, w2, None, 160, "swiglu"))
