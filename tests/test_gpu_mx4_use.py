"""The MX4 operators as they are used: one after another, in captured graphs, on
other streams, with shared and split K, in buffers with neighbours."""
import numpy as np
import pytest
import torch

from oracle import mx4_oracle as X
from paper_2406_18832_amd import ot, quality, synth
from tests.test_gpu_mx4 import (dev, draw_activations, draw_moe, draw_mx4, host, moe_expected,
                                y_tolerance)

pytestmark = pytest.mark.gpu

NAN16 = float("nan")


def guarded(rows, cols, dtype, extra=64):
    """A contiguous [rows, cols] view of a buffer of a fixed byte, and a check that
    the buffer's rest still holds it."""
    size = torch.empty((), dtype=dtype).element_size()
    raw = torch.full((rows * cols * size + 2 * extra,), 0x7B, dtype=torch.uint8, device="cuda")
    view = raw[extra:extra + rows * cols * size].view(dtype).reshape(rows, cols)

    def untouched():
        return bool((raw[:extra] == 0x7B).all()) and bool((raw[extra + rows * cols * size:] == 0x7B).all())
    return view, untouched


def linear_operands(r, M, N, K, spread=3):
    x, w = draw_mx4(r, M, K, spread), draw_mx4(r, N, K, spread)
    return x, w, r.standard_normal(N).astype(np.float32)


# Shared K: each tile that shares it, ragged in tokens, channels and K; parts of
# unequal length; fewer tokens than the tile has
SPLITS = [(33, 100, 16416), (60, 512, 20512), (200, 130, 9248), (17, 67, 13088), (65, 2727, 12448), (40, 4200, 24544),
          (65, 4161, 20928)]


@pytest.mark.parametrize("M,N,K", SPLITS)
def test_linear_with_shared_k(M, N, K):
    assert "split-K" in ot.ot_qlinear_mx4_plan(M, N, K, True)
    r = np.random.default_rng([M, N, K])
    x, w, bias = linear_operands(r, M, N, K)
    some = np.unique(np.r_[r.integers(0, N, 300), 0, N - 1])
    y, mags = X.linear(X.values(*x), X.values(w[0][some], w[1][:, some]), bias[some])
    Wp = ot.pack_weights_mx4(*map(dev, w))
    need = ot.ot_qlinear_mx4_workspace_size(M, N, K)
    ws, ws_ok = guarded(1, need, torch.uint8)
    Y, y_ok = guarded(M, N, torch.float16)
    for _ in range(2):
        ws.fill_(0xFF)  # NaNs
        Y.fill_(NAN16)
        ot.ot_qlinear_mx4(*map(dev, x), Wp, N, dev(bias), Y, ws.reshape(-1))
        got = host(Y).astype(np.float64)
        assert np.all(np.abs(got[:, some] - y) <= y_tolerance(y, mags, K))
        assert ws_ok() and y_ok()
    # without a workspace: the same sums in another order
    alone = host(ot.qlinear_mx4(*map(dev, x), Wp, N, dev(bias), False)).astype(np.float64)
    assert np.all(np.abs(alone[:, some] - y) <= y_tolerance(y, mags, K))
    assert not np.isnan(got).any()


def test_linear_with_shared_k_on_the_widest_tile():
    M, N, K = 200, 8332, 36352
    assert ot.ot_qlinear_mx4_plan(M, N, K, True) == "tiles 256x256 split-K 6"
    r = np.random.default_rng(3)
    x, w, bias = linear_operands(r, M, N, K)
    some = np.unique(np.r_[r.integers(0, N, 200), 0, N - 1])
    y, mags = X.linear(X.values(*x), X.values(w[0][some], w[1][:, some]), bias[some])
    got = ot.qlinear_mx4(*map(dev, x), ot.pack_weights_mx4(*map(dev, w)), N, dev(bias), True)
    assert not bool(got.isnan().any())
    assert np.all(np.abs(host(got)[:, some].astype(np.float64) - y) <= y_tolerance(y, mags, K))


@pytest.mark.parametrize("M,N,K", [(1, 65, 96), (7, 33, 288), (30, 70, 544), (50, 100, 1056),
                                   (70, 65, 96), (130, 257, 544), (300, 1000, 1056), (65, 70, 3488)])
def test_linear_neighbours_and_rows_of_nan(M, N, K):
    """Nothing is written outside Y; a NaN block of a token is its row's alone, one
    of a weight row its channel's, an infinite bias its own."""
    r = np.random.default_rng([M, N, K])
    (xc, xe), (wc, we), bias = linear_operands(r, M, N, K)
    clean, c_ok = guarded(M, N, torch.float16)
    Y, y_ok = guarded(M, N, torch.float16)
    ws = ot.qlinear_mx4_workspace_for(M, N, K)
    ot.ot_qlinear_mx4(dev(xc), dev(xe), ot.pack_weights_mx4(dev(wc), dev(we)), N, dev(bias), clean, ws)
    m, n, inf = M // 2, N // 3, N - 1
    last = K // 32 - 1
    xe[last // 8, m, last % 8] = 255
    we[0, n, 0] = 255
    bias[inf] = np.inf
    ot.ot_qlinear_mx4(dev(xc), dev(xe), ot.pack_weights_mx4(dev(wc), dev(we)), N, dev(bias), Y, ws)
    a, b = host(clean), host(Y)
    assert not np.isnan(a).any() and c_ok() and y_ok()
    assert np.isnan(b[m]).all() and np.isnan(b[:, n]).all()
    rows, cols = np.arange(M) != m, (np.arange(N) != n) & (np.arange(N) != inf)
    assert np.array_equal(a[rows][:, cols], b[rows][:, cols])
    assert (b[rows, inf] == np.inf).all()


@pytest.mark.parametrize("M,K", [(1, 32), (5, 544), (130, 2080)])
def test_quantizers_write_their_outputs_alone(M, K):
    r = np.random.default_rng([M, K])
    x, z, inv_s = draw_activations(r, M, K)
    g, b = (r.standard_normal(K).astype(np.float16) for _ in range(2))
    tiles = -(-K // 256)
    Xc, c_ok = guarded(M, K // 2, torch.uint8)
    Xe, e_ok = guarded(tiles * M, 8, torch.uint8)
    y, y_ok = guarded(M, K, torch.float32)
    Wp, p_ok = guarded(1, ot.ot_packed_weights_mx4_size(M, K), torch.uint8)
    bp, b_ok = guarded(1, M, torch.float32)
    e3 = Xe.view(tiles, M, 8)
    ot.ot_quantize_act_mx4(dev(x), dev(z), dev(inv_s), Xc, e3)
    ot.ot_dequantize_mx4(Xc, e3, y)
    ot.ot_pack_weights_mx4(Xc, e3, Wp.reshape(-1))
    assert np.array_equal(host(Wp)[0], X.pack(host(Xc), host(e3)))
    ot.ot_ln_quantize_act_mx4(dev(x), dev(g), dev(b), 1e-5, dev(z), dev(inv_s), Xc, e3)
    ot.ot_fold_weights_mx4(dev(x), None, dev(z), dev(inv_s), Xc, e3, bp.reshape(-1))
    assert all(ok() for ok in (c_ok, e_ok, y_ok, p_ok, b_ok))


def test_fold_of_more_rows_than_a_launch_has_workgroups():
    """Beyond 2^21 rows the workgroups take several pairs of rows each."""
    N, K = (1 << 21) + 3, 32
    g = torch.Generator(device="cuda").manual_seed(1)
    W = torch.randn(N, K, device="cuda", generator=g).half()
    z = torch.randn(K, device="cuda", generator=g)
    Wc, We, bp = ot.fold_weights_mx4(W, None, z, None)
    for part in (slice(0, 1000), slice(N - 1000, N), slice((1 << 21) - 500, (1 << 21) + 3)):
        c, e, b = X.fold(host(W[part]), None, host(z), None)
        assert np.array_equal(host(Wc[part]), c) and np.array_equal(host(We[:, part]), e)
        # one rounding of the fp64 sum, itself off by far less
        assert np.all(np.abs(host(bp[part]) - b) <= np.abs(b) * 2.0 ** -23 + 1e-30)
    # every row: the largest level of a block is 4 or 6 and its scale is the row's
    y = ot.dequantize_mx4(Wc, We)
    assert bool(((y - W.float()).abs().amax(1) <= W.float().abs().amax(1) / 4).all())
    assert bool((bp - W.double() @ z.double()).abs().max() < 1e-4)


def moe_call(x, logits, k, w1, b1, w2, b2, F, act, Y, ws):
    ot.ot_moe_mx4(dev(x[0]), dev(x[1]), dev(logits), k, ot.pack_weights_mx4(*map(dev, w1)),
                  dev(b1), ot.pack_weights_mx4(*map(dev, w2)), dev(b2), F, act, Y, ws)


# the second kernel's K tiles shared between workgroups: few output channels, and
# experts enough (the last one has one part all the same)
@pytest.mark.parametrize("M,H,F,E,k", [(40, 96, 1056, 32, 2), (17, 512, 1312, 20, 2), (64, 32, 544, 70, 3),
                                       (5, 256, 800, 30, 4), (1, 32, 4128, 16, 8), (9, 288, 96, 4, 2)])
@pytest.mark.parametrize("act", ["relu", "swiglu"])
def test_moe_with_shared_k(M, H, F, E, k, act):
    r = np.random.default_rng([M, H, F, E, k])
    x, logits, w1, b1, w2, b2 = draw_moe(r, M, H, F, E, act)
    logits[M // 2] = -np.inf  # a token without an expert
    y, tol = moe_expected(x, logits, k, w1, b1, w2, b2, F, act)
    ws, ws_ok = guarded(1, ot.ot_moe_mx4_workspace_size(M, H, F, E, k), torch.uint8)
    Y, y_ok = guarded(M, H, torch.float16)
    outs = []
    for fill in (0xFF, 0x00):
        ws.fill_(fill)
        Y.fill_(NAN16)
        moe_call(x, logits, k, w1, b1, w2, b2, F, act, Y, ws.reshape(-1))
        assert ws_ok() and y_ok()
        outs.append(Y.clone())
    assert torch.equal(outs[0], outs[1])
    assert np.all(np.abs(host(outs[0]).astype(np.float64) - y) <= tol)
    assert not host(outs[0])[M // 2].any()


def test_moe_nan_blocks_stay_with_their_tokens_and_experts():
    """A NaN block of a token reaches that token alone, one of an expert's weights
    the tokens that chose it."""
    M, H, F, E, k = 20, 128, 96, 6, 2
    r = np.random.default_rng(8)
    x, logits, w1, b1, w2, b2 = draw_moe(r, M, H, F, E, "relu")
    ws = ot.moe_mx4_workspace_for(M, H, F, E, k)
    clean, Y = (torch.empty(M, H, dtype=torch.float16, device="cuda") for _ in range(2))
    moe_call(x, logits, k, w1, b1, w2, b2, F, "relu", clean, ws)
    chosen = X.top_k(logits, k)
    x[1][0, 3, 1] = 255
    w2[1][0, 4 * H:5 * H, 0] = 255
    moe_call(x, logits, k, w1, b1, w2, b2, F, "relu", Y, ws)
    bad = (chosen == 4).any(1)
    bad[3] = True
    assert not clean.isnan().any() and 1 < bad.sum() < M
    assert bool(Y[dev(bad)].isnan().all()) and torch.equal(Y[dev(~bad)], clean[dev(~bad)])


# --- the largest sizes: element numbers past 32 bits --------------------------------

def random_mx4(rows, K, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    c = torch.randint(0, 256, (rows, K // 2), dtype=torch.uint8, device="cuda", generator=g)
    e = torch.randint(122, 127, ((K + 255) // 256, rows, 8), dtype=torch.uint8, device="cuda", generator=g)
    if K % 256:
        e[-1, :, K % 256 // 32:] = 0
    return c, e


@pytest.mark.parametrize("M", [1, 20, 65])
def test_linear_of_the_most_channels(M):
    N, K = (1 << 26) - 1, 32
    w, x = random_mx4(N, K, 1), random_mx4(M, K, 2)
    bias = torch.randn(N, device="cuda")
    Wp = ot.pack_weights_mx4(*w)
    Y = ot.qlinear_mx4(*x, Wp, N, bias, True)
    some = np.unique(np.r_[0:40, N // 2:N // 2 + 40, (1 << 25) - 20:(1 << 25) + 20, N - 300:N])
    at = torch.from_numpy(some).cuda()
    y, mags = X.linear(X.values(*map(host, x)), X.values(host(w[0][at]), host(w[1][:, at])),
                       host(bias[at]))
    assert np.all(np.abs(host(Y[:, at]).astype(np.float64) - y) <= y_tolerance(y, mags, K))
    del Wp, w
    assert not bool(Y[-1].isnan().any())


def test_linear_of_the_most_tokens():
    """The last rows that a launch takes, whose byte numbers pass 2^35."""
    M, N, K = (1 << 31) - 256, 1, 32
    assert ot.ot_qlinear_mx4_plan(M, N, K) != "none"
    w = random_mx4(N, K, 1)
    x = (torch.empty(M, K // 2, dtype=torch.uint8, device="cuda"),
         torch.zeros(1, M, 8, dtype=torch.uint8, device="cuda"))
    some = np.unique(np.r_[0:300, (1 << 30) - 200:(1 << 30) + 200, M - 600:M])
    at = torch.from_numpy(some).cuda()
    part = random_mx4(some.size, K, 3)
    x[0][at], x[1][:, at] = part
    bias = torch.randn(N, device="cuda")
    Y, y_ok = guarded(M, N, torch.float16, 512)
    ot.ot_qlinear_mx4(*x, ot.pack_weights_mx4(*w), N, bias, Y, ot.qlinear_mx4_workspace_for(M, N, K))
    y, mags = X.linear(X.values(*map(host, part)), X.values(*map(host, w)), host(bias))
    assert np.all(np.abs(host(Y[at]).astype(np.float64) - y) <= y_tolerance(y, mags, K))
    assert y_ok()


def test_linear_of_the_longest_rows():
    """With one scale each, of 1/2 and 1, the products are multiples of 1/8, and the
    sums (of random signs: far below 2^21) multiples of 1/8 that fp32 holds: exact in
    any order. What remains is the bias, half a step of fp32, and half one of fp16."""
    N, K = 64, 1 << 22
    for M in (3, 40, 70):
        x, w = random_mx4(M, K, 4), random_mx4(N, K, 5)
        x[1].fill_(126)
        w[1].fill_(127)
        bias = torch.randn(N, device="cuda")
        Y = ot.qlinear_mx4(*x, ot.pack_weights_mx4(*w), N, bias, True)
        xv, wv = (ot.dequantize_mx4(*t).double() for t in (x, w))
        y = host(xv @ wv.t() + bias.double())
        assert 2000 < np.abs(y).max() < 65000
        assert np.all(np.abs(host(Y).astype(np.float64) - y) <= np.abs(y) * (2.0 ** -11 + 2.0 ** -23)
                      + 2.0 ** -22)


def test_quantizers_past_32_bits():
    M, K = (1 << 27) + 5, 32  # 2^32 + 160 elements
    part = np.r_[0:100, M // 2:M // 2 + 100, M - 100:M]
    at = torch.from_numpy(part).cuda()
    r = np.random.default_rng(6)
    h, z, inv_s = draw_activations(r, part.size, K)
    x = torch.zeros(M, K, dtype=torch.float16, device="cuda")
    x[at] = dev(h)
    c, e = ot.quantize_act_mx4(x, dev(z), dev(inv_s))
    wc, we = X.to_mx4(X.activations(h, z, inv_s))
    assert np.array_equal(host(c[at]), wc) and np.array_equal(host(e[:, at]), we)
    wc, we, bp = X.fold(h, None, z, inv_s)
    c, e, b = ot.fold_weights_mx4(x, None, dev(z), dev(inv_s))
    assert np.array_equal(host(c[at]), wc) and np.array_equal(host(e[:, at]), we)
    assert np.all(np.abs(host(b[at]) - bp) <= np.abs(bp) * 2.0 ** -23 + 1e-30)
    del x
    y = ot.dequantize_mx4(c, e)
    assert np.array_equal(host(y[at]), X.values(wc, we).astype(np.float32))


def test_moe_of_many_wide_experts():
    """Weights whose byte numbers pass 32 bits: the last experts' are the right ones
    (the plain form has the chosen experts alone)."""
    M, H, F, E, k = 5, 32768, 1024, 256, 2
    r = np.random.default_rng(7)
    some = [0, 131, 254, 255]
    x, small, _, b1, _, b2 = draw_moe(r, M, H, F, len(some), "relu")
    logits = np.full((M, E), -np.inf, np.float16)
    logits[:, some] = small
    parts, packed = [], []
    for rows, K in ((F, H), (H, F)):
        c, e = random_mx4(E * rows, K, rows)
        e[:] = 123 + (e & 1)
        packed.append(ot.pack_weights_mx4(c, e))
        at = torch.cat([torch.arange(i * rows, (i + 1) * rows) for i in some]).cuda()
        parts.append((host(c[at]), host(e[:, at])))
        del c, e
    bias = [np.zeros((E, v.shape[1]), np.float32) for v in (b1, b2)]
    for v, small_v in zip(bias, (b1, b2)):
        v[some] = small_v
    got = ot.moe_mx4(*map(dev, x), dev(logits), k, packed[0], dev(bias[0]), packed[1], dev(bias[1]),
                     F, "relu")
    y, tol = moe_expected(x, small, k, parts[0], b1, parts[1], b2, F, "relu")
    assert np.median(tol) <= 0.05 * np.sqrt(np.mean(y * y))
    assert np.all(np.abs(host(got).astype(np.float64) - y) <= tol)


# --- one after another ----------------------------------------------------------

def layer(r, N, K):
    W = (r.standard_normal((N, K)) * K ** -0.5).astype(np.float16)
    b = r.standard_normal(N).astype(np.float16)
    return W, b


def fold(W, b, z, s):
    Wc, We, bp = ot.fold_weights_mx4(dev(W), dev(b), dev(z), dev(s))
    return ot.pack_weights_mx4(Wc, We), bp


@pytest.mark.parametrize("M", [1, 9, 40, 150])
def test_a_block_of_layers(M):
    """LayerNorm and quantizer, a linear, a quantizer, a linear, and a mixture of
    experts behind a LayerNorm: each output against the plain form of what went
    in (a code apart would be a step of the next operator, so each is checked by
    itself on the values that the GPU handed on)."""
    r = np.random.default_rng(M)
    H, F, E, top = 288, 1056, 6, 2
    h, z, inv_s = draw_activations(r, M, H)
    gamma, beta = (r.standard_normal(H).astype(np.float16) for _ in range(2))
    (W1, b1), (W2, b2) = layer(r, F, H), layer(r, H, F)
    P1, p1 = fold(W1, b1, z, 1 / inv_s)
    Xc, Xe = ot.ln_quantize_act_mx4(dev(h), dev(gamma), dev(beta), 1e-5, dev(z), dev(inv_s))
    Y1 = ot.qlinear_mx4(Xc, Xe, P1, F, p1, True)
    c, e, bias = X.fold(W1, b1, z, 1 / inv_s)
    y, mags = X.linear(X.values(host(Xc), host(Xe)), X.values(c, e), bias)
    # bprime is rounded to fp32 once
    tol = y_tolerance(y, mags, H) + np.abs(bias) * 2.0 ** -24
    assert np.all(np.abs(host(Y1).astype(np.float64) - y) <= tol)

    z2, s2 = np.zeros(F, np.float32) + 0.25, r.uniform(0.5, 2, F).astype(np.float32)
    P2, p2 = fold(W2, b2, z2, s2)
    A = Y1.relu()
    Ac, Ae = ot.quantize_act_mx4(A, dev(z2), dev((1 / s2).astype(np.float32)))
    Y2 = ot.qlinear_mx4(Ac, Ae, P2, H, p2, True)
    c, e = X.to_mx4(X.activations(host(A), z2, (1 / s2).astype(np.float32)))
    assert np.array_equal(host(Ac), c) and np.array_equal(host(Ae), e)
    wc, we, bias = X.fold(W2, b2, z2, s2)
    y, mags = X.linear(X.values(c, e), X.values(wc, we), bias)
    tol = y_tolerance(y, mags, F) + np.abs(bias) * 2.0 ** -24
    assert np.all(np.abs(host(Y2).astype(np.float64) - y) <= tol)

    if M > 64:
        return
    Bc, Be = ot.ln_quantize_act_mx4(Y2, dev(gamma), dev(beta), 1e-5, dev(z * 0), dev(inv_s * 0 + 1))
    _, logits, w1, b1, w2, b2 = draw_moe(r, M, H, 96, E, "swiglu")
    P1, P2 = (ot.pack_weights_mx4(*map(dev, w)) for w in (w1, w2))
    out = ot.moe_mx4(Bc, Be, dev(logits), top, P1, dev(b1), P2, dev(b2), 96, "swiglu")
    x = (host(Bc), host(Be))
    y, tol = moe_expected(x, logits, top, w1, b1, w2, b2, 96, "swiglu")
    assert np.all(np.abs(host(out).astype(np.float64) - y) <= tol)


# --- graphs and streams -----------------------------------------------------------

class Step:
    """A decode step on buffers of its own: LayerNorm, quantizers, a wide linear, one
    with shared K and a mixture of experts."""
    M, H, N, E, F, TOP = 40, 2080, 24544, 5, 160, 2

    def __init__(self, seed):
        r = np.random.default_rng(seed)
        self.h = dev(draw_activations(r, self.M, self.H)[0])
        one = torch.ones(self.H, device="cuda")
        self.norm = (one.half(), (one * 0.5).half(), 1e-5, one * 0.25, one * 0.5)
        self.fc1 = ot.pack_weights_mx4(*map(dev, draw_mx4(r, self.N, self.H, 1)))
        self.fc2 = ot.pack_weights_mx4(*map(dev, draw_mx4(r, self.H, self.N, 1)))
        self.b1, self.b2 = torch.randn(self.N, device="cuda"), torch.randn(self.H, device="cuda")
        _, logits, w1, _, w2, _ = draw_moe(r, self.M, self.H, self.F, self.E, "relu")
        self.logits, self.w1, self.w2 = dev(logits), *(ot.pack_weights_mx4(*map(dev, w)) for w in (w1, w2))
        codes = lambda k: ot._mx4_empty(self.M, k, "cuda")
        half = lambda k: torch.empty(self.M, k, dtype=torch.float16, device="cuda")
        self.x, self.a, self.c = codes(self.H), codes(self.N), codes(self.H)
        self.y1, self.y2, self.out = half(self.N), half(self.H), half(self.H)
        assert "split-K" in ot.ot_qlinear_mx4_plan(self.M, self.H, self.N, True)
        self.ws1 = ot.qlinear_mx4_workspace_for(self.M, self.N, self.H)
        self.ws2 = ot.qlinear_mx4_workspace_for(self.M, self.H, self.N)
        self.ws = ot.moe_mx4_workspace_for(self.M, self.H, self.F, self.E, self.TOP)

    def run(self):
        ot.ot_ln_quantize_act_mx4(self.h, *self.norm, *self.x)
        ot.ot_qlinear_mx4(*self.x, self.fc1, self.N, self.b1, self.y1, self.ws1)
        ot.ot_quantize_act_mx4(self.y1, None, None, *self.a)
        ot.ot_qlinear_mx4(*self.a, self.fc2, self.H, self.b2, self.y2, self.ws2)
        ot.ot_ln_quantize_act_mx4(self.y2, *self.norm, *self.c)
        ot.ot_moe_mx4(*self.c, self.logits, self.TOP, self.w1, None, self.w2, None, self.F, "relu",
                      self.out, self.ws)

    def clear(self):
        for t in (*self.x, *self.a, *self.c, self.y1, self.y2, self.out, self.ws):
            t.zero_()

    def outputs(self):
        return [t.clone() for t in (self.y1, self.y2, self.out)]


def equal(a, b):
    return all(torch.equal(x, y) for x, y in zip(a, b))


def test_captured_and_replayed():
    step = Step(1)
    step.run()
    torch.cuda.synchronize()
    eager = step.outputs()
    assert all(bool(t.isfinite().all()) and bool(t.abs().max() > 0) for t in eager)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step.run()
    other = dev(draw_activations(np.random.default_rng(9), Step.M, Step.H)[0])
    first = step.h.clone()
    for i in range(4):
        step.clear()
        step.h.copy_(first)
        graph.replay()
        torch.cuda.synchronize()
        assert equal(step.outputs(), eager), i
        # other inputs through the same graph, and eagerly between the replays
        step.clear()
        step.h.copy_(other)
        graph.replay()
        replayed = step.outputs()
        step.clear()
        step.run()
        torch.cuda.synchronize()
        assert equal(replayed, step.outputs()) and not equal(replayed, eager), i


def test_two_graphs_at_once_on_streams_of_their_own():
    steps, streams = [Step(2), Step(3)], [torch.cuda.Stream() for _ in range(2)]
    wanted, graphs = [], []
    for step, s in zip(steps, streams):
        step.run()
        torch.cuda.synchronize()
        wanted.append(step.outputs())
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            step.run()
        graphs.append(g)
    for _ in range(3):
        for step in steps:
            step.clear()
        torch.cuda.synchronize()
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                for _ in range(5):
                    g.replay()
        torch.cuda.synchronize()
        assert all(equal(step.outputs(), w) for step, w in zip(steps, wanted))


def test_eager_on_two_streams_and_by_handle():
    steps, streams = [Step(4), Step(5)], [torch.cuda.Stream() for _ in range(2)]
    wanted = []
    for step in steps:
        step.run()
        torch.cuda.synchronize()
        wanted.append(step.outputs())
        step.clear()
    torch.cuda.synchronize()
    for _ in range(10):
        for step, s in zip(steps, streams):
            with torch.cuda.stream(s):
                step.run()
    torch.cuda.synchronize()
    assert all(equal(step.outputs(), w) for step, w in zip(steps, wanted))
    # the stream as an argument, the current one another
    step, s = steps[0], streams[0]
    y = torch.empty_like(step.y1)
    torch.cuda.synchronize()
    ot.ot_qlinear_mx4(*step.x, step.fc1, step.N, step.b1, y, step.ws1, s.cuda_stream)
    s.synchronize()
    assert torch.equal(y, wanted[0][0])


# --- the method on the format -------------------------------------------------------

def test_symmetrization_helps_where_channels_are_offset():
    """One linear of the workload that shifts every channel: the MX4 product with
    the shift and scale of the channels taken out first, with the scale alone and
    with neither."""
    wl = synth.WORKLOADS["opt13b_w6a6"]
    Xh, W, b, minmax = quality.layer_inputs(wl, 0, 64, 64, 2)
    ref = torch.matmul(Xh.double(), W.double().t()) + b.double()
    errs = {label: quality.errors(quality.run_config(Xh, W, b, minmax, *how), ref)["rel_fro"]
            for label, *how in quality.MX4_CONFIGS}
    assert errs["MX4"] < errs["MX4 no-sym"] and errs["MX4"] < errs["MX4 plain"], errs
    # and the configuration is the plain form's product
    c, e = X.to_mx4(X.activations(host(Xh)))
    some = np.random.default_rng(1).integers(0, W.shape[0], 500)
    wc, we, bias = X.fold(host(W)[some], host(b)[some], None, None)
    y, mags = X.linear(X.values(c, e), X.values(wc, we), bias)
    got = host(quality.run_config(Xh, W, b, minmax, 4, 4, "mx4-plain")).astype(np.float64)[:, some]
    assert np.all(np.abs(got - y) <= y_tolerance(y, mags, W.shape[1]))
