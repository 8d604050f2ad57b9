"""One workspace of the MX4 calls for batches of several sizes."""
import numpy as np
import pytest
import torch

from oracle import mx4_oracle as X
from paper_2406_18832_amd import ot
from tests.test_gpu_mx4 import dev, draw_moe, draw_mx4, host, moe_expected, run_moe, y_tolerance


def test_one_workspace_for_all_batches_up_to_the_largest():
    """ot_qlinear_mx4_workspace_max is the most of ot_qlinear_mx4_workspace_size over
    all smaller numbers of tokens, where that size itself may fall."""
    size, most = ot.ot_qlinear_mx4_workspace_size, ot.ot_qlinear_mx4_workspace_max
    r = np.random.default_rng(4)
    falls = 0
    sizes = [(9216, 36864), (5120, 20480), (512, 36864), (64, 4 << 20), (1, 1024), (32768, 36864)]
    sizes += [(int(2 ** r.uniform(0, 14)), 32 * int(2 ** r.uniform(3, 11))) for _ in range(25)]
    for N, K in sizes:
        up_to = 0
        for M in (*range(1, 1100), *range(1100, 40000, 77)):
            n = size(M, N, K)
            falls += n < up_to
            up_to = max(up_to, n)
            if M < 1100:  # every smaller one was visited
                if M < 200 or M % 64 < 2 or M % 7 == 0:
                    assert most(M, N, K) == up_to, (M, N, K)
            else:
                assert most(M, N, K) >= up_to, (M, N, K)
    assert falls > 100
    for M, N, K in ((0, 64, 64), (-1, 64, 64), (64, 0, 4096), (64, 1 << 26, 64), (64, 64, 40),
                    (1 << 31, 64, 64), (64, 64, (1 << 22) + 32)):
        assert most(M, N, K) == 0
    assert most((1 << 31) - 256, 16, 36864) == max(size(M, 16, 36864) for M in range(1, 33000, 32))
    assert most(1024, 9216, 36864) > size(1024, 9216, 36864) == 0
    ws = ot.qlinear_mx4_workspace_for(1024, 9216, 36864, "cpu", up_to=True)
    assert ws.numel() == most(1024, 9216, 36864) and ws.dtype == torch.uint8
    assert ot.qlinear_mx4_workspace_for(16, 9216, 36864, "cpu", up_to=True) is None


def test_moe_workspace_grows_with_the_tokens():
    """So the buffer of the largest batch serves the smaller ones."""
    r = np.random.default_rng(5)
    for _ in range(300):
        H, F = (32 * int(2 ** r.uniform(0, 9)) for _ in range(2))
        E = int(r.integers(1, 257))
        k = int(r.integers(1, min(E, 16) + 1))
        sizes = [ot.ot_moe_mx4_workspace_size(M, H, F, E, k) for M in range(1, 65)]
        assert all(a <= b for a, b in zip(sizes, sizes[1:])), (H, F, E, k)


TWO_PARTS = (17, 1600, 704, 24, 3)  # 100 workgroups of 16 channels, 72 K tiles


def test_moe_shares_its_second_linear_between_two_workgroups():
    """Where that fills the CUs (256 without a GPU) and leaves each wave two K tiles:
    the workspace has two fp32 sums of every output behind the hidden values."""
    for M, H, F, E, k in (TWO_PARTS, (64, 2048, 1408, 32, 4), (1, 512, 2048, 20, 8)):
        hidden = E * -(-M // 16) * -(-F // 256) * 2048 * 9 // 8
        slots = 2 * (-(-M * k * 4 // 16) * 16)
        assert ot.ot_moe_mx4_workspace_size(M, H, F, E, k) == hidden + slots + 2 * M * H * 4


@pytest.mark.gpu
@pytest.mark.parametrize("act", ["relu", "swiglu"])
def test_moe_of_two_parts(act):
    M, H, F, E, k = TWO_PARTS
    r = np.random.default_rng(7)
    x, logits, w1, b1, w2, b2 = draw_moe(r, M, H, F, E, act)
    y, tol = moe_expected(x, logits, k, w1, b1, w2, b2, F, act)
    assert np.median(tol) <= 0.05 * np.sqrt(np.mean(y * y))
    got = host(run_moe(x, logits, k, w1, b1, w2, b2, F, act)).astype(np.float64)
    assert np.all(np.abs(got - y) <= tol)


@pytest.mark.gpu
def test_one_workspace_serves_batches_of_any_size():
    N, K, most = 200, 20512, 700
    r = np.random.default_rng(6)
    w, bias = draw_mx4(r, N, K), r.standard_normal(N).astype(np.float32)
    wv, Wp = X.values(*w), ot.pack_weights_mx4(*map(dev, w))
    n = ot.ot_qlinear_mx4_workspace_max(most, N, K)
    raw = torch.full((n + 128,), 0xFF, dtype=torch.uint8, device="cuda")
    used = set()
    for M in (most, 512, 257, 130, 65, 64, 33, 17, 5):
        used.add(ot.ot_qlinear_mx4_workspace_size(M, N, K))
        x = draw_mx4(r, M, K)
        y, mags = X.linear(X.values(*x), wv, bias)
        Y = ot.qlinear_mx4(*map(dev, x), Wp, N, dev(bias), raw[64:64 + n])
        assert np.all(np.abs(host(Y).astype(np.float64) - y) <= y_tolerance(y, mags, K)), M
    assert len(used) > 3 and max(used) == n
    assert bool((raw[:64] == 0xFF).all()) and bool((raw[64 + n:] == 0xFF).all())
