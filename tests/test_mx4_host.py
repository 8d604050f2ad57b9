"""The MX4 entry points without a GPU: what they refuse (before any HIP call, so
these calls are safe without a device), the sizes of workspaces and packed
weights, the launch plans, the register budgets, and the oracle's format against
values written out by hand."""
import ctypes
import os

import numpy as np
import pytest

from oracle import mx4_oracle as X
from paper_2406_18832_amd import build_lib, ot
from tests.test_kernel_resources import kernel_resources

OK, EINVAL, ESHAPE = 0, 1, 2
vp, i64, f32, ci = ctypes.c_void_p, ctypes.c_int64, ctypes.c_float, ctypes.c_int
P, ODD = 4096, 4100  # an aligned and a misaligned address, never read
TOP = 1 << 31

# name: (arguments in order, the positions of its pointers, of those that may be
# null, the position of K); every size is one that the call takes
CALLS = {
    "ot_quantize_act_mx4": ([vp(P), i64(3), i64(64), vp(P), vp(P), vp(P), vp(P), None],
                            (0, 3, 4, 5, 6), (), 2),
    "ot_ln_quantize_act_mx4": ([vp(P), i64(3), i64(64), vp(P), vp(P), f32(1e-5), vp(P), vp(P),
                                vp(P), vp(P), None], (0, 3, 4, 6, 7, 8, 9), (), 2),
    "ot_fold_weights_mx4": ([vp(P), vp(0), i64(3), i64(64), vp(0), vp(0), vp(P), vp(P), vp(P),
                             None], (0, 6, 7), (1, 4, 5), 3),
    "ot_dequantize_mx4": ([vp(P), vp(P), i64(3), i64(64), vp(P), None], (0, 1, 4), (), 3),
    "ot_pack_weights_mx4": ([vp(P), vp(P), i64(3), i64(64), vp(P), None], (0, 1, 4), (), 3),
    "ot_qlinear_mx4": ([vp(P), vp(P), vp(P), vp(P), i64(3), i64(5), i64(64), vp(P), vp(0), None],
                       (0, 1, 2, 3, 7), (8,), 6),
    "ot_moe_mx4": ([vp(P), vp(P), vp(P), vp(P), vp(0), vp(P), vp(0), i64(3), i64(64), i64(32),
                    i64(4), i64(2), ci(0), vp(P), vp(P), None], (0, 1, 2, 3, 5, 13, 14), (4, 6), 8),
}


def status(name, args):
    f = getattr(ot.lib(), name)
    f.restype = ci
    return f(*args)


def put(args, i, v):
    old = args[i]
    return args[:i] + [type(old)(v)] + args[i + 1:]


@pytest.mark.parametrize("name", CALLS)
def test_null_and_misaligned_pointers_are_refused(name):
    args, pointers, optional, _ = CALLS[name]
    for i in pointers:
        assert status(name, put(args, i, 0)) == EINVAL, i
        assert status(name, put(args, i, ODD)) == EINVAL, i
    for i in optional:
        if (name, i) != ("ot_fold_weights_mx4", 1):  # read by elements
            # the required ones null as well, so that nothing could run
            assert status(name, put(put(args, i, ODD), pointers[0], 0)) == EINVAL, i
    if name == "ot_quantize_act_mx4":  # z without inv_s, and the other way round
        assert status(name, put(args, 3, 0)) == EINVAL
        assert status(name, put(args, 4, 0)) == EINVAL


@pytest.mark.parametrize("name", CALLS)
def test_sizes_outside_the_documented_ones_are_refused(name):
    args, _, _, k = CALLS[name]
    for K in (0, 16, 31, 33, 48, (1 << 22) + 32, 1 << 40):
        assert status(name, put(args, k, K)) == ESHAPE, K
    for i, a in enumerate(args):
        if isinstance(a, i64):
            assert status(name, put(args, i, -1)) == EINVAL, i
            assert status(name, put(args, i, -(1 << 40))) == EINVAL, i
            if i != k:
                assert status(name, put(args, i, 1 << 40)) == ESHAPE, i
    rows = {"ot_ln_quantize_act_mx4": (1, 1 << 22), "ot_qlinear_mx4": (5, 1 << 26),
            "ot_moe_mx4": (7, 65)}.get(name, (args.index(next(a for a in args if isinstance(a, i64))),
                                              TOP))
    assert status(name, put(args, *rows)) == ESHAPE
    if name == "ot_ln_quantize_act_mx4":
        for eps in (-1e-5, float("nan"), float("inf")):
            assert status(name, put(args, 5, eps)) == EINVAL
        assert status(name, put(args, 2, 65568)) == ESHAPE


def test_moe_sizes():
    name = "ot_moe_mx4"
    args = CALLS[name][0]
    M, H, F, E, k, act = 7, 8, 9, 10, 11, 12
    for i, bad in ((H, (65568, 48)), (F, (0, 16, 40, 65568)), (E, (0, 257, 1)),
                   (k, (0, 5, 17)), (M, (65,))):
        for v in bad:
            assert status(name, put(args, i, v)) == ESHAPE, (i, v)
    assert status(name, put(put(args, E, 256), k, 17)) == ESHAPE
    for v in (-1, 2, 7):
        assert status(name, put(args, act, v)) == EINVAL


def test_no_rows_is_no_work():
    for name, i in (("ot_quantize_act_mx4", 1), ("ot_ln_quantize_act_mx4", 1),
                    ("ot_dequantize_mx4", 2), ("ot_qlinear_mx4", 4), ("ot_moe_mx4", 7)):
        args, pointers, _, _ = CALLS[name]
        args = put(args, i, 0)
        for p in pointers:
            args = put(args, p, 0)
        assert status(name, args) == OK, name
    for name in ("ot_fold_weights_mx4", "ot_pack_weights_mx4"):  # weights have rows
        assert status(name, put(CALLS[name][0], 2, 0)) == ESHAPE
    assert status("ot_qlinear_mx4", put(CALLS["ot_qlinear_mx4"][0], 5, 0)) == ESHAPE


def test_packed_size():
    size = ot.ot_packed_weights_mx4_size
    for N, K in ((1, 32), (32, 256), (33, 257 * 32), (700, 4128), (1 << 26, 1 << 22)):
        assert size(N, K) == 4352 * -(-K // 256) * -(-N // 32)
    for N, K in ((0, 32), (-1, 32), (5, 0), (5, 40), (5, (1 << 22) + 32), (TOP, 32)):
        assert size(N, K) == 0
    r = np.random.default_rng(1)
    for N, K in ((1, 32), (33, 288)):
        e = np.zeros((-(-K // 256), N, 8), np.uint8)
        assert X.pack(r.integers(0, 256, (N, K // 2), dtype=np.uint8), e).size == size(N, K)


def test_moe_workspace_size():
    size = ot.ot_moe_mx4_workspace_size
    assert size(0, 64, 32, 4, 2) == 0
    for bad in ((65, 64, 32, 4, 2), (3, 48, 32, 4, 2), (3, 64, 40, 4, 2), (3, 64, 32, 257, 2),
                (3, 64, 32, 4, 5), (3, 64, 32, 4, 0), (-1, 64, 32, 4, 2)):
        assert size(*bad) == 0
    # room for a row of codes, its scales, an expert and a weight per choice
    for M, H, F, E, k in ((1, 64, 32, 4, 2), (64, 4096, 65536, 256, 16), (17, 96, 288, 3, 2)):
        assert size(M, H, F, E, k) >= M * k * (F // 2 + F // 32 + 8)


def random_linears(n):
    r = np.random.default_rng(2)
    for _ in range(n):
        yield (int(2 ** r.uniform(0, 12)), int(2 ** r.uniform(0, 15)),
               32 * int(2 ** r.uniform(0, 11)))


def test_linear_workspace_holds_its_plans_sums():
    """One fp32 sum per output of a tile and part; the parts have at least two K
    tiles each and the workgroups one pass over the CUs (256 without a GPU)."""
    splits = 0
    for M, N, K in random_linears(3000):
        n, plan = ot.ot_qlinear_mx4_workspace_size(M, N, K), ot.ot_qlinear_mx4_plan(M, N, K, True)
        assert "split" not in ot.ot_qlinear_mx4_plan(M, N, K)
        if " split-K " not in plan:
            assert n == 0
            continue
        splits += 1
        bn, bm = map(int, plan.split()[1].split("x"))
        parts, tiles = int(plan.split()[-1]), -(-M // bm) * -(-N // bn)
        assert M > 16 and 2 <= parts <= 16 and tiles * parts <= 256 and -(-K // 256) >= 2 * parts
        assert n == tiles * parts * bn * bm * 4
    assert splits > 100
    for M, N, K in ((0, 64, 64), (-1, 64, 64), (64, 0, 4096), (64, 1 << 26, 64), (64, 64, 40),
                    (TOP, 64, 64), (64, 64, (1 << 22) + 32)):
        assert ot.ot_qlinear_mx4_workspace_size(M, N, K) == 0


def test_linear_plans():
    plan = ot.ot_qlinear_mx4_plan
    assert plan(0, 64, 64) == "none"
    assert {plan(M, 768, 768) for M in (1, 16, 32, 64)} == {"decode 16 rows"}
    assert plan(8, 20480, 5120) == "decode 32 rows"
    assert plan(64, 20480, 5120) == plan(64, 20480, 5120, True) == "tiles 128x64"
    assert plan(65, 64, 32) == "tiles 64x64"
    assert plan(512, 9216, 36864) == "tiles 192x128"
    assert plan(512, 9216, 36864, True) == "tiles 256x256 split-K 3"
    # the most tokens and channels: fewer than 2^32 work-items
    for M, N in (((1 << 31) - 256, 16), (1 << 24, 30000), (1 << 30, 256), (65, (1 << 26) - 1)):
        bn, bm = map(int, plan(M, N, 32).split()[1].split("x"))
        threads = 256 if bn == 64 else 512
        assert -(-M // bm) * -(-N // bn) * threads < 1 << 32
    L = ot.lib()
    buf = ctypes.create_string_buffer(8)
    assert L.ot_qlinear_mx4_plan(65, 64, 32, 0, buf, 8) == OK and buf.value == b"tiles 6"
    assert L.ot_qlinear_mx4_plan(65, 64, 32, 0, None, 8) == EINVAL
    assert L.ot_qlinear_mx4_plan(65, 64, 32, 0, buf, 0) == EINVAL
    assert L.ot_qlinear_mx4_plan(-1, 64, 32, 0, buf, 8) == EINVAL
    for bad in ((65, 0, 32), (65, 64, 40), (65, 1 << 26, 32), (TOP, 64, 32),
                # more tiles than a launch has work-items for
                (TOP - 1, 16, 32), (TOP - 1, (1 << 26) - 1, 32)):
        assert L.ot_qlinear_mx4_plan(*bad, 0, buf, 8) == ESHAPE, bad


@pytest.mark.timeout(900)
@pytest.mark.parametrize("src", ["ot_mx4_quant.hip", "ot_mx4_gemm.hip", "ot_mx4_decode.hip",
                                 "ot_mx4_moe.hip"])
def test_kernels_do_not_spill(src, tmp_path):
    res = kernel_resources(os.path.join(build_lib.CSRC, src), tmp_path)
    assert res and all(v["spill"] == 0 for v in res.values()), res


def test_oracle_format_by_hand():
    v = np.zeros((1, 288), np.float32)
    v[0, :8] = [4.0, -0.5, 0.25, 0.75, 5.0, 7.9, -2.5, 0.0]       # E = 129: b = 127, scale 1
    v[0, 32:36] = [1.0, -0.3, 0.0625, 0.07]                       # b = 125: 4, -1.2, 0.25, 0.28
    v[0, 64:66] = [2.0 ** -149, 2.0 ** -126]                      # E = 1: b = 0, scale 2^-127
    v[0, 96] = np.inf
    v[0, 128] = np.nan
    v[0, 256:258] = [3.0e38, -1.0e38]                             # E = 254: b = 252
    c, e = X.to_mx4(v)
    assert e[0, 0].tolist() == [127, 125, 0, 255, 255, 0, 0, 0] and e[1, 0].tolist() == [252] + [0] * 7
    code = lambda k: (c[0, k // 2] >> (4 * (k & 1))) & 15
    #        4, -0.5, 0 (tie), 1 (tie), 4 (tie), 6, -2 (tie), 0
    assert [code(k) for k in range(8)] == [6, 9, 0, 2, 6, 7, 12, 0]
    assert [code(k) for k in range(32, 36)] == [6, 10, 0, 1]
    # 2^-149 is 2^-22 of the scale; 2^-126 twice the scale
    assert [code(64), code(65)] == [0, 4]
    assert not c[0, 48:80].any()
    assert [code(256), code(257)] == [7 if 3.0e38 / 2.0 ** 125 > 5 else 6, 12]
    y = X.values(c, e)[0]
    assert y[:8].tolist() == [4, -0.5, 0, 1, 4, 6, -2, 0] and y[32:36].tolist() == [1, -.25, 0, .125]
    assert y[65] == 2.0 ** -126 and np.isnan(y[96:160]).all() and not np.isnan(y[160:]).any()
