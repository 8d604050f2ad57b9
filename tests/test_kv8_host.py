"""The 8-bit cache's entry points without a GPU: argument checks (every call returns
before any HIP call), sizes, plans and the binding's refusals."""
import numpy as np
import pytest
import torch

from oracle import kv8_oracle as O
from paper_2406_18832_amd import ot

P = 4096  # a plausible, aligned pointer that no refused call follows
NAN, INF = float("nan"), float("inf")


def append(T=4, B=2, H=2, D=64, most=3, pages=8, ldk=None, ldv=None, k=P, v=P, cu=P, kv_len=P,
           table=P, Kc=P, Vc=P, Ks=P, Vs=P):
    ldk, ldv = (H * D if x is None else x for x in (ldk, ldv))
    return ot.lib().ot_kv8_append(k, ldk, v, ldv, T, B, H, D, cu, kv_len, table, most, pages, Kc,
                                  Vc, Ks, Vs, None)


def read(T=4, B=2, H=2, D=64, most=3, pages=8, k=P, v=P, cu=P, start=P, table=P, Kc=P, Vc=P, Ks=P,
         Vs=P):
    return ot.lib().ot_kv8_read(Kc, Vc, Ks, Vs, pages, cu, start, table, most, T, B, H, D, k, v,
                                None)


def attend(T=4, B=2, Hq=4, Hkv=2, D=64, most=3, pages=8, ldq=None, scale=0.125, causal=1, window=0,
           max_q=2, q=P, cu=P, kv_len=P, table=P, Kc=P, Vc=P, Ks=P, Vs=P, Y=P, lse=P, ws=None):
    ldq = Hq * D if ldq is None else ldq
    return ot.lib().ot_attn_kv8(q, ldq, T, B, Hq, Hkv, D, cu, kv_len, table, most, pages, Kc, Vc,
                                Ks, Vs, scale, causal, window, max_q, Y, lse, ws, None)


SHAPES = [dict(D=0), dict(D=8), dict(D=72), dict(D=272), dict(B=65536), dict(T=(1 << 24) + 1),
          dict(most=0), dict(most=(1 << 24) + 1), dict(pages=0), dict(pages=1 << 31)]
NEGATIVE = [dict(T=-1), dict(B=-1), dict(D=-16), dict(most=-1), dict(pages=-1)]


@pytest.mark.parametrize("call", [append, read, attend])
def test_sizes(call):
    for s in SHAPES:
        assert call(**s) == ot.OT_ESHAPE, s
    for s in NEGATIVE:
        assert call(**s) == ot.OT_EINVAL, s
    for s in (dict(T=0), dict(B=0)):  # no work: no pointer is looked at
        for name in ("k", "q", "cu", "table", "Kc"):
            if name in call.__code__.co_varnames:
                assert call(**s, **{name: None}) == ot.OT_OK


@pytest.mark.parametrize("call", [append, read])
def test_head_counts(call):
    assert call(H=0) == ot.OT_ESHAPE and call(H=1025) == ot.OT_ESHAPE and call(H=-1) == ot.OT_EINVAL
    # more waves than a launch has
    assert call(T=1 << 24, B=60000, H=1024) == ot.OT_ESHAPE


def test_attention_heads_and_launches():
    for s in (dict(Hq=0), dict(Hkv=0), dict(Hq=3), dict(Hq=1, Hkv=2), dict(Hq=16386, Hkv=2),
              dict(Hkv=1025, Hq=2050), dict(T=1 << 24, Hq=1024, Hkv=1, D=16, max_q=1),
              dict(T=1 << 24, Hq=1024, Hkv=1024, D=16, max_q=1),
              dict(T=65535, B=65535, Hq=1024, Hkv=1024, max_q=1)):
        assert attend(**s) == ot.OT_ESHAPE, s
    for s in (dict(Hq=-4), dict(Hkv=-2)):
        assert attend(**s) == ot.OT_EINVAL, s


def test_attention_arguments():
    for s in (dict(scale=NAN), dict(scale=INF), dict(window=-1), dict(window=5, causal=0),
              dict(max_q=0), dict(max_q=5), dict(max_q=-1)):
        assert attend(**s) == ot.OT_EINVAL, s


@pytest.mark.parametrize("call", [append, read, attend])
def test_pointers(call):
    names = [n for n in call.__code__.co_varnames[:call.__code__.co_argcount]
             if call.__defaults__[call.__code__.co_varnames.index(n)] == P]
    assert len(names) >= 9
    for n in names:
        if n != "lse":
            assert call(**{n: None}) == ot.OT_EINVAL, n
        small = 2 if n in ("cu", "kv_len", "start", "table", "Ks", "Vs", "lse") else 8
        assert call(**{n: P + small}) == ot.OT_EINVAL, n
    if call is attend:
        assert attend(ws=P + 8) == ot.OT_EINVAL


def test_row_distances():
    for ld in (127, 132, 0, -128, 1 << 32):
        assert append(ldk=ld) == ot.OT_EINVAL and append(ldv=ld) == ot.OT_EINVAL
        assert attend(ldq=ld) == ot.OT_EINVAL
    assert attend(ldq=255) == ot.OT_EINVAL


def test_row_sizes():
    for D in range(16, 257, 16):
        assert ot.ot_kv8_row_size(D) == O.row_size(D)
    for D in (-16, 0, 8, 24, 272):
        assert ot.ot_kv8_row_size(D) == 0
        with pytest.raises(ValueError, match="multiple of 16"):
            ot.kv8_cache(4, 2, D, "cpu")


def test_workspaces_and_plans():
    size, plan = ot.ot_attn_kv8_workspace_size, ot.ot_attn_kv8_plan
    assert plan(0, 4, 8, 8, 64, 1) == "none" and plan(4, 0, 8, 8, 64, 1) == "none"
    assert size(0, 4, 8, 8, 64, 1) == 0 and size(4, 4, 8, 3, 64, 1) == 0 and size(4, 4, 8, 8, 65, 1) == 0
    assert size(4, 4, 8, 8, 64, 5) == 0 and size(4, 4, 8, 8, 64, 0) == 0
    with pytest.raises(ot.OTError):
        plan(4, 4, 8, 3, 64, 1)
    with pytest.raises(ot.OTError):
        plan(4, 4, 8, 8, 64, 5)
    # one sequence's next token on few heads is shared between workgroups
    assert size(1, 1, 12, 12, 64, 1) > 0
    assert plan(1, 1, 12, 12, 64, 1) == "few 16 rows"
    assert plan(1, 1, 12, 12, 64, 1, True).startswith("few 16 rows, ")
    assert plan(5, 1, 32, 8, 128, 5).startswith("few 32 rows")
    assert plan(8192, 1, 72, 72, 128, 8192, True).startswith("tiles")


def _tensors(T=3, B=2, H=2, G=2, D=64, device="cpu"):
    f16 = lambda *s: torch.zeros(s, dtype=torch.float16, device=device)
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32, device=device)
    x = f16(T, (G + 2) * H * D)
    q, k, v = x.split((G * H * D, H * D, H * D), 1)
    return dict(q=q.view(T, G * H, D), k=k.view(T, H, D), v=v.view(T, H, D), cu=i32(B + 1),
                kv_len=i32(B), table=i32(B, 3), cache=ot.kv8_cache(8, H, D, device),
                out=(f16(T, H, D), f16(T, H, D)), Y=f16(T, G * H, D),
                lse=torch.zeros(T, G * H, device=device))


def test_binding_refuses_host_tensors():
    t = _tensors()
    with pytest.raises(ValueError, match="k must be on the GPU"):
        ot.ot_kv8_append(t["k"], t["v"], t["cu"], t["kv_len"], t["table"], *t["cache"])
    with pytest.raises(ValueError, match="must be on the GPU"):
        ot.ot_kv8_read(*t["cache"], t["cu"], t["kv_len"], t["table"], *t["out"])
    with pytest.raises(ValueError, match="q must be on the GPU"):
        ot.ot_attn_kv8(t["q"], t["cu"], t["kv_len"], t["table"], *t["cache"], 0.1, True, 0, 1, t["Y"])


def test_binding_refuses_numbers_past_64_bits():
    t = _tensors()
    for window, max_q in ((2 ** 64 + 5, 1), (0, 2 ** 64 + 1), (-2 ** 64, 1)):
        with pytest.raises(ValueError, match="64 bits"):
            ot.ot_attn_kv8(t["q"], t["cu"], t["kv_len"], t["table"], *t["cache"], 0.1, True, window, max_q,
                           t["Y"])


def test_binding_names_rows_that_are_not_dense():
    t = _tensors()
    for bad in (t["k"][:, :, ::2], t["k"].transpose(1, 2), t["k"][:, ::2]):
        if bad.shape[1] > 1 or bad.stride(2) != 1:
            with pytest.raises(ValueError, match="dense rows"):
                ot._kv8_rows(bad, "k")
    with pytest.raises(ValueError, match=r"\[T, heads, D\]"):
        ot._kv8_rows(t["k"][0], "k")


def test_oracle_scale_rule():
    """Least k with most <= 127.5 old 2^k; no growth where it fits; NaN stays."""
    r = np.random.default_rng(3)
    for _ in range(2000):
        old = np.float32(r.uniform(0.5, 1.0) * 2.0 ** r.integers(-31, 9))
        most = np.float32(np.float16(r.uniform(0.5, 1.0) * 2.0 ** r.integers(-20, 16)))
        s, k = O.new_scale(most, old)
        top = float(np.float32(np.float32(127.5) * old))
        assert most <= top * 2.0 ** k and (k == 0 or most > top * 2.0 ** (k - 1))
        assert float(s) == float(old) * 2.0 ** k
        assert np.abs(O.codes(most, s)) <= 127
    assert np.isnan(O.new_scale(1.0, np.float32(np.nan))[0])
    assert np.isnan(O.new_scale(np.inf, np.float32(1))[0])
    assert O.new_scale(127.0, None) == (1.0, 0) and O.new_scale(127.0, np.float32(0)) == (1.0, 0)
    assert O.new_scale(0.0, None) == (0.0, 0) and O.new_scale(0.0, np.float32(2)) == (2.0, 0)


@pytest.mark.parametrize("seed", range(4))
def test_oracle_error_bound_however_tokens_are_written(seed):
    """A token is within half a step of its value when written and below one step of the
    page's scale ever after, in whatever pieces and sizes the tokens come."""
    r = np.random.default_rng(seed)
    n, H, D = 150, 2, 16
    table = np.arange(3, dtype=np.int32)[None]
    cache = O.empty_cache(3, H, D)
    x = (r.normal(size=(n, H, D)) * 2.0 ** r.uniform(-4, 4, (n, 1, 1))).astype(np.float16)
    at = 0
    while at < n:
        m = min(n - at, int(r.integers(1, 40 if seed % 2 else 2)))
        cu = np.array([0, m])
        O.append(cache, x[at:at + m], x[at:at + m], cu, [at + m], table)
        at += m
        k, v = O.keys_values(cache, table, 0, at, D)
        step = np.repeat(cache["Ks"].astype(np.float64), 64, 0)[:at].T[:, :, None]
        assert np.array_equal(k, v)
        err = np.abs(k - x[:at].transpose(1, 0, 2))
        assert (err < step * (1 + 2.0 ** -20)).all()
        assert (err[:, at - m:] <= step[:, at - m:] * (0.5 + 2.0 ** -16)).all()
