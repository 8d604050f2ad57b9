"""The 8-bit cache as it is used: in decoder steps between the quantized linears, in
captured graphs, on other streams, two calls at once, with pages shared and used again,
at the largest sizes."""
import numpy as np
import pytest
import torch

from oracle import kv8_oracle as O
from oracle import ot_oracle as Q
from paper_2406_18832_amd import ot, quality, synth
from tests import _kv8 as K
from tests._tol import assert_fp16_close

pytestmark = pytest.mark.gpu


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def equal(a, b):
    return all(torch.equal(x, y) for x, y in zip(a, b))


def within(Y, lse, want):
    """Y [T, Hq, D] and lse [T, Hq] (tensors) within the oracle's tolerances."""
    y, l, tol, ltol = want
    Y = Y.cpu().numpy().astype(np.float64)
    assert np.all(np.abs(Y - y) <= tol), float((np.abs(Y - y) - tol).max())
    if lse is not None:
        lse = lse.cpu().numpy().astype(np.float64)
        assert np.array_equal(np.isinf(lse), np.isinf(l))
        ok = np.isfinite(l)
        assert np.all(np.abs(lse[ok] - l[ok]) <= ltol[ok])


# --- a decoder layer's attention, from LayerNorm to the out linear --------------------

class Layer:
    """LayerNorm + quantizer, qkv linear (with fewer key heads than query heads), cache,
    attention, per-token quantizer and out linear."""
    H, HQ, HKV, D, PAGES, COLS = 512, 8, 2, 64, 24, 6

    def __init__(self, seed):
        r = np.random.default_rng(seed)
        H, n = self.H, (self.HQ + 2 * self.HKV) * self.D
        self.r = r
        x = r.normal(size=(200, H)).astype(np.float16)
        self.norm = [dev((1 + 0.1 * r.normal(size=H)).astype(np.float16)),
                     dev((0.1 * r.normal(size=H)).astype(np.float16))]
        _, z, s, inv_s = ot.calibrate([x], 8)
        w = (r.normal(size=(n, H)) * 0.04).astype(np.float16)
        self.qkv = ot.fold_weights(dev(w), dev(r.normal(size=n).astype(np.float16)), 8, z, s)
        self.act = z, inv_s
        wo = (r.normal(size=(H, self.HQ * self.D)) * 0.04).astype(np.float16)
        self.out = ot.fold_weights_per_token(dev(wo), dev(r.normal(size=H).astype(np.float16)), None, 8)
        self.cache = ot.kv8_cache(self.PAGES, self.HKV, self.D)
        for t in self.cache[:2]:
            t.fill_(0x5A)
        self.free = list(r.permutation(self.PAGES))

    def split(self, y):
        a, b = self.HQ * self.D, self.HKV * self.D
        return [t.view(len(y), -1, self.D) for t in y.split((a, b, b), 1)]

    def run(self, x, cu, kv_len, table, max_q, ws=None, outs=None):
        """(qkv's output, attention, lse, the layer's) of new tokens x."""
        z, inv_s = self.act
        y = ot.qlinear(ot.ln_quantize_act(x, *self.norm, 1e-5, 8, z, inv_s), *self.qkv, 8, 8)
        q, k, v = self.split(y)
        ot.kv8_append(k, v, cu, kv_len, table, self.cache)
        a, lse = outs or (torch.empty_like(q, memory_format=torch.contiguous_format),
                          torch.empty(q.shape[:2], device="cuda"))
        ot.ot_attn_kv8(q, cu, kv_len, table, *self.cache, self.D ** -0.5, True, 0, max_q, a, lse, ws)
        Xq, sX = ot.quantize_act_per_token(a.view(len(x), -1), 8)
        Wq, sW, bp = self.out
        return y, a, lse, ot.qlinear_per_token(Xq, Wq, sX, sW, bp, 8, 8)


def test_prompts_then_tokens_through_a_layer():
    """Continuous batching: prompts of several sequences, in two pieces, then tokens and
    drafts; a sequence ends and another takes its pages.  Cache, attention and the out
    linear agree with the oracles at every step."""
    L = Layer(1)
    D, Hkv = L.D, L.HKV
    want = K.host(L.cache)
    sequences = {}  # slot -> [length, pages]
    table = np.full((4, L.COLS), -1, np.int32)
    steps = [{0: 70, 1: 5, 2: 130}, {0: 60, 2: 1}, {0: 1, 1: 1, 2: 1}, {1: 40, 3: 63},
             {0: 1, 1: 1, 2: 1, 3: 1}, {0: 3, 1: 2, 2: 4, 3: 2}, "end 2", {2: 150, 0: 1}, {0: 1, 1: 1, 2: 1, 3: 1}]
    for step in steps:
        if step == "end 2":
            L.free += sequences.pop(2)[1]
            table[2] = -1
            continue
        counts = [step.get(b, 0) for b in range(4)]
        for b, n in enumerate(counts):
            s = sequences.setdefault(b, [0, []]) if n else sequences.get(b, [0, []])
            s[0] += n
            while len(s[1]) * 64 < s[0]:
                s[1].append(L.free.pop())
                table[b, len(s[1]) - 1] = s[1][-1]
        lens = [sequences.get(b, [0])[0] for b in range(4)]
        cu, T = K.rows_of(counts), sum(counts)
        x = dev(L.r.normal(size=(T, L.H)).astype(np.float16))
        max_q = max(counts)
        ws = ot.attn_kv8_workspace_for(T, 4, L.HQ, Hkv, D, max_q)
        y, a, lse, out = L.run(x, K.ints(cu), K.ints(lens), K.ints(table), max_q, ws)
        q, k, v = (t.cpu().numpy() for t in L.split(y))
        O.append(want, k, v, cu, lens, table)
        K.assert_same_cache(K.host(L.cache), want, table, lens, D)
        within(a, lse, O.attend(want, q, cu, lens, table, D ** -0.5))
        Xq, sX = Q.quantize_act_per_token(a.view(T, -1).cpu().numpy(), 8)
        Wq, sW, bp = (t.cpu().numpy() for t in L.out)
        assert_fp16_close(out.cpu().numpy(), Q.epilogue_per_token(Q.int_gemm(Xq, Wq), sX, sW, bp))


def test_read_gives_what_attention_takes():
    """Attention over the values that ot_kv8_read returns, in float64, is ot_attn_kv8's;
    reading adds fp16's rounding of keys and values."""
    r = np.random.default_rng(3)
    H, D, lens, counts = 3, 80, [200, 64, 333], [1, 20, 70]
    cache, table = K.filled(r, lens, H, D)
    q = r.normal(size=(sum(counts), H, D)).astype(np.float16)
    cu = K.rows_of(counts)
    c = K.device(cache)
    k, v = ot.kv8_read(c, K.ints(K.rows_of(lens)), K.ints([0] * 3), K.ints(table), sum(lens), D)
    Y = ot.attn_kv8(dev(q), K.ints(cu), K.ints(lens), K.ints(table), c, max_q=70).double()
    want = O.attend(cache, q, cu, lens, table, D ** -0.5)
    tol = torch.from_numpy(want[2]).cuda()
    at = 0
    for b, n in enumerate(lens):
        kk, vv = (t[at:at + n].double() for t in (k, v))
        at += n
        for h in range(H):
            qq = dev(q[cu[b]:cu[b + 1], h]).double()
            x = qq @ kk[:, h].t() * D ** -0.5
            see = torch.from_numpy(O.visible(counts[b], n, True, 0)).cuda()
            # keys off by half a step of fp16: scores by that of sum |q k|; p changes by twice
            # that, values by half a step more
            dx = (qq.abs() @ kk[:, h].abs().t()).max() * D ** -0.5 * 2.0 ** -11
            p = x.masked_fill(~see, float("-inf")).softmax(1)
            limit = tol[cu[b]:cu[b + 1], h] + (2 * torch.expm1(dx) + 2.0 ** -11) * (p @ vv[:, h].abs()) + 2.0 ** -24
            assert bool(((Y[cu[b]:cu[b + 1], h] - p @ vv[:, h]).abs() <= limit).all())


def test_sequences_that_share_full_pages():
    """A prefix's full pages in two tables: read by both, written by none."""
    r = np.random.default_rng(4)
    H, D = 2, 128
    cache, table = K.filled(r, [128, 1], H, D)
    shared = np.array([[table[0, 0], table[0, 1], table[1, 0]], [table[0, 0], table[0, 1], len(cache["Ks"]) - 1]], np.int32)
    spare = [p for p in range(len(cache["Ks"])) if p not in table[0, :2]]
    shared[:, 2] = spare[:2]
    lens, cu = [130, 170], np.array([0, 2, 44])
    k, v = K.heads_of(r, 44, H, D), K.heads_of(r, 44, H, D)
    q = r.normal(size=(44, 2 * H, D)).astype(np.float16)
    c = K.device(cache)
    O.append(cache, k, v, cu, lens, shared)
    args = K.ints(cu), K.ints(lens), K.ints(shared)
    ot.kv8_append(dev(k), dev(v), *args, c)
    K.assert_same_cache(K.host(c), cache, shared, lens, D)
    within(*ot.attn_kv8(dev(q), *args, c, max_q=42, want_lse=True),
           O.attend(cache, q, cu, lens, shared, D ** -0.5))


# --- graphs and streams ---------------------------------------------------------------

class Step:
    """Writing and attention of one step on buffers of its own."""

    def __init__(self, seed, counts, lens, Hq=8, H=4, D=128, rows=None):
        r = np.random.default_rng(seed)
        self.H, self.D, self.Hq, self.r = H, D, Hq, r
        self.rows = rows or sum(counts)
        self.cols = -(-max(lens) // 64) + 20  # wide tables: keys are shared out
        B = len(lens)
        self.pages = B * self.cols
        self.cache = ot.kv8_cache(self.pages, H, D)
        self.x = torch.zeros(self.rows, (Hq + 2 * H) * D, dtype=torch.float16, device="cuda")
        self.q, self.k, self.v = (t.view(self.rows, -1, D) for t in self.x.split((Hq * D, H * D, H * D), 1))
        self.cu, self.lens = (torch.zeros(n, dtype=torch.int32, device="cuda") for n in (B + 1, B))
        self.table = torch.zeros(B, self.cols, dtype=torch.int32, device="cuda")
        self.max_q = max(counts)
        self.ws = ot.attn_kv8_workspace_for(self.rows, B, Hq, H, D, self.max_q)
        self.Y = torch.empty(self.rows, Hq, D, dtype=torch.float16, device="cuda")
        self.lse = torch.empty(self.rows, Hq, device="cuda")
        self.load(counts, lens)

    def load(self, counts, lens):
        """Another batch: tokens, lengths, pages, and what the cache holds of it before."""
        r = self.r
        before = [n - c for n, c in zip(lens, counts)]
        table = r.permutation(self.pages).astype(np.int32).reshape(len(lens), -1)
        self.table.copy_(dev(table))
        self.cu.copy_(K.ints(K.rows_of(counts)))
        self.lens.copy_(K.ints(lens))
        self.x.copy_(torch.randn(self.x.shape, device="cuda"))
        n = sum(before)
        k, v = (torch.randn(n, self.H, self.D, device="cuda").half() for _ in range(2))
        ot.kv8_append(k, v, K.ints(K.rows_of(before)), K.ints(before), self.table, self.cache)
        torch.cuda.synchronize()

    def run(self):
        ot.kv8_append(self.k, self.v, self.cu, self.lens, self.table, self.cache)
        ot.ot_attn_kv8(self.q, self.cu, self.lens, self.table, *self.cache, self.D ** -0.5, True, 0,
                       self.max_q, self.Y, self.lse, self.ws)

    def clear(self):
        self.Y.fill_(float("nan"))
        self.lse.fill_(float("nan"))
        if self.ws is not None:
            self.ws.fill_(0xFF)

    def outputs(self):
        return self.Y.clone(), self.lse.clone(), *(t.clone() for t in self.cache)

    def wanted(self):
        """What an eager run gives, from the state that run() finds now."""
        saved = [t.clone() for t in self.cache]
        self.clear()
        self.run()
        torch.cuda.synchronize()
        out = self.outputs()
        for t, s in zip(self.cache, saved):
            t.copy_(s)
        self.clear()
        torch.cuda.synchronize()
        return out


DECODE = dict(counts=[1, 1, 1], lens=[2000, 70, 64 * 21])
PROMPT = dict(counts=[70, 40, 33], lens=[2500, 40, 1100])


@pytest.mark.parametrize("batch", [DECODE, PROMPT], ids=["decode", "prompt"])
def test_captured_step_replays_with_other_lengths_and_pages(batch):
    s = Step(5, rows=sum(batch["counts"]) + 2, **batch)  # two padded rows
    assert s.ws is not None
    s.wanted()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s.run()
    n = batch["counts"]
    others = [(n, batch["lens"]), ([n[0], 0, n[2]], [n[0], 0, 1500]), (n, [900, 1290, 65]),
              ([0, 0, 0], [5, 5, 5]), ([max(1, c // 2) for c in n], [2047, 777, 1409])]
    for counts, lens in others + others[:1]:
        s.load(counts, lens)
        want = s.wanted()
        graph.replay()
        torch.cuda.synchronize()
        got, m = s.outputs(), sum(counts)
        assert equal([t[:m] for t in got[:2]], [t[:m] for t in want[:2]]) and equal(got[2:], want[2:])
        assert all(bool(t[m:].isnan().all()) for t in got[:2])  # padded rows are as they were
        assert bool(got[0][:m].isfinite().all())
        graph.replay()  # the same tokens again: nothing changes
        torch.cuda.synchronize()
        assert equal([t[:m] for t in s.outputs()[:2]], [t[:m] for t in want[:2]])
        assert equal(s.outputs()[2:], want[2:])


def test_two_graphs_share_a_workspace_in_turn():
    a, b = Step(6, **DECODE), Step(7, **PROMPT)
    shared = torch.empty(max(a.ws.numel(), b.ws.numel()), dtype=torch.uint8, device="cuda")
    wants, graphs = [], []
    for s in (a, b):
        s.ws = shared
        wants.append(s.wanted())
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            s.run()
        graphs.append(g)
    for _ in range(3):
        for s in (a, b):
            s.clear()
        for g in graphs + graphs:
            g.replay()
        torch.cuda.synchronize()
        assert all(equal(s.outputs(), w) for s, w in zip((a, b), wants))


def test_two_calls_at_once_and_streams_by_handle():
    steps, streams = [Step(8, **DECODE), Step(9, **PROMPT), Step(10, **PROMPT)], [torch.cuda.Stream() for _ in range(3)]
    wants = [s.wanted() for s in steps]
    for _ in range(10):
        for s, st in zip(steps, streams):
            with torch.cuda.stream(st):
                s.run()
    torch.cuda.synchronize()
    assert all(equal(s.outputs(), w) for s, w in zip(steps, wants))
    # the stream as an argument, the current one another
    s, st = steps[0], streams[1]
    s.clear()
    torch.cuda.synchronize()
    ot.ot_kv8_append(s.k, s.v, s.cu, s.lens, s.table, *s.cache, st.cuda_stream)
    ot.ot_attn_kv8(s.q, s.cu, s.lens, s.table, *s.cache, s.D ** -0.5, True, 0, s.max_q, s.Y, s.lse, s.ws,
                   st.cuda_stream)
    k, v = (torch.empty(len(s.lens), s.H, s.D, dtype=torch.float16, device="cuda") for _ in range(2))
    torch.cuda.synchronize()
    ot.ot_kv8_read(*s.cache, s.cu, s.lens - 1, s.table, k, v, st.cuda_stream)
    st.synchronize()
    assert equal(s.outputs(), wants[0])
    assert bool(((k - s.k).abs() < 0.05).all()) and bool(((v - s.v).abs() < 0.05).all())


# --- the largest sizes ----------------------------------------------------------------

def test_pool_past_32_bits():
    """Pages whose codes lie past 2^32 bytes, beside pages at the start."""
    H, D, pages = 40, 128, 16000
    assert pages * H * 64 * D > 1 << 32
    c = ot.kv8_cache(pages, H, D)
    r = np.random.default_rng(11)
    lens = [150, 65, 200]
    table = np.array([[15999, 1, 15997, 0], [0, 15998, 0, 0], [13200, 13106, 13108, 13107]], np.int32)
    small = np.array([[0, 1, 2, 9], [3, 4, 9, 9], [5, 6, 7, 8]], np.int32)
    k, v = K.heads_of(r, sum(lens), H, D), K.heads_of(r, sum(lens), H, D)
    want = O.append(O.empty_cache(10, H, D), k, v, K.rows_of(lens), lens, small)
    cu, l, t = K.ints(K.rows_of(lens)), K.ints(lens), K.ints(table)
    ot.kv8_append(dev(k), dev(v), cu, l, t, c)
    order = torch.from_numpy(np.array([15999, 1, 15997, 0, 15998, 13200, 13106, 13108, 13107])).cuda()
    K.assert_same_cache(K.host([x[order] for x in c]), {n: x for n, x in want.items()}, small, lens, D)
    gk, gv = ot.kv8_read(c, cu, K.ints([0] * 3), t, sum(lens), D)
    wk, wv = O.read(want, K.rows_of(lens), [0] * 3, small, sum(lens), D)
    assert np.array_equal(gk.cpu().numpy(), wk) and np.array_equal(gv.cpu().numpy(), wv)
    for counts in ([1, 1, 1], [40, 33, 50]):
        q = r.normal(size=(sum(counts), H, D)).astype(np.float16)
        Y = ot.attn_kv8(dev(q), K.ints(K.rows_of(counts)), l, t, c, max_q=max(counts))
        within(Y, None, O.attend(want, q, K.rows_of(counts), lens, small, D ** -0.5))


def test_rows_past_32_bits():
    """Tokens so far apart that their elements lie past 2^32, and outputs that do."""
    r = np.random.default_rng(12)
    H, D, T, ld = 2, 64, 70, 1 << 26
    assert T * ld > 1 << 32
    x = torch.empty(T * ld, dtype=torch.float16, device="cuda")
    k, v, q = (x.as_strided((T, H, D), (ld, D, 1), 256 * i) for i in range(3))
    a, b, c = (r.normal(size=(T, H, D)).astype(np.float16) for _ in range(3))
    for t, s in ((k, a), (v, b), (q, c)):
        t.copy_(dev(s))
    table = np.array([[2, 0]], np.int32)
    cu, lens = np.array([0, T]), [T]
    want = O.append(O.empty_cache(3, H, D), a, b, cu, lens, table)
    cache = ot.kv8_cache(3, H, D)
    args = K.ints(cu), K.ints(lens), K.ints(table)
    ot.kv8_append(k, v, *args, cache)
    K.assert_same_cache(K.host(cache), want, table, lens, D)
    within(ot.attn_kv8(q, *args, cache, max_q=T), None, O.attend(want, c, cu, lens, table, D ** -0.5))
    one = K.ints(np.arange(T + 1)), K.ints(np.arange(1, T + 1)), K.ints(np.repeat(table, T, 0))
    within(ot.attn_kv8(q, *one, cache, max_q=1), None, O.attend(want, c, cu, lens, table, D ** -0.5))
    # outputs: 1200 sequences of 60 rows of 256 heads of 256 channels on one page each
    del x, k, v, q
    B, n, Hq, D = 1200, 60, 256, 256
    T = B * n
    assert T * Hq * D > 1 << 32
    cache, table = K.filled(r, [64], 1, D)
    q = torch.randn(n, Hq, D, device="cuda").half().repeat(B, 1, 1)
    Y = torch.empty_like(q)
    lens = K.ints([64] * B)
    ot.ot_attn_kv8(q, K.ints(np.arange(B + 1) * n), lens, K.ints(np.repeat(table, B, 0)), *K.device(cache),
                   0.0625, True, 0, n, Y)
    assert bool((Y.view(B, n, Hq, D) == Y[:n]).all())
    within(Y[:n], None, O.attend(cache, q[:n].cpu().numpy(), [0, n], [64], table, 0.0625))


def test_long_context():
    """160 thousand keys of one sequence, read by one token and by a prompt's piece."""
    r = np.random.default_rng(13)
    H, D, n = 1, 64, 160003
    pages = -(-n // 64)
    table = r.permutation(pages).astype(np.int32)[None]
    cache = O.empty_cache(pages, H, D)
    cache["Kc"][:] = r.integers(1, 256, cache["Kc"].shape)
    cache["Vc"][:] = r.integers(1, 256, cache["Vc"].shape)
    for s in ("Ks", "Vs"):
        cache[s][:] = r.uniform(0.001, 0.02, cache[s].shape)
    for count in (1, 33):
        q = r.normal(size=(count, 2, D)).astype(np.float16)
        cu = [0, count]
        got = ot.attn_kv8(dev(q), K.ints(cu), K.ints([n]), K.ints(table), K.device(cache), max_q=count,
                          want_lse=True)
        within(*got, O.attend(cache, q, cu, [n], table, D ** -0.5))


# --- the method's path ----------------------------------------------------------------

def test_attention_behind_the_qkv_linear():
    """The quality sweep's attention: within what its codes can be off, and every
    configuration of a workload."""
    r = np.random.default_rng(14)
    q, k, v = (dev(r.normal(size=(90, 3, 64)).astype(np.float16)) for _ in range(3))
    ref = quality.attention_ref(q, k, v)
    Y = quality.attention_kv8(q, k, v).double()
    # a code is off by less than one step of its page's scale, amax / 127 and growing by less
    # than 2: values by one step, scores by |q| . step / 8, weights by e^(2 that)
    sk, sv = (2 * float(t.abs().max()) / 127 for t in (k, v))
    dx = float(q.double().abs().sum(2).max()) * sk / 8
    assert float((Y - ref).abs().max()) <= sv + np.expm1(2 * dx) * float(v.abs().max())
    recs = quality.attention_sweep(workloads=("opt13b_w6a6",), rows=64, calib_rows=64, calib_batches=1)
    by = {x["config"]: x["rel_fro"] for x in recs}
    assert list(by) == [c[0] for c in quality.ATTENTION_CONFIGS]
    assert all(0 < e < float("inf") for e in by.values())
