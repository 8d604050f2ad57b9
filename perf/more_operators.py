"""Performance cases of the 8-bit key/value cache, with their plain forms.

The cache holds keys and values in pages of 64 tokens.  A page of a head has
64 x Dp codes of 8 bits (Dp: the head's width D rounded up to 64, 96, 128, 192
or 256) and one fp32 scale, for the keys and for the values: a byte b stands for
(b - 128) times the scale.  Key pages are [64 tokens, Dp], value pages
[Dp, 64 tokens].  Token j of sequence b lies in page table[b, j // 64].

A case is one pass through an operator:

  write   new tokens' keys and values are quantized into the pages behind those
          that the sequences have, and the pages that they touched read back
  read    tokens of the cache back in fp16
  attend  attention of new tokens over the cache

`own` chooses between the plain forms in torch and paper_2406_18832_amd.ot.
"""
import math

import torch

own = False

PAGE = 64
WIDTHS = (64, 96, 128, 192, 256)  # of a page's rows


# ---------------------------------------------------------------------------
# The cases.  Sequence b has c tokens in the cache, spread over c_lo..c_hi, and
# n new ones (or n to be read, from token c on), spread over n_lo..n_hi.
# ---------------------------------------------------------------------------
def _write(name, H, D, B, c, n):
    return {"name": name, "kind": "write", "H": H, "G": 1, "D": D, "B": B, "c_lo": c[0],
            "c_hi": c[1], "n_lo": n[0], "n_hi": n[1]}


def _read(name, H, D, B, c, n):
    return {**_write(name, H, D, B, c, n), "kind": "read"}


def _attend(name, H, G, D, B, c, n, causal=True, window=0):
    return {**_write(name, H, D, B, c, n), "kind": "attend", "G": G, "causal": causal,
            "window": window}


def listed():
    return [
        # the smallest: one sequence's next token, OPT-125m, where launches count
        _write("write_125m_1seq", 12, 64, 1, (100, 100), (1, 1)),
        # a decode step's keys and values of 64 sequences, OPT-13B
        _write("write_13b_64seq", 40, 128, 64, (100, 1900), (1, 1)),
        # four prompts of about 2048 tokens, one behind a cached prefix, OPT-30B
        _write("write_30b_prompts", 56, 128, 4, (0, 95), (1900, 2048)),
        # the last tokens of one sequence for another program, from inside a page on
        _read("read_125m_1seq", 12, 64, 1, (37, 37), (300, 300)),
        # the caches of eight sequences handed over, OPT-13B
        _read("read_13b_8seq", 40, 128, 8, (0, 0), (500, 2000)),
        # decode of one short sequence, OPT-125m
        _attend("decode_125m_1seq", 12, 1, 64, 1, (200, 200), (1, 1)),
        # a decode step of 64 sequences of very different lengths, OPT-13B
        _attend("decode_13b_64seq", 40, 1, 128, 64, (100, 2047), (1, 1)),
        # decode over long documents, four query heads to a key head
        _attend("decode_long_4seq", 8, 4, 128, 4, (32000, 131000), (1, 1)),
        # five drafted tokens of 16 sequences checked at once, grouped heads
        _attend("drafts_16seq", 8, 4, 128, 16, (900, 8000), (5, 5)),
        # prompts of very different lengths in one batch, narrow heads of odd width
        _attend("prompts_7seq", 32, 1, 80, 7, (0, 0), (1, 2000)),
        # a piece of two long prompts over what the cache holds, in a sliding window
        _attend("window_piece_2seq", 8, 4, 128, 2, (15000, 20001), (1000, 1024),
                window=4096),
        # the largest: an 8192-token prompt, OPT-66B
        _attend("prompt_66b_8192tok", 72, 1, 128, 1, (0, 0), (8192, 8192)),
    ]


MOST_FLOPS = 4 * 72 * 128 * (8192 * 8193 // 2)
MOST_HELD = 345000 * 8 * 128        # keys in the cache
MOST_NEW = 8192 * 56 * 128          # new keys written or read


def _log_int(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def _heads(rng):
    """Key heads, query heads to each and width."""
    D = rng.choice((64, 64, 80, 96, 112, 128, 128, 128, 144, 256, 16 * rng.randint(1, 16)))
    G = rng.choice((1, 1, 1, 2, 4, 5, 8, 16, 24))
    return _log_int(rng, 1, max(1, 72 // G)), G, D


def _two(rng, lo, hi):
    a, b = _log_int(rng, lo, hi), _log_int(rng, lo, hi)
    return min(a, b), max(a, b)


def draw(rng):
    kind = rng.choice(("write", "write", "read", "decode", "decode", "decode", "drafts",
                       "prompt", "prompt", "piece"))
    H, G, D = _heads(rng)
    B = _log_int(rng, 1, 128)
    if kind in ("write", "read"):
        c = _two(rng, 1, 4096) if rng.random() < 0.8 else (0, 0)
        n = (1, 1) if kind == "write" and rng.random() < 0.4 else _two(rng, 1, 4096)
        make = _write if kind == "write" else _read
        case = make("", H, D, B, c, n)
    else:
        window, causal = 0, True
        if kind == "decode":
            c, n = _two(rng, 1, 131072), (1, 1)
        elif kind == "drafts":
            c, n = _two(rng, 64, 32768), _two(rng, 2, 16)
        elif kind == "prompt":
            c, n = (0, 0), _two(rng, 1, 8192)
            causal = rng.random() < 0.8
        else:
            c, n = _two(rng, 256, 65536), _two(rng, 16, 2048)
        if causal and rng.random() < 0.25:
            window = _log_int(rng, 16, 8192)
        case = _attend("", H, G, D, B, c, n, causal, window)
    while _cost(case) > 1:  # fewer sequences, then shorter ones
        if case["B"] > 1:
            case["B"] = (case["B"] + 1) // 2
        else:
            case["c_lo"], case["c_hi"] = case["c_lo"] // 2, case["c_hi"] // 2
            case["n_lo"], case["n_hi"] = (case["n_lo"] + 1) // 2, (case["n_hi"] + 1) // 2
    return {k: v for k, v in case.items() if k != "name"}


def _spread(lo, hi, B):
    """B whole numbers evenly over lo..hi, neither rising nor falling."""
    if B == 1:
        return [hi]
    even = [lo + (hi - lo) * i // (B - 1) for i in range(B)]
    step = next(s for s in range(max(1, (5 * B) // 8), 2 * B) if math.gcd(s, B) == 1)
    return [even[i * step % B] for i in range(B)]


def _lengths(case):
    """(tokens before, new tokens) of each sequence."""
    return (_spread(case["c_lo"], case["c_hi"], case["B"]),
            _spread(case["n_lo"], case["n_hi"], case["B"])[::-1])


def _cost(case):
    """The largest share of a listed case's most that a case takes."""
    c, n = _lengths(case)
    HD = case["H"] * case["D"]
    held = sum(c) + sum(n)
    share = held * HD / MOST_HELD
    if case["kind"] == "attend":
        return max(share, 4 * case["G"] * HD * _pairs(case) / MOST_FLOPS,
                   sum(n) * case["G"] * HD / MOST_NEW)
    return max(share, sum(n) * HD / MOST_NEW)


def _pairs(case):
    """Visible (query, key) pairs of a query head."""
    total = 0
    for c, n in zip(*_lengths(case)):
        if not case["causal"]:
            total += n * (c + n)
        elif not case["window"]:
            total += n * c + n * (n + 1) // 2
        else:
            full = max(0, min(n, c + n - case["window"] + 1))  # queries with a full window
            total += full * case["window"] + (n - full) * c + (n - full) * (n - full + 1) // 2
    return total


# ---------------------------------------------------------------------------
# Inputs, from the seed alone
# ---------------------------------------------------------------------------
class _Draws:
    """Seeded draws on the GPU."""

    def __init__(self, seed):
        self.g = torch.Generator(device="cuda")
        self.g.manual_seed(seed)

    def normal(self, *shape):
        return torch.randn(*shape, generator=self.g, device="cuda")

    def uniform(self, *shape, lo, hi):
        return torch.rand(*shape, generator=self.g, device="cuda") * (hi - lo) + lo

    def order(self, n):
        return torch.rand(n, generator=self.g, device="cuda").argsort()


def _gains(d, H, D):
    """[H, D] sizes of a head's key channels (a few are much larger than the rest)
    and of its value channels."""
    big = d.uniform(H, D, lo=0.0, hi=1.0) < 0.03
    key = torch.where(big, d.uniform(H, D, lo=4.0, hi=10.0), d.uniform(H, D, lo=0.3, hi=1.2))
    return key, d.uniform(H, D, lo=0.1, hi=1.0)


def _plan(case, d):
    """cu [B + 1], tokens before and after [B], page table [B, most pages + 1] (pages
    in random order, -1 behind a sequence's own), the number of pages, three of them no
    sequence's, and cu as a list."""
    c, n = _lengths(case)
    pages = [-(-(a + b) // PAGE) for a, b in zip(c, n)]
    num = sum(pages) + 3
    order = d.order(num).int()
    table = torch.full((case["B"], max(pages) + 1), -1, dtype=torch.int32, device="cuda")
    at = 0
    for b, p in enumerate(pages):
        table[b, :p] = order[at:at + p]
        at += p
    cu = [0]
    for v in n:
        cu.append(cu[-1] + v)
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    return ints(cu), ints(c), ints([a + b for a, b in zip(c, n)]), table, num, cu


def _held_tokens(case, table, num):
    """[num] tokens that a page holds before the pass."""
    c, n = _lengths(case)
    held = torch.zeros(num, dtype=torch.int64, device="cuda")
    for b in range(case["B"]):
        count = c[b] if case["kind"] == "write" else c[b] + n[b]
        p = -(-count // PAGE)
        if p:
            fill = torch.full((p,), PAGE, device="cuda")
            fill[-1] = count - (p - 1) * PAGE
            held[table[b, :p].long()] = fill
    return held


def _raw_pages(d, case, num):
    """Pages' keys and values before they are quantized, fp16 [pages, H, 64, D], some
    pages at a time: (first page, keys, values)."""
    H, D = case["H"], case["D"]
    gk, gv = _gains(d, H, D)
    step = max(1, (1 << 26) // (H * PAGE * D))
    for at in range(0, num, step):
        p = min(step, num - at)
        k = d.normal(p, H, PAGE, D).mul_(gk[:, None]).half()
        v = d.normal(p, H, PAGE, D).mul_(gv[:, None]).half()
        yield at, k, v


def _draw_tokens(d, case):
    """The new tokens' queries, keys and values as the linear in front leaves them:
    fp16 [T, (H G + 2 H) D]."""
    T, H, G, D = sum(_lengths(case)[1]), case["H"], case["G"], case["D"]
    gk, gv = _gains(d, H, D)
    x = d.normal(T, (G + 2) * H, D)
    x[:, G * H:(G + 1) * H] *= gk
    x[:, (G + 1) * H:] *= gv
    return x.half().reshape(T, -1)


def _split(x, H, G, D):
    """Queries, keys and values [T, heads, D] in x, without a copy."""
    T = x.shape[0]
    q, k, v = x.split((H * G * D, H * D, H * D), 1)
    return q.view(T, H * G, D), k.view(T, H, D), v.view(T, H, D)


# ---------------------------------------------------------------------------
# The format in torch
# ---------------------------------------------------------------------------
def _codes(x, s):
    """Codes of x for the scales s (fp32, broadcast); 0 where the scale is 0."""
    inv = torch.where(s > 0, 1 / s, torch.zeros_like(s))
    return torch.round(x.float() * inv).clamp_(-127, 127)


def _quantized(raw, held):
    """fp16 [pages, H, 64, D] of which page p's first held[p] tokens count ->
    codes (fp32, 0 past those) and scales [pages, H]."""
    live = (torch.arange(PAGE, device="cuda") < held[:, None])[:, None, :, None]
    raw = torch.where(live, raw, torch.zeros_like(raw))
    s = raw.abs().amax((2, 3)).float() / 127
    return _codes(raw, s[:, :, None, None]), s


def _cache(d, case, table, num):
    """(Kc, Vc, Ks, Vs)."""
    H, D = case["H"], case["D"]
    Dp = next(w for w in WIDTHS if w >= D)
    Kc = torch.zeros(num, H, PAGE, Dp, dtype=torch.uint8, device="cuda")
    Vc = torch.zeros(num, H, Dp, PAGE, dtype=torch.uint8, device="cuda")
    Ks, Vs = (torch.zeros(num, H, device="cuda") for _ in range(2))
    held = _held_tokens(case, table, num)
    for at, k, v in _raw_pages(d, case, num):
        here = slice(at, at + k.shape[0])
        codes, Ks[here] = _quantized(k, held[here])
        Kc[here, :, :, :D] = (codes + 128).byte()
        codes, Vs[here] = _quantized(v, held[here])
        Vc[here, :, :D] = (codes + 128).byte().transpose(2, 3)
    return Kc, Vc, Ks, Vs


# ---------------------------------------------------------------------------
# What a program has in hand before the call
# ---------------------------------------------------------------------------
def _empty(dtype, *shape):
    return torch.empty(shape, dtype=dtype, device="cuda")


def _first_touched(case):
    """Where each sequence's pages with new tokens begin, and their tokens from there."""
    c, n = _lengths(case)
    first = [v // PAGE * PAGE for v in c]
    return first, [a + b - f for a, b, f in zip(c, n, first)]


def prepare(case, seed):
    d = _Draws(seed)
    H, G, D = case["H"], case["G"], case["D"]
    cu, before, after, table, num, rows = _plan(case, d)
    state = {"case": case, "cu": cu, "before": before, "after": after, "table": table,
             "lengths": _lengths(case), "cache": _cache(d, case, table, num)}
    if case["kind"] != "read":
        state["x"] = _draw_tokens(d, case)
    if case["kind"] == "attend":
        state["Y"] = _empty(torch.float16, rows[-1], H * G, D)
        state["scale"] = D ** -0.5
        return state
    free = torch.ones(num, dtype=torch.bool, device="cuda")
    free[table[table >= 0].long()] = False
    state["spare"] = int(free.nonzero()[0])  # takes what the plain form has no page for
    first, count = _first_touched(case) if case["kind"] == "write" else state["lengths"]
    state["first"] = torch.tensor(first, dtype=torch.int32, device="cuda")
    state["back"] = torch.tensor([0] + count, device="cuda").cumsum(0).int()
    total = sum(count)
    state["out"] = tuple(_empty(torch.float16, total, H, D) for _ in range(2))
    return state


# ---------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------
def _positions(cu, first, total):
    """Sequence and position of each row: row cu[b] + i is token first[b] + i."""
    rows = torch.arange(total, device="cuda")
    b = torch.searchsorted(cu[1:].long(), rows, right=True)
    return b, rows - cu[b] + first[b]


def _plain_write(state, pages, scales, x, keys):
    """x [T, H, D] into one half of the cache (pages and scales), in place."""
    case, table = state["case"], state["table"]
    H, D, P = case["H"], case["D"], table.shape[1]
    b, pos = _positions(state["cu"], state["before"], x.shape[0])
    # the largest new value in each page and head
    spot = b * P + pos // PAGE
    most = torch.zeros(case["B"] * P, H, device="cuda")
    most.index_reduce_(0, spot, x.float().abs().amax(2), "amax")
    # pages that hold earlier tokens: at most a sequence's first
    col = state["before"].long() // PAGE
    n0 = state["before"].long() % PAGE
    n0 = torch.where(state["after"] > state["before"], n0, torch.zeros_like(n0))
    here = torch.arange(case["B"], device="cuda") * P + col
    s = most / 127
    page = table.gather(1, col[:, None])[:, 0].clamp(min=0).long()
    old = scales[page]
    wide = old * 127.5
    k = torch.where(old > 0, most[here] / wide, torch.ones_like(old)).log2().ceil().clamp(min=0)
    k = k + (torch.ldexp(wide, k) < most[here]).float()       # the logarithm's rounding
    k = k - ((k > 0) & (torch.ldexp(wide, k - 1) >= most[here])).float()
    grown = torch.where(old > 0, torch.ldexp(old, k), s[here])
    kept = (n0 > 0)[:, None]
    s[here] = torch.where(kept, grown, s[here])
    # their earlier codes under the new scale
    block = pages[page] if keys else pages[page].transpose(2, 3)
    codes = block.float() - 128
    shrunk = torch.round(torch.ldexp(codes, torch.where(kept, -k, 0 * k)[:, :, None, None]))
    live = (torch.arange(PAGE, device="cuda") < n0[:, None])[:, None, :, None]
    block = torch.where(live, (shrunk + 128).byte(), block)
    target = torch.where(n0 > 0, page, torch.full_like(page, state["spare"]))
    pages[target] = block if keys else block.transpose(2, 3)
    rows = table[b, pos // PAGE].long()
    scales[rows] = s[spot]
    c = (_codes(x, s[spot][:, :, None]) + 128).byte()
    if keys:
        pages[rows, :, pos % PAGE, :D] = c
    else:
        pages[rows, :, :D, pos % PAGE] = c


def _plain_read(state, pages, scales, keys):
    D = state["case"]["D"]
    b, pos = _positions(state["back"], state["first"], state["out"][0].shape[0])
    page, at = state["table"][b, pos // PAGE].long(), pos % PAGE
    codes = pages[page, :, at, :D] if keys else pages[page, :, :D, at]
    return ((codes.float() - 128) * scales[page][:, :, None]).half()


def _plain_attend(state):
    case = state["case"]
    H, G, D = case["H"], case["G"], case["D"]
    q, _, _ = _split(state["x"], H, G, D)
    Kc, Vc, Ks, Vs = state["cache"]
    at = 0
    for b, (c, n) in enumerate(zip(*state["lengths"])):
        L = c + n
        page = state["table"][b, :-(-L // PAGE)].long()
        i, j = torch.arange(c, L, device="cuda"), torch.arange(L, device="cuda")
        hidden = None
        if case["causal"]:
            hidden = j > i[:, None]
            if case["window"]:
                hidden = hidden | (j <= i[:, None] - case["window"])
        step = max(1, (1 << 28) // (G * n * L))  # heads at a time
        for h in range(0, H, step):
            here = slice(h, min(h + step, H))
            k = (Kc[page, here, :, :D].float() - 128) * Ks[page, here][:, :, None, None]
            k = k.permute(1, 3, 0, 2).reshape(k.shape[1], D, -1)[:, :, :L].contiguous()
            v = (Vc[page, here, :D].float() - 128) * Vs[page, here][:, :, None, None]
            v = v.permute(1, 0, 3, 2).reshape(v.shape[1], -1, D)[:, :L].contiguous()
            x = q[at:at + n, h * G:(h + k.shape[0]) * G].float().reshape(n, -1, G, D)
            x = x.permute(1, 2, 0, 3).reshape(k.shape[0], G * n, D)
            s = (torch.bmm(x, k) * state["scale"]).reshape(-1, G, n, L)
            if hidden is not None:
                s.masked_fill_(hidden, float("-inf"))
            s = (s - s.amax(3, keepdim=True)).exp_()
            y = torch.bmm(s.reshape(-1, G * n, L), v) / s.sum(3).reshape(-1, G * n, 1)
            y = y.reshape(-1, G, n, D).permute(2, 0, 1, 3).reshape(n, -1, D)
            state["Y"][at:at + n, h * G:(h + k.shape[0]) * G] = y.half()
        at += n
    return state["Y"]


def _run_plain(state):
    case = state["case"]
    if case["kind"] == "attend":
        return _plain_attend(state)
    Kc, Vc, Ks, Vs = state["cache"]
    if case["kind"] == "write":
        _, k, v = _split(state["x"], case["H"], 1, case["D"])
        _plain_write(state, Kc, Ks, k, True)
        _plain_write(state, Vc, Vs, v, False)
    return _plain_read(state, Kc, Ks, True), _plain_read(state, Vc, Vs, False)


def _run_own(state):
    from paper_2406_18832_amd import ot
    case = state["case"]
    H, G, D = case["H"], case["G"], case["D"]
    if case["kind"] == "attend":
        n = case["n_hi"]
        q, _, _ = _split(state["x"], H, G, D)
        if "scratch" not in state:
            state["scratch"] = ot.attn_kv8_workspace_for(q.shape[0], case["B"], H * G, H, D, n)
        ot.ot_attn_kv8(q, state["cu"], state["after"], state["table"], *state["cache"],
                       state["scale"], case["causal"], case["window"], n, state["Y"], None,
                       state["scratch"])
        return state["Y"]
    if case["kind"] == "write":
        _, k, v = _split(state["x"], H, G, D)
        ot.ot_kv8_append(k, v, state["cu"], state["after"], state["table"], *state["cache"])
    ot.ot_kv8_read(*state["cache"], state["back"], state["first"], state["table"],
                   *state["out"])
    return state["out"]


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ---------------------------------------------------------------------------
# What a pass cannot do without
# ---------------------------------------------------------------------------
def work(case):
    c, n = _lengths(case)
    H, G, D = case["H"], case["G"], case["D"]
    pages = sum(-(-(a + b) // PAGE) for a, b in zip(c, n))
    if case["kind"] == "write":
        first, count = _first_touched(case)
        old = sum(a - f for a, f in zip(c, first))
        return {"bytes": 6 * sum(n) * H * D + 2 * old * H * D + 4 * sum(count) * H * D,
                "flops": 0}
    if case["kind"] == "read":
        return {"bytes": 6 * sum(n) * H * D, "flops": 0}
    if case["window"]:  # keys that some query sees
        seen = sum(min(a + b, case["window"] + b - 1) for a, b in zip(c, n))
    else:
        seen = sum(c) + sum(n)
    return {"bytes": 2 * seen * H * D + 8 * pages * H + 4 * sum(n) * H * G * D,
            "flops": 4 * H * G * D * _pairs(case)}


# ---------------------------------------------------------------------------
# The same outputs from the definitions in 64 bits
# ---------------------------------------------------------------------------
def _r32(v):
    return v.float().double()


def _exact_scale(most):
    return (most.double() / 127).float().double()


def _exact_codes(x, s):
    inv = torch.where(s > 0, _r32(1 / s.clamp(min=1e-300)), 0 * s)
    return _r32(x.double() * inv).round().clamp(-127, 127)


def _exact_pages(d, case, table, num, wanted):
    """Codes [len(wanted), H, 64, D] and scales, float64, of keys and of values of the
    wanted pages (the draws of the others are passed over)."""
    H, D = case["H"], case["D"]
    held = _held_tokens(case, table, num)
    out = [torch.zeros(len(wanted), H, PAGE, D, dtype=torch.int8, device="cuda") for _ in range(2)]
    scale = [torch.zeros(len(wanted), H, dtype=torch.float64, device="cuda") for _ in range(2)]
    where = torch.full((num,), -1, dtype=torch.int64, device="cuda")
    where[wanted] = torch.arange(len(wanted), device="cuda")
    for at, k, v in _raw_pages(d, case, num):
        to = where[at:at + k.shape[0]]
        some = (to >= 0).nonzero()[:, 0]
        if not some.numel():
            continue
        for i, x in enumerate((k, v)):
            x = x[some].clone()
            for t in range(PAGE):
                x[held[at + some] <= t, :, t] = 0
            s = _exact_scale(x.reshape(x.shape[0], H, -1).abs().max(2).values)
            out[i][to[some]] = _exact_codes(x, s[:, :, None, None]).to(torch.int8)
            scale[i][to[some]] = s
    return out, scale


def exact(case, seed):
    d = _Draws(seed)
    H, G, D = case["H"], case["G"], case["D"]
    c, n = _lengths(case)
    _, _, _, table, num, cu = _plan(case, d)
    spans = [range((a if case["kind"] != "attend" else 0) // PAGE, -(-(a + m) // PAGE))
             for a, m in zip(c, n)]
    wanted = torch.cat([table[b, r.start:r.stop] for b, r in enumerate(spans)]).long()
    codes, scale = _exact_pages(d, case, table, num, wanted)
    x = None if case["kind"] == "read" else _draw_tokens(d, case)
    if case["kind"] == "read":
        parts, at = ([], []), 0
        for b, r in enumerate(spans):
            for i in range(2):
                page = codes[i][at:at + len(r)].double() * scale[i][at:at + len(r), :, None, None]
                rows = page.transpose(1, 2).reshape(-1, H, D)
                parts[i].append(rows[c[b] - r.start * PAGE:c[b] + n[b] - r.start * PAGE])
            at += len(r)
        return torch.cat(parts[0]), torch.cat(parts[1])
    if case["kind"] == "write":
        new = _split(x, H, G, D)[1:]
        parts, at = ([], []), 0
        for b, r in enumerate(spans):
            for p in r:
                lo, hi = max(c[b], p * PAGE), min(c[b] + n[b], (p + 1) * PAGE)
                had = max(0, c[b] - p * PAGE)  # tokens that the page had
                for i in range(2):
                    rows = new[i][cu[b] + lo - c[b]:cu[b] + hi - c[b]]
                    most = rows.abs().amax((0, 2))
                    s, old = _exact_scale(most), codes[i][at, :, :had].double()
                    if had:
                        before = scale[i][at]
                        k = torch.zeros_like(before)
                        top = _r32(before * 127.5)
                        while bool(((before > 0) & (top * 2 ** k < most)).any()):
                            k += ((before > 0) & (top * 2 ** k < most)).double()
                        s = torch.where(before > 0, before * 2 ** k, s)
                        old = (old * (2 ** -k)[:, None, None]).round()
                    fresh = _exact_codes(rows, s[None, :, None])
                    parts[i].append(torch.cat((old.transpose(0, 1), fresh)) * s[None, :, None])
                at += 1
        return torch.cat(parts[0]), torch.cat(parts[1])
    q = _split(x, H, G, D)[0].double()
    Y = torch.zeros(q.shape[0], H * G, D, dtype=torch.float64, device="cuda")
    at = 0
    for b, r in enumerate(spans):
        L, pos = c[b] + n[b], torch.arange(c[b], c[b] + n[b], device="cuda")
        key = torch.arange(L, device="cuda")
        for h in range(H):
            k, v = ((codes[i][at:at + len(r), h].double()
                     * scale[i][at:at + len(r), h, None, None]).reshape(-1, D)[:L]
                    for i in range(2))
            for g in range(h * G, (h + 1) * G):
                rows = q[cu[b]:cu[b + 1], g]
                s = rows @ k.t() / math.sqrt(D)
                if case["causal"]:
                    ahead = key[None, :] - pos[:, None]
                    s[ahead > 0] = -math.inf
                    if case["window"]:
                        s[ahead <= -case["window"]] = -math.inf
                Y[cu[b]:cu[b + 1], g] = torch.softmax(s, 1) @ v
        at += len(r)
    return Y
