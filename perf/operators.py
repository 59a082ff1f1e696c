"""The operators of a paged key/value cache, as cases that can be timed and compared.

The framework forms the cache of a request as contiguous rows.  A server that answers many requests keeps them in pages
instead, and a decode step over pages needs three things: the pages and rows that the new tokens go to (worked out where
the lengths are, on the GPU), the new tokens' heads normalised, rotated and written to those rows, and the attention of
one new token per request over the pages.

kind     "map"     block tables, slots, position ids and lengths of a batch from its lengths, `cached` tokens held and
                   `new` ones coming per request; the slot arrays have room for `pad` tokens more
         "append"  query and key heads normalised (RMS) and rotated, keys and values written to their slots
         "decode"  one new token per request over its pages; window > 0: the last `window` keys and the first `sinks`
shape    name in SHAPES; page: tokens per page; mix: seed of the sizes

`own` false: plain torch in 32 bits (angles in 64).  `own` true: the calls of `paper_2410_07590_amd.binding`.
"""
import math

import numpy as np
import torch

own = False

#         query heads, KV heads, channels of a head, type
SHAPES = {
    "qwen2-7b": (28, 4, 128, "bf16"),
    "llama3-8b": (32, 8, 128, "bf16"),
    "tiny": (4, 4, 64, "f32"),
    "heads-64": (16, 4, 64, "bf16"),
}
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
EPS = 1e-6
LAYOUTS = {"interleaved": 0, "half": 1}
ORIGINAL_LEN = 8192  # trained context that a "parts" scaling starts from
SLOW_TURNS, FAST_TURNS = 1.0, 32.0


def listed():
    return [
        # the smallest call: five requests of a quiet hour, one new token each
        dict(name="map-5-decode", kind="map", n_req=5, cached_lo=300, cached_hi=3000, new_lo=1, new_hi=1, pad=0, page=16, mix=1),
        # a full batch of prompts behind assembled documents, padded to a fixed launch size
        dict(name="map-256-prompts", kind="map", n_req=256, cached_lo=0, cached_hi=4000, new_lo=0, new_hi=1500, pad=4096, page=16, mix=2),
        # a short question at the tiny fp32 shape: half of each head is rotated
        dict(name="append-tiny-f32-16", kind="append", shape="tiny", tokens=16, pad=0, page=16, layout="interleaved", rot=32,
             scaling="none", factor=1.0, norm=True, queries=True, packed=False, far=0, mix=3),
        # one new token for each request of a full batch
        dict(name="append-decode-64", kind="append", shape="qwen2-7b", tokens=64, pad=0, page=64, layout="half", rot=128,
             scaling="none", factor=1.0, norm=True, queries=True, packed=True, far=4096, mix=4),
        # prompts far behind the trained context, heads of one packed projection, an odd count and padding
        dict(name="append-prompts-16001", kind="append", shape="llama3-8b", tokens=16001, pad=383, page=16, layout="half", rot=128,
             scaling="parts", factor=16.0, norm=True, queries=True, packed=True, far=100000, mix=5),
        # rows of documents into pages: keys turned once, neither norm nor queries
        dict(name="append-documents-24000", kind="append", shape="qwen2-7b", tokens=24000, pad=0, page=32, layout="interleaved", rot=128,
             scaling="none", factor=1.0, norm=False, queries=False, packed=False, far=0, mix=6),
        # one short request by itself, where latency counts
        dict(name="decode-1x700", kind="decode", shape="llama3-8b", n_req=1, lo=700, hi=700, empty=0, page=16, window=0, sinks=0, mix=7),
        # the few requests of a quiet hour, each with its own length, one of them just given up
        dict(name="decode-5-ragged", kind="decode", shape="llama3-8b", n_req=5, lo=300, hi=3000, empty=1, page=16, window=0, sinks=0, mix=8),
        # a full batch
        dict(name="decode-64x4096", kind="decode", shape="qwen2-7b", n_req=64, lo=4096, hi=4096, empty=0, page=64, window=0, sinks=0, mix=9),
        # one very long context by itself: the whole chip on eight heads
        dict(name="decode-1x131071", kind="decode", shape="llama3-8b", n_req=1, lo=131071, hi=131071, empty=0, page=16, window=0, sinks=0, mix=10),
        # long contexts through a window that keeps the first tokens
        dict(name="decode-32-window", kind="decode", shape="llama3-8b", n_req=32, lo=500, hi=32000, empty=0, page=32, window=4000, sinks=4, mix=11),
        # the tiny fp32 shape, ragged
        dict(name="decode-tiny-f32-9", kind="decode", shape="tiny", n_req=9, lo=1, hi=2500, empty=1, page=16, window=0, sinks=0, mix=12),
    ]


# ---- drawn cases ------------------------------------------------------------------------------------------------------------


def _log(rng, lo, hi):
    """An integer of [lo, hi], spread over its logarithm."""
    return max(lo, min(hi, int(round(lo * (hi / lo) ** rng.random()))))


def draw(rng):
    kind = rng.choice(["map", "append", "append", "decode", "decode", "decode"])
    c = dict(kind=kind, page=rng.choice([16, 16, 32, 64, 128, 256]), mix=rng.randrange(1, 1 << 30))
    if kind == "map":
        c["n_req"] = _log(rng, 1, 256)
        c["cached_lo"] = rng.choice([0, rng.randint(0, 2000)])
        c["cached_hi"] = rng.randint(c["cached_lo"], 4000)
        c["new_lo"] = rng.choice([0, 1])
        c["new_hi"] = rng.choice([1, _log(rng, 1, 1500)])
        c["pad"] = rng.choice([0, rng.randint(1, 4096)])
        return c
    c["shape"] = rng.choice(["qwen2-7b", "llama3-8b", "llama3-8b", "heads-64", "tiny"])
    hq, hk, d, t = SHAPES[c["shape"]]
    if kind == "append":
        c["tokens"] = _log(rng, 1, 16000)
        c["pad"] = rng.choice([0, rng.randint(1, 1 + c["tokens"] // 8)])
        c["layout"] = rng.choice(["interleaved", "half"])
        c["rot"] = rng.choice([d, d, d // 2, d // 4])
        c["scaling"] = rng.choice(["none", "linear", "base", "parts"])
        c["factor"] = 1.0 if c["scaling"] == "none" else rng.choice([2.0, 4.0, 16.0])
        c["norm"] = rng.random() < 0.7
        c["queries"] = rng.random() < 0.8
        c["packed"] = rng.random() < 0.5
        c["far"] = rng.choice([0, _log(rng, 100, 500000)])
        return c
    room = 64 * 4096 * 4 * 128 * 2 // (hk * d * (4 if t == "f32" else 2))  # rows that cost what the largest listed case does
    c["n_req"] = _log(rng, 1, 256)
    top = min(131071 if c["n_req"] < 4 else 16384, room // c["n_req"])
    c["lo"] = _log(rng, 1, top)
    c["hi"] = rng.randint(c["lo"], top)
    c["empty"] = rng.choice([0, 0, c["n_req"] // 4])
    c["window"] = rng.choice([0, 0, _log(rng, 1, 4096)])
    c["sinks"] = rng.choice([0, rng.randint(1, 100)]) if c["window"] else 0
    return c


# ---- sizes: functions of the case alone ---------------------------------------------------------------------------------------


def _sizes(case):
    rng = np.random.Generator(np.random.PCG64([20241007, case["mix"]]))
    kind = case["kind"]
    if kind == "map":
        cached = rng.integers(case["cached_lo"], case["cached_hi"] + 1, case["n_req"])
        new = rng.integers(case["new_lo"], case["new_hi"] + 1, case["n_req"])
        first = cached + rng.integers(-50, 51, case["n_req"])  # position ids differ from row indices under composite positions
        return cached, new, np.maximum(first, 0)
    if kind == "append":
        return None
    lens = rng.integers(case["lo"], case["hi"] + 1, case["n_req"])
    if case["empty"]:
        lens[rng.permutation(case["n_req"])[:case["empty"]]] = 0
    return lens


def _visible(case, lens):
    if not case["window"]:
        return lens
    return np.minimum(lens, case["window"] + np.minimum(case["sinks"], np.maximum(lens - case["window"], 0)))


def _pages(tokens, page):
    return -(-tokens // page)


# ---- what a program has in hand before the call ---------------------------------------------------------------------------------


def _ints(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed * 1000003 + case["mix"])
    order = np.random.Generator(np.random.PCG64([seed, case["mix"]]))
    kind, page = case["kind"], case["page"]

    def normal(*size, dtype=torch.float32, scale=1.0, shift=0.0):
        return (torch.randn(*size, generator=gen, device="cuda") * scale + shift).to(dtype)

    st = dict(case=case)
    if kind == "map":
        cached, new, first = _sizes(case)
        have, need = _pages(cached, page), _pages(cached + new, page)
        n = case["n_req"]
        pool = order.permutation(int(need.sum()) + 64)  # pages of the pool in the order in which they came free
        table = np.full((n, int(need.max()) + 3), -1)
        at = 0
        for r in range(n):
            table[r, :have[r]] = pool[at:at + have[r]]
            at += have[r]
        room = int(new.sum()) + case["pad"]
        i32 = dict(dtype=torch.int32, device="cuda")
        st.update(cached=_ints(cached), new=_ints(new), first=_ints(first), free=_ints(pool[at:]), table=_ints(table),
                  kv_lens=torch.empty(n, **i32), cu=torch.empty(n + 1, **i32), slots=torch.empty(room, **i32),
                  pos=torch.empty(room, **i32), counts=torch.empty(2, **i32))
        return st

    hq, hk, d, t = SHAPES[case["shape"]]
    dtype = DTYPES[t]
    if kind == "append":
        n, rows = case["tokens"], case["tokens"] + case["pad"]
        n_pages = _pages(n, page) + 2
        slots = np.full(rows, -1)
        taken = order.permutation(n_pages)[:_pages(n, page)]
        slots[:n] = (taken[:, None] * page + np.arange(page)).reshape(-1)[:n]
        pos = np.zeros(rows)
        pos[:n] = case["far"] + order.integers(0, 64) + np.arange(n)
        if case["packed"]:
            qkv = normal(rows, hq + 2 * hk, d, dtype=dtype)
            q, k, v = qkv[:, :hq], qkv[:, hq:hq + hk], qkv[:, hq + hk:]
        else:
            q, k, v = normal(rows, hq, d, dtype=dtype), normal(rows, hk, d, dtype=dtype), normal(rows, hk, d, dtype=dtype)
        if not case["queries"]:
            q = None
        st.update(q=q, k=k, v=v, pos=_ints(pos), slots=_ints(slots),
                  q_out=torch.empty(rows, hq, d, dtype=dtype, device="cuda") if case["queries"] else None,
                  k_pages=normal(n_pages, page, hk, d, dtype=dtype), v_pages=normal(n_pages, page, hk, d, dtype=dtype),
                  q_norm=normal(d, dtype=dtype, scale=0.2, shift=1.0) if case["norm"] and case["queries"] else None,
                  k_norm=normal(d, dtype=dtype, scale=0.2, shift=1.0) if case["norm"] else None)
        if own:
            from paper_2410_07590_amd import binding as B
            st["shape"] = B.make_shape(hq, hk, d, t, 1e6, LAYOUTS[case["layout"]])
            st["rotary"] = B.tr_rotary_init(LAYOUTS[case["layout"]], case["rot"], 1e6,
                                            {"none": B.TR_SCALE_NONE, "linear": B.TR_SCALE_LINEAR, "base": B.TR_SCALE_BASE,
                                             "parts": B.TR_SCALE_PARTS}[case["scaling"]],
                                            case["factor"], ORIGINAL_LEN, SLOW_TURNS, FAST_TURNS, _amplitude(case))
            st["pages"] = B.make_pages(st["k_pages"], st["v_pages"])
        return st

    lens = _sizes(case)
    need = _pages(lens, page)
    n, n_pages = case["n_req"], int(need.sum()) + 2
    pool = order.permutation(n_pages)
    table = np.full((n, max(int(need.max()), 1)), -1)
    at = 0
    for r in range(n):
        table[r, :need[r]] = pool[at:at + need[r]]
        at += need[r]
    # queries of twice the keys' size: some keys weigh much more than others, as they do where a context is searched
    st.update(q=normal(n, hq, d, dtype=dtype, scale=2.0), k_pages=normal(n_pages, page, hk, d, dtype=dtype),
              v_pages=normal(n_pages, page, hk, d, dtype=dtype), table=_ints(table), kv_lens=_ints(lens),
              out=torch.empty(n, hq, d, dtype=dtype, device="cuda"))
    if own:
        from paper_2410_07590_amd import binding as B
        st["shape"] = B.make_shape(hq, hk, d, t, 1e6)
        st["pages"] = B.make_pages(st["k_pages"], st["v_pages"])
        st["ws"] = B.workspace(B.tr_paged_decode_attn_workspace_size(st["shape"], n, table.shape[1], page))
    return st


# ---- one pass -------------------------------------------------------------------------------------------------------------------


def run(st):
    case = st["case"]
    kind = case["kind"]
    if own:
        from paper_2410_07590_amd import binding as B
        if kind == "map":
            B.tr_page_map(st["cached"], st["new"], st["first"], case["page"], st["free"], st["table"], st["kv_lens"], st["cu"],
                          st["slots"], st["pos"], st["counts"])
        elif kind == "append":
            B.tr_paged_append(st["shape"], st["rotary"], st["q"], st["k"], st["v"], st["q_norm"], st["k_norm"], EPS, st["pos"],
                              st["slots"], st["q_out"], st["pages"])
        else:
            B.tr_paged_decode_attn(st["shape"], st["q"], st["pages"], st["table"], st["kv_lens"], case["window"], case["sinks"],
                                   st["out"], st["ws"])
    elif kind == "map":
        _map_plain(st)
    elif kind == "append":
        _append_plain(st)
    else:
        _decode_plain(st)
    if kind == "map":
        return [st[x] for x in ("table", "kv_lens", "cu", "slots", "pos", "counts")]
    if kind == "append":
        return [st[x] for x in ("q_out", "k_pages", "v_pages") if st[x] is not None]
    return st["out"]


def _map_plain(st):
    page, table = st["case"]["page"], st["table"]
    cached, new = st["cached"].long(), st["new"].long()
    have, need = (cached + page - 1) // page, (cached + new + page - 1) // page
    ends, pages_end = new.cumsum(0), (need - have).cumsum(0)
    first_page = pages_end - (need - have)
    block = torch.arange(table.shape[1], device="cuda")
    taken = (block >= have[:, None]) & (block < need[:, None])
    rank = torch.where(taken, first_page[:, None] + block - have[:, None], 0)
    n_free = st["free"].numel()
    page_id = torch.where(rank < n_free, st["free"][rank.clamp(max=n_free - 1)], -1)
    table.copy_(torch.where(taken, page_id, table))
    t = torch.arange(st["slots"].numel(), device="cuda")
    r = (t[:, None] >= ends).sum(1)  # the request of each token; n_req behind the last one
    live = r < new.numel()
    r = r.clamp(max=new.numel() - 1)
    i = t - (ends - new)[r]
    row = torch.where(live, cached[r] + i, 0)
    blk = (row // page).clamp(max=table.shape[1] - 1)
    page_id = table[r, blk].long()
    held = live & (row // page < table.shape[1]) & (page_id >= 0)
    st["slots"].copy_(torch.where(held, page_id * page + row % page, -1))
    st["pos"].copy_(torch.where(live, st["first"].long()[r] + i, 0))
    st["kv_lens"].copy_(cached + new)
    st["cu"][1:].copy_(ends)
    st["cu"][:1].zero_()
    st["counts"].copy_(torch.stack([ends[-1], pages_end[-1]]))


def _amplitude(case):
    return 0.1 * math.log(case["factor"]) + 1.0 if case["scaling"] == "parts" else 1.0


def _frequencies(case):
    """Radians per position of each pair, in 64 bits."""
    r, base, s = case["rot"], 1e6, case["factor"]
    m = torch.arange(r // 2, dtype=torch.float64, device="cuda")
    if case["scaling"] == "base":
        base = base * s ** (r / (r - 2))
    theta = base ** (-2.0 * m / r)
    if case["scaling"] == "linear":
        theta = theta / s
    if case["scaling"] == "parts":
        turns = ORIGINAL_LEN * theta / (2 * math.pi)
        kept = ((turns - SLOW_TURNS) / (FAST_TURNS - SLOW_TURNS)).clamp(0, 1)
        theta = theta * (kept + (1 - kept) / s)
    return theta


def _append_plain(st):
    case = st["case"]
    angle = st["pos"].double()[:, None] * _frequencies(case)
    cos, sin = ((f(angle) * _amplitude(case)).float()[:, None] for f in (torch.cos, torch.sin))

    def heads(x, weight):
        y, c, s, r = x.float(), cos[:len(x)], sin[:len(x)], case["rot"]
        if weight is not None:
            y = y * torch.rsqrt((y * y).mean(-1, keepdim=True) + EPS) * weight.float()
        if case["layout"] == "half":
            a, b = y[..., :r // 2], y[..., r // 2:r]
            turned = torch.cat([a * c - b * s, b * c + a * s], -1)
        else:
            a, b = y[..., 0:r:2], y[..., 1:r:2]
            turned = torch.stack([a * c - b * s, b * c + a * s], -1).flatten(-2)
        return torch.cat([turned, y[..., r:]], -1).to(x.dtype)

    if st["q"] is not None:
        st["q_out"].copy_(heads(st["q"], st["q_norm"]))
    n = case["tokens"]  # the padding is behind them
    slots = st["slots"][:n].long()
    st["k_pages"].flatten(0, 1)[slots] = heads(st["k"][:n], st["k_norm"])
    st["v_pages"].flatten(0, 1)[slots] = st["v"][:n]


def _decode_plain(st):
    case, q = st["case"], st["q"]
    n, hq, d = q.shape
    hk = st["k_pages"].shape[2]
    step = max(1, (1 << 20) // (st["table"].shape[1] * case["page"]))  # requests whose gathered rows are held at a time
    for r in range(0, n, step):
        table, lens = st["table"][r:r + step], st["kv_lens"][r:r + step, None]
        b, rows = table.shape[0], table.shape[1] * case["page"]
        k, v = (x[table.clamp(min=0)].reshape(b, rows, hk, d).transpose(1, 2).float() for x in (st["k_pages"], st["v_pages"]))
        key = torch.arange(rows, device="cuda")
        seen = key < lens
        if case["window"]:
            seen = seen & ((key < case["sinks"]) | (key >= lens - case["window"]))
        s = torch.matmul(q[r:r + step].float().reshape(b, hk, hq // hk, d), k.transpose(2, 3)) / math.sqrt(d)
        s = torch.where(seen[:, None, None], s, -math.inf)
        top = s.amax(-1, keepdim=True)
        p = torch.exp(s - torch.where(top == -math.inf, 0.0, top))
        total = p.sum(-1, keepdim=True)
        o = torch.matmul(p, torch.where(seen[:, None, :, None], v, 0.0))
        o = torch.where(total > 0, o / total, 0.0)
        st["out"][r:r + step] = o.reshape(b, hq, d).to(q.dtype)


# ---- bytes and operations that a pass cannot do without ---------------------------------------------------------------------------


def work(case):
    kind, page = case["kind"], case["page"]
    if kind == "map":
        cached, new, _ = _sizes(case)
        have, need = _pages(cached, page), _pages(cached + new, page)
        held = int(((cached % page > 0) & (new > 0)).sum())  # entries of pages that are held and take new rows
        tokens = int(new.sum()) + case["pad"]
        words = 3 * case["n_req"] + held + 2 * int((need - have).sum()) + 2 * tokens + 2 * case["n_req"] + 3
        return {"bytes": 4 * words, "flops": 4.0 * tokens}
    hq, hk, d, t = SHAPES[case["shape"]]
    e = 4 if t == "f32" else 2
    if kind == "append":
        rows, n = case["tokens"] + case["pad"], case["tokens"]
        q_heads = rows * hq if case["queries"] else 0
        turned = q_heads + n * hk
        per = 3.0 * case["rot"] + (4.0 * d if case["norm"] else 0.0)
        return {"bytes": 2 * e * d * (q_heads + 2 * n * hk) + 8 * rows, "flops": per * turned}
    lens = _sizes(case)
    seen = int(_visible(case, lens).sum())
    return {"bytes": 2 * e * hk * d * seen + 2 * e * case["n_req"] * hq * d + 4 * int(_pages(lens, page).sum()) + 4 * case["n_req"],
            "flops": 4.0 * hq * d * seen}


# ---- the operators' definitions, in 64 bits -----------------------------------------------------------------------------------------


def exact(case, seed):
    st = prepare(case, seed)
    return {"map": _map_exact, "append": _append_exact, "decode": _decode_exact}[case["kind"]](st)


def _map_exact(st):
    page = st["case"]["page"]
    cached, new, first, free = (st[x].cpu().numpy().astype(np.int64) for x in ("cached", "new", "first", "free"))
    table = st["table"].cpu().numpy().astype(np.int64)
    slots, pos = np.full(st["slots"].numel(), -1, np.int64), np.zeros(st["pos"].numel(), np.int64)
    at = used = 0
    cu = [0]
    for r in range(len(new)):
        for blk in range(-(-int(cached[r]) // page), -(-int(cached[r] + new[r]) // page)):
            table[r, blk] = free[used] if used < len(free) else -1
            used += 1
        rows = cached[r] + np.arange(new[r])
        slots[at:at + new[r]] = table[r, rows // page] * page + rows % page
        pos[at:at + new[r]] = first[r] + np.arange(new[r])
        at += int(new[r])
        cu.append(at)
    return [_ints(x) for x in (table, cached + new, np.array(cu), slots, pos, np.array([at, used]))]


def _append_exact(st):
    case = st["case"]
    r, half = case["rot"], case["rot"] // 2
    s, n = case["factor"], case["tokens"]
    theta = np.array([1e6 ** (-2.0 * m / r) for m in range(half)])
    if case["scaling"] == "linear":
        theta = theta / s
    if case["scaling"] == "base":
        theta = np.array([(1e6 * s ** (r / (r - 2.0))) ** (-2.0 * m / r) for m in range(half)])
    if case["scaling"] == "parts":
        ramp = np.clip((ORIGINAL_LEN * theta / (2 * np.pi) - SLOW_TURNS) / (FAST_TURNS - SLOW_TURNS), 0.0, 1.0)
        theta = theta * ramp + theta / s * (1.0 - ramp)
    a = 1.0 + 0.1 * np.log(s) if case["scaling"] == "parts" else 1.0
    turn = torch.polar(torch.full((len(st["pos"]), half), a, dtype=torch.float64, device="cuda"),
                       st["pos"].double()[:, None] * torch.from_numpy(theta).cuda())

    def heads(x, weight):
        y = x.double().clone()
        if weight is not None:
            y = y / torch.sqrt(y.square().sum(-1, keepdim=True) / y.shape[-1] + EPS) * weight.double()
        re, im = (slice(0, half), slice(half, r)) if case["layout"] == "half" else (slice(0, r, 2), slice(1, r, 2))
        z = torch.complex(y[..., re], y[..., im]) * turn[:len(x), None]
        y[..., re], y[..., im] = z.real, z.imag
        return y

    k_pages, v_pages = st["k_pages"].double(), st["v_pages"].double()
    slots = st["slots"][:n].long()
    page, row = slots // case["page"], slots % case["page"]
    k_pages[page, row] = heads(st["k"][:n], st["k_norm"])
    v_pages[page, row] = st["v"][:n].double()
    return ([heads(st["q"], st["q_norm"])] if st["q"] is not None else []) + [k_pages, v_pages]


def _decode_exact(st):
    case = st["case"]
    n, hq, d = st["q"].shape
    hk = st["k_pages"].shape[2]
    out = torch.zeros(n, hq, d, dtype=torch.float64, device="cuda")
    for r, length in enumerate(_sizes(case).tolist()):
        keys = [j for j in range(length) if not case["window"] or j < case["sinks"] or j >= length - case["window"]]
        if not keys:
            continue
        keys = torch.tensor(keys, device="cuda")
        page = st["table"][r].long()[keys // case["page"]]
        k, v = (x[page, keys % case["page"]].double() for x in (st["k_pages"], st["v_pages"]))
        for h in range(hk):
            heads = slice(h * (hq // hk), (h + 1) * (hq // hk))
            s = (k[:, h] @ st["q"][r, heads].double().T) * d ** -0.5  # [keys, heads]
            w = torch.exp(s - s.max(0).values)
            out[r, heads] = (w / w.sum(0)).T @ v[:, h]
    return out
