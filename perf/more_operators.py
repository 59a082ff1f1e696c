"""The operators of a paged key/value cache held in 8 bits, as cases that can be timed and compared.

A cache in 8 bits holds twice the tokens and, where attention is bound by reading it, answers in half the time.  Keys and values
are e4m3 codes; each block of 16 rows of a page has, for each KV head, one scale for its keys and one for its values, a power of
two (e8m0): the smallest 2^e with |x| <= 448 * 2^e for all x of the block.  Three operators go with such a cache:

kind     "append"  query and key heads normalised (RMS) and rotated, keys and values quantised as they are written to their slots.  A
                   block whose first row is written starts anew; of any other the scale is what it was or, where new rows need
                   it, a larger one, at which the rows that it holds are written again.
         "read"    the rows of a batch of requests back from the pages as contiguous rows (what prefill attention reads)
         "decode"  attention of one new token per request over the pages; window > 0: the last `window` keys and the first `sinks`
shape    name in SHAPES; page: tokens per page; order "rows": pools [page, row, head, channel], "heads": [page, head, row, channel];
mix      seed of the sizes

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
BLOCK = 16             # rows that share a scale
LEAST, MOST = -117, 120  # exponents of scales: every value that a code stands for is a normal fp32 and bf16 number
MOST_TOKENS = 16400    # of a drawn append


def listed():
    return [
        # the smallest call: one request, one new token
        dict(name="append-1", kind="append", shape="qwen2-7b", n_req=1, cached_lo=700, cached_hi=700, new_lo=1, new_hi=1, pad=0, page=16,
             order="rows", layout="half", rot=128, norm=True, queries=True, packed=True, far=0, mix=1),
        # one new token for each request of a full batch, at any row of its block
        dict(name="append-decode-64", kind="append", shape="qwen2-7b", n_req=64, cached_lo=100, cached_hi=9000, new_lo=1, new_hi=1, pad=0,
             page=64, order="rows", layout="half", rot=128, norm=True, queries=True, packed=True, far=0, mix=2),
        # prompts behind what is held already, heads of one packed projection, padded to a fixed launch size
        dict(name="append-prompts-16000", kind="append", shape="llama3-8b", n_req=16, cached_lo=0, cached_hi=300, new_lo=1000, new_hi=1000,
             pad=384, page=16, order="rows", layout="half", rot=128, norm=False, queries=True, packed=True, far=0, mix=3),
        # short questions at the tiny fp32 shape: half of each head is rotated
        dict(name="append-tiny-f32-6", kind="append", shape="tiny", n_req=6, cached_lo=0, cached_hi=90, new_lo=1, new_hi=40, pad=5, page=32,
             order="heads", layout="interleaved", rot=32, norm=True, queries=True, packed=False, far=4096, mix=4),
        # one short request
        dict(name="read-1x700", kind="read", shape="qwen2-7b", n_req=1, lo=700, hi=700, empty=0, page=16, order="rows", mix=5),
        # the documents of a batch whose questions are answered next, a request just given up among them
        dict(name="read-16-ragged", kind="read", shape="llama3-8b", n_req=16, lo=300, hi=9000, empty=1, page=64, order="rows", mix=6),
        # the tiny fp32 shape, ragged
        dict(name="read-tiny-f32-9", kind="read", shape="tiny", n_req=9, lo=1, hi=2500, empty=2, page=32, order="heads", mix=7),
        # one short request by itself, where latency counts
        dict(name="decode-1x700", kind="decode", shape="llama3-8b", n_req=1, lo=700, hi=700, empty=0, page=16, order="rows", window=0, sinks=0, mix=8),
        # the few requests of a quiet hour at the tiny fp32 shape, each with its own length, one of them just given up
        dict(name="decode-tiny-f32-9", kind="decode", shape="tiny", n_req=9, lo=1, hi=2500, empty=1, page=32, order="rows", window=0, sinks=0, mix=9),
        # a full batch of long contexts
        dict(name="decode-64x8192", kind="decode", shape="qwen2-7b", n_req=64, lo=8192, hi=8192, empty=0, page=64, order="rows", window=0, sinks=0, mix=10),
        # one very long context by itself: the whole chip on eight heads
        dict(name="decode-1x131071", kind="decode", shape="llama3-8b", n_req=1, lo=131071, hi=131071, empty=0, page=16, order="rows", window=0, sinks=0,
             mix=11),
        # long contexts through a window that keeps the first tokens
        dict(name="decode-32-window", kind="decode", shape="llama3-8b", n_req=32, lo=500, hi=16000, empty=0, page=32, order="heads", window=4000, sinks=4,
             mix=12),
    ]


# ---- drawn cases ------------------------------------------------------------------------------------------------------------


def _log(rng, lo, hi):
    """An integer of [lo, hi], spread over its logarithm."""
    return max(lo, min(hi, int(round(lo * (hi / lo) ** rng.random()))))


def draw(rng):
    kind = rng.choice(["append", "append", "read", "decode", "decode", "decode"])
    c = dict(kind=kind, shape=rng.choice(["qwen2-7b", "llama3-8b", "llama3-8b", "heads-64", "tiny"]), n_req=_log(rng, 1, 256),
             page=rng.choice([16, 16, 32, 64, 128, 256]), order=rng.choice(["rows", "heads"]), mix=rng.randrange(1, 1 << 30))
    hq, hk, d, t = SHAPES[c["shape"]]
    if kind == "append":
        c["cached_lo"] = rng.choice([0, rng.randint(0, 2000)])
        c["cached_hi"] = rng.randint(c["cached_lo"], 4000)
        c["new_hi"] = rng.choice([1, _log(rng, 1, MOST_TOKENS // c["n_req"])])
        c["new_lo"] = rng.randint(1, c["new_hi"])
        c["pad"] = rng.choice([0, rng.randint(1, 512)])
        c["layout"] = rng.choice(["interleaved", "half"])
        c["rot"] = rng.choice([d, d, d // 2, d // 4])
        c["norm"] = rng.random() < 0.7
        c["queries"] = rng.random() < 0.8
        c["packed"] = rng.random() < 0.5
        c["far"] = rng.choice([0, _log(rng, 100, 500000)])
        return c
    # rows that cost what the largest listed cases do
    room = 64 * 8192 * 4 * 128 // (hk * d) if kind == "decode" else 60000 * 8 * 128 * 2 // (hk * d * (4 if t == "f32" else 2))
    top = min(131071 if c["n_req"] < 4 else 16384, room // c["n_req"])
    c["lo"] = _log(rng, 1, top)
    c["hi"] = rng.randint(c["lo"], top)
    c["empty"] = rng.choice([0, 0, c["n_req"] // 4])
    if kind == "decode":
        c["window"] = rng.choice([0, 0, _log(rng, 1, 4096)])
        c["sinks"] = rng.choice([0, rng.randint(1, 100)]) if c["window"] else 0
    return c


# ---- sizes: functions of the case alone ---------------------------------------------------------------------------------------


def _sizes(case):
    rng = np.random.Generator(np.random.PCG64([20241007, case["mix"]]))
    if case["kind"] == "append":
        cached = rng.integers(case["cached_lo"], case["cached_hi"] + 1, case["n_req"])
        return cached, rng.integers(case["new_lo"], case["new_hi"] + 1, case["n_req"])
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


def _pool(case, n_pages, normal):
    """Codes and scales of a pool that is in use: a few channels of each head are several times as large as the others."""
    _, hk, d, _ = SHAPES[case["shape"]]
    page = case["page"]

    def side(outliers):
        x = normal(n_pages, page // BLOCK, BLOCK, hk, d)
        if outliers:
            x[..., ::29] *= 6.0
        e = _exponent(x.abs().amax((2, 4)))
        codes = torch.ldexp(x, -e[:, :, None, :, None]).to(torch.float8_e4m3fn).reshape(n_pages, page, hk, d)
        if case["order"] == "heads":
            codes = codes.transpose(1, 2).contiguous().transpose(1, 2)
        return codes, (e + 127).to(torch.uint8).transpose(1, 2).contiguous().view(torch.float8_e8m0fnu)

    (k, ks), (v, vs) = side(True), side(False)
    return dict(k_pages=k, v_pages=v, k_scale=ks, v_scale=vs)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed * 1000003 + case["mix"])
    order = np.random.Generator(np.random.PCG64([seed, case["mix"]]))
    kind, page, n = case["kind"], case["page"], case["n_req"]
    hq, hk, d, t = SHAPES[case["shape"]]
    dtype = DTYPES[t]

    def normal(*size, dtype=torch.float32, scale=1.0, shift=0.0):
        return (torch.randn(*size, generator=gen, device="cuda") * scale + shift).to(dtype)

    st = dict(case=case)
    if kind == "append":
        cached, new = _sizes(case)
        tokens = int(new.sum())
        rows = tokens + case["pad"]
        first_page = cached // page  # pages in front of it are not touched, and not made
        need = _pages(cached + new, page) - first_page
        pool, at, slots, pos = order.permutation(int(need.sum()) + 2), 0, [], []
        for r in range(n):
            row = cached[r] + np.arange(new[r])
            slots.append(pool[at + row // page - first_page[r]] * page + row % page)
            pos.append(case["far"] + row)
            at += int(need[r])
        slots = np.concatenate(slots + [np.full(case["pad"], -1)])
        pos = np.concatenate(pos + [np.zeros(case["pad"])])
        if case["packed"]:
            qkv = normal(rows, hq + 2 * hk, d, dtype=dtype)
            q, k, v = qkv[:, :hq], qkv[:, hq:hq + hk], qkv[:, hq + hk:]
        else:
            q, k, v = normal(rows, hq, d, dtype=dtype), normal(rows, hk, d, dtype=dtype), normal(rows, hk, d, dtype=dtype)
        queries, norm = case["queries"], case["norm"]
        st.update(_pool(case, len(pool), normal), tokens=tokens, q=q if queries else None, k=k, v=v, pos=_ints(pos), slots=_ints(slots),
                  q_out=torch.empty(rows, hq, d, dtype=dtype, device="cuda") if queries else None,
                  q_norm=normal(d, dtype=dtype, scale=0.2, shift=1.0) if norm and queries else None,
                  k_norm=normal(d, dtype=dtype, scale=0.2, shift=1.0) if norm else None)
        if own:
            from paper_2410_07590_amd import binding as B
            st["shape"] = B.make_shape(hq, hk, d, t, 1e6, LAYOUTS[case["layout"]])
            st["rotary"] = B.tr_rotary_init(LAYOUTS[case["layout"]], case["rot"], 1e6)
            st["pages"] = B.make_pages_q8(st["k_pages"], st["v_pages"], st["k_scale"], st["v_scale"])
        return st

    lens = _sizes(case)
    need = _pages(lens, page)
    pool = order.permutation(int(need.sum()) + 2)
    table = np.full((n, max(int(need.max()), 1)), -1)
    at = 0
    for r in range(n):
        table[r, :need[r]] = pool[at:at + need[r]]
        at += need[r]
    st.update(_pool(case, len(pool), normal), table=_ints(table), kv_lens=_ints(lens))
    if kind == "read":
        total = int(lens.sum())
        st.update(row_start=_ints(np.concatenate([[0], np.cumsum(lens)])), out_k=torch.empty(total, hk, d, dtype=dtype, device="cuda"),
                  out_v=torch.empty(total, hk, d, dtype=dtype, device="cuda"))
    else:
        st.update(q=normal(n, hq, d, dtype=dtype), out=torch.empty(n, hq, d, dtype=dtype, device="cuda"))
    if own:
        from paper_2410_07590_amd import binding as B
        st["shape"] = B.make_shape(hq, hk, d, t, 1e6)
        st["pages"] = B.make_pages_q8(st["k_pages"], st["v_pages"], st["k_scale"], st["v_scale"])
        if kind == "decode":
            st["ws"] = B.workspace(B.tr_paged_decode_attn_q8_workspace_size(st["shape"], n, table.shape[1], page))
    return st


# ---- one pass -------------------------------------------------------------------------------------------------------------------


def run(st):
    case = st["case"]
    kind = case["kind"]
    if own:
        from paper_2410_07590_amd import binding as B
        if kind == "append":
            B.tr_paged_append_q8(st["shape"], st["rotary"], st["q"], st["k"], st["v"], st["q_norm"], st["k_norm"], EPS, st["pos"],
                                 st["slots"], st["q_out"], st["pages"])
        elif kind == "read":
            B.tr_paged_read_q8(st["shape"], st["pages"], st["table"], st["kv_lens"], st["row_start"], st["out_k"], st["out_v"])
        else:
            B.tr_paged_decode_attn_q8(st["shape"], st["q"], st["pages"], st["table"], st["kv_lens"], case["window"], case["sinks"],
                                      st["out"], st["ws"])
    elif kind == "append":
        _append_plain(st)
    elif kind == "read":
        _read_plain(st)
    else:
        _decode_plain(st)
    if kind == "append":  # codes and scales as tensors of their 8-bit types: the numbers that they stand for, not their bits
        return [st[x] for x in ("q_out", "k_pages", "v_pages", "k_scale", "v_scale") if st[x] is not None]
    return [st["out_k"], st["out_v"]] if kind == "read" else st["out"]


def _exponent(top):
    """The smallest e with top <= 448 * 2^e = 0.875 * 2^(e + 9)."""
    m, e = torch.frexp(top)
    return torch.where(top > 0, e - 9 + (m > 0.875), LEAST).clamp(LEAST, MOST)


def _append_plain(st):
    case = st["case"]
    theta = 1e6 ** (-2.0 * torch.arange(case["rot"] // 2, dtype=torch.float64, device="cuda") / case["rot"])
    angle = st["pos"].double()[:, None] * theta
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]

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
        return torch.cat([turned, y[..., r:]], -1)

    if st["q"] is not None:
        st["q_out"].copy_(heads(st["q"], st["q_norm"]))
    n, page = st["tokens"], case["page"]  # the padding is behind them
    slots = st["slots"][:n].long()
    block, member = torch.unique(slots // BLOCK, return_inverse=True)
    at, of = block // (page // BLOCK), block % (page // BLOCK)
    anew = torch.zeros_like(block).index_add_(0, member, (slots % BLOCK == 0).long()) > 0
    rows = (at[:, None], of[:, None] * BLOCK + torch.arange(BLOCK, device="cuda"))

    def write(x, codes, scale):
        codes, scale = codes.view(torch.uint8), scale.view(torch.uint8)
        top = torch.zeros(len(block), x.shape[1], device="cuda").index_reduce_(0, member, x.abs().amax(-1), "amax")
        need, old = _exponent(top), scale[at, :, of].int() - 127
        e = torch.where(anew[:, None], need, torch.maximum(need, old))
        step = torch.where(anew[:, None], 0, old - e)[:, None, :, None]  # rows of a block that starts anew stay as they are
        held = codes[rows]
        again = torch.ldexp(held.view(torch.float8_e4m3fn).float(), step).to(torch.float8_e4m3fn).view(torch.uint8)
        codes[rows] = torch.where(step < 0, again, held)
        codes[slots // page, slots % page] = torch.ldexp(x, -e[member][..., None]).to(torch.float8_e4m3fn).view(torch.uint8)
        scale[at, :, of] = (e + 127).to(torch.uint8)

    write(heads(st["k"][:n], st["k_norm"]), st["k_pages"], st["k_scale"])
    write(st["v"][:n].float(), st["v_pages"], st["v_scale"])


def _values(codes, scale, table):
    """[requests, heads, rows, channels] in fp32: what the pages of each row of the table stand for."""
    at = table.clamp(min=0).long()
    x = codes.view(torch.uint8)[at].view(torch.float8_e4m3fn).float()  # [requests, blocks, page, heads, channels]
    e = scale.view(torch.uint8)[at].int() - 127  # [requests, blocks, heads, page / 16]
    x = torch.ldexp(x, e.repeat_interleave(BLOCK, 3).transpose(2, 3)[..., None])
    return x.flatten(1, 2).transpose(1, 2)


def _read_plain(st):
    k, v = (_values(st[c], st[s], st["table"]).transpose(1, 2) for c, s in (("k_pages", "k_scale"), ("v_pages", "v_scale")))
    held = torch.arange(k.shape[1], device="cuda") < st["kv_lens"][:, None]
    st["out_k"].copy_(k[held])
    st["out_v"].copy_(v[held])


def _decode_plain(st):
    case, q = st["case"], st["q"]
    n, hq, d = q.shape
    hk = st["k_pages"].shape[2]
    k, v = _values(st["k_pages"], st["k_scale"], st["table"]), _values(st["v_pages"], st["v_scale"], st["table"])
    key, lens = torch.arange(k.shape[2], device="cuda"), st["kv_lens"][:, None]
    seen = key < lens
    if case["window"]:
        seen = seen & ((key < case["sinks"]) | (key >= lens - case["window"]))
    s = torch.matmul(q.float().reshape(n, hk, hq // hk, d), k.transpose(2, 3)) / math.sqrt(d)
    s = torch.where(seen[:, None, None], s, -math.inf)
    top = s.amax(-1, keepdim=True)
    p = torch.exp(s - torch.where(top == -math.inf, 0.0, top))
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p, torch.where(seen[:, None, :, None], v, 0.0))
    st["out"].copy_(torch.where(total > 0, o / total, 0.0).reshape(n, hq, d))


# ---- bytes and operations that a pass cannot do without ---------------------------------------------------------------------------


def work(case):
    page, n = case["page"], case["n_req"]
    hq, hk, d, t = SHAPES[case["shape"]]
    e = 4 if t == "f32" else 2
    if case["kind"] == "append":
        cached, new = _sizes(case)
        tokens = int(new.sum())
        rows = tokens + case["pad"]
        q_heads = rows * hq if case["queries"] else 0
        blocks = int((_pages(cached + new, BLOCK) - cached // BLOCK).sum())
        kept = int((cached % BLOCK > 0).sum())  # scales that are read
        per = 3.0 * case["rot"] + (4.0 * d if case["norm"] else 0.0)
        return {"bytes": 2 * e * d * q_heads + 2 * (e + 1) * d * tokens * hk + 2 * hk * (blocks + kept) + 8 * rows,
                "flops": per * (q_heads + tokens * hk) + 3.0 * d * 2 * hk * tokens}
    lens = _sizes(case)
    if case["kind"] == "read":
        total = int(lens.sum())
        return {"bytes": 2 * hk * ((1 + e) * d * total + int(_pages(lens, BLOCK).sum())) + 4 * int(_pages(lens, page).sum()) + 8 * n + 4,
                "flops": 2.0 * hk * d * total}
    seen = int(_visible(case, lens).sum())
    return {"bytes": 2 * hk * d * seen + 2 * hk * _pages(seen, BLOCK) + 2 * e * n * hq * d + 4 * _pages(seen, page) + 4 * n,
            "flops": 4.0 * hq * d * seen + 2.0 * hk * d * seen}


# ---- the operators' definitions, in 64 bits -----------------------------------------------------------------------------------------


def exact(case, seed):
    st = prepare(case, seed)
    return {"append": _append_exact, "read": _read_exact, "decode": _decode_exact}[case["kind"]](st)


def _append_exact(st):
    """Codes as the numbers that they round, in units of the scale.  No value for the scales of keys: next to a border those of 32
    and of 64 bits may be a step apart."""
    case = st["case"]
    r, half, n, page = case["rot"], case["rot"] // 2, st["tokens"], case["page"]
    theta = np.array([1e6 ** (-2.0 * m / r) for m in range(half)])
    turn = torch.polar(torch.ones(len(st["pos"]), half, dtype=torch.float64, device="cuda"),
                       st["pos"].double()[:, None] * torch.from_numpy(theta).cuda())

    def heads(x, weight):
        y = x.double().clone()
        if weight is not None:
            y = y / torch.sqrt(y.square().sum(-1, keepdim=True) / y.shape[-1] + EPS) * weight.double()
        re, im = (slice(0, half), slice(half, r)) if case["layout"] == "half" else (slice(0, r, 2), slice(1, r, 2))
        z = torch.complex(y[..., re], y[..., im]) * turn[:len(x), None]
        y[..., re], y[..., im] = z.real, z.imag
        return y

    slots = st["slots"][:n].cpu().numpy()
    starts = np.flatnonzero(np.diff(slots // BLOCK, prepend=-1))  # of the runs of tokens that go to one block
    out = [heads(st["q"], st["q_norm"])] if st["q"] is not None else []
    scales = []
    for x, codes, scale in ((heads(st["k"][:n], st["k_norm"]), st["k_pages"], st["k_scale"]), (st["v"][:n].double(), st["v_pages"], st["v_scale"])):
        codes, scale = codes.double(), scale.double()
        tops = torch.stack([x[a:b].abs().amax((0, 2)) for a, b in zip(starts, [*starts[1:], n])])
        needs = 2.0 ** torch.ceil(torch.log2(tops / 448.0))
        needs = torch.where(tops > 448.0 * needs, 2.0 * needs, torch.where(tops <= 224.0 * needs, 0.5 * needs, needs))  # a rounded logarithm
        for i, a in enumerate(starts):
            b = starts[i + 1] if i + 1 < len(starts) else n
            p, row = divmod(int(slots[a]), page)
            blk, first = divmod(row, BLOCK)
            to = needs[i]
            if first:
                to = torch.maximum(needs[i], scale[p, :, blk])
                codes[p, blk * BLOCK:(blk + 1) * BLOCK] *= (scale[p, :, blk] / to)[:, None]
            codes[p, row:row + b - a] = x[a:b] / to[:, None]
            scale[p, :, blk] = to
        out.append(codes)
        scales.append(scale)
    return out + [None, scales[1]]


def _rows_exact(st, r, rows):
    """Keys and values of some rows of request r."""
    page = st["case"]["page"]
    p, i = st["table"][r].long()[rows // page], rows % page
    return [st[c].view(torch.uint8)[p, i].view(torch.float8_e4m3fn).double() * st[s].double()[p, :, i // BLOCK][..., None]
            for c, s in (("k_pages", "k_scale"), ("v_pages", "v_scale"))]


def _read_exact(st):
    parts = [_rows_exact(st, r, torch.arange(int(length), device="cuda")) for r, length in enumerate(_sizes(st["case"]))]
    return [torch.cat([p[side] for p in parts]) for side in (0, 1)]


def _decode_exact(st):
    case = st["case"]
    n, hq, d = st["q"].shape
    hk = st["k_pages"].shape[2]
    out = torch.zeros(n, hq, d, dtype=torch.float64, device="cuda")
    for r, length in enumerate(_sizes(case).tolist()):
        keys = [j for j in range(length) if not case["window"] or j < case["sinks"] or j >= length - case["window"]]
        if not keys:
            continue
        k, v = _rows_exact(st, r, torch.tensor(keys, device="cuda"))
        for h in range(hk):
            heads = slice(h * (hq // hk), (h + 1) * (hq // hk))
            s = (k[:, h] @ st["q"][r, heads].double().T) * d ** -0.5  # [keys, heads]
            w = torch.exp(s - s.max(0).values)
            out[r, heads] = (w / w.sum(0)).T @ v[:, h]
    return out
