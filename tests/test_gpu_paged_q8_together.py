"""The calls over a paged cache in 8 bits together: a server's steps, captured ones, the question's prefill behind documents that are read back,
pools of more than 4 GiB, work on two streams."""
import numpy as np
import pytest
import torch

from tests import helpers as H
from tests import paged_q8_reference as Q
from tests import paged_reference as R
from tests.test_gpu_paged import DT, ints, randn, tables

pytestmark = pytest.mark.gpu
EPS = 1e-6


@pytest.fixture(scope="module")
def B():
    from paper_2410_07590_amd import binding
    binding.lib()
    return binding


class Server:
    """Three requests whose caches grow in pages, prompts and then one token at a time; a step maps, appends, decodes and reads everything
    back, in buffers that a captured graph can keep."""

    def __init__(self, B, dt="bf16", page=32, room=48, seed=0):
        self.B, self.dt, self.dtype, self.page, self.room = B, dt, DT[dt], page, room
        self.hq, self.hk, self.d, self.rot = 6, 2, 128 if dt == "bf16" else 64, 32
        self.gs = B.make_shape(self.hq, self.hk, self.d, dt, 1e4, 1)
        self.rotary, self.freq = B.tr_rotary_init(1, self.rot, 1e4), R.frequencies(self.rot, 1e4)
        self.order = np.random.default_rng(seed).permutation(32)
        self.k = [x.cuda() for x in Q.random_pool(32, page, self.hk, self.d, seed + 1)]   # pages that were in use before: codes and scales
        self.v = [x.cuda() for x in Q.random_pool(32, page, self.hk, self.d, seed + 2)]
        self.pages = B.make_pages_q8(self.k[0], self.v[0], self.k[1], self.v[1])
        i32 = lambda *s: torch.zeros(*s, dtype=torch.int32, device="cuda")   # noqa: E731
        self.cached, self.new, self.lens, self.free, self.starts = i32(3), i32(3), i32(3), i32(32), i32(4)
        self.table = torch.full((3, 12), -1, dtype=torch.int32, device="cuda")
        self.cu, self.counts, self.slots, self.pos, self.last = i32(4), i32(2), i32(room), i32(room), i32(3)
        blank = lambda n, h: torch.zeros(n, h, self.d, dtype=self.dtype, device="cuda")   # noqa: E731
        self.xq, self.xk, self.xv, self.q_out, self.out = blank(room, self.hq), blank(room, self.hk), blank(room, self.hk), blank(room, self.hq), blank(3, self.hq)
        self.rows = [blank(400, self.hk), blank(400, self.hk)]
        self.qw, self.kw = (randn(self.d, seed=50 + i, dtype=self.dtype).cuda() for i in (0, 1))
        self.ws = B.workspace(B.tr_paged_decode_attn_q8_workspace_size(self.gs, 3, 12, page))
        self.used, self.held = 0, [0, 0, 0]

    def load(self, new, seed):
        total = sum(new)
        self.x = [randn(total, h, self.d, seed=seed + i, dtype=self.dtype, scale=1.0 + seed % 7) for i, h in enumerate((self.hq, self.hk, self.hk))]
        self.cached.copy_(ints(self.held))
        self.new.copy_(ints(new))
        self.free.copy_(ints(np.concatenate([self.order[self.used:], np.zeros(self.used)])))
        for dst, src in zip((self.xq, self.xk, self.xv), self.x):
            dst[:total].copy_(src)
        self.last.copy_(ints(np.maximum(np.cumsum(new) - 1, 0)))
        self.starts.copy_(ints(np.concatenate([[0], np.cumsum(np.array(self.held) + new)])))
        self.step_new, self.before = new, [[t.cpu() for t in side] for side in (self.k, self.v)]

    def step(self):
        B = self.B
        B.tr_page_map(self.cached, self.new, None, self.page, self.free, self.table, self.lens, self.cu, self.slots, self.pos, self.counts)
        B.tr_paged_append_q8(self.gs, self.rotary, self.xq, self.xk, self.xv, self.qw, self.kw, EPS, self.pos, self.slots, self.q_out, self.pages)
        B.tr_paged_decode_attn_q8(self.gs, self.q_out[self.last.long()], self.pages, self.table, self.lens, 50, 3, self.out, self.ws)
        B.tr_paged_read_q8(self.gs, self.pages, self.table, self.lens, self.starts, *self.rows)

    def check(self):
        torch.cuda.synchronize()
        _, k, v = self.x
        n = sum(self.step_new)
        slots = self.slots.cpu().numpy().astype(np.int64)
        assert (slots[:n] >= 0).all() and (slots[n:] == -1).all()
        pos = torch.cat([torch.arange(h, h + m) for h, m in zip(self.held, self.step_new)])
        keys, size = R.heads(k, self.kw.cpu(), EPS, pos, self.freq, 1)
        if n:
            Q.check_append(self.k[0].cpu(), self.k[1].cpu(), *self.before[0], keys, 26 * 2.0 ** -24 * size + 1e-37, slots[:n], "keys")
            Q.check_append(self.v[0].cpu(), self.v[1].cpu(), *self.before[1], v.double(), 0, slots[:n], "values")
        self.held = [h + m for h, m in zip(self.held, self.step_new)]
        self.used += int(self.counts[1])
        table, at = self.table.cpu(), 0
        worth = [Q.values(*(t.cpu() for t in side)) for side in (self.k, self.v)]
        for r, held in enumerate(self.held):
            j = torch.arange(held)
            page = table[r].long()[j // self.page]
            kc, vc = (w[page, j % self.page] for w in worth)
            assert torch.equal(self.rows[0][at:at + held].cpu().double(), kc) and torch.equal(self.rows[1][at:at + held].cpu().double(), vc)
            at += held
            seen = R.visible(held, 50, 3)
            want, bound = R.decode(self.q_out[int(self.last[r])].cpu(), kc[seen], vc[seen], seen, self.hq // self.hk)
            R.assert_within(self.out[r], want, torch.finfo(self.dtype).eps / 2 * want.abs() * 1.01 + bound, "request %d" % r)


STEPS = [[17, 0, 3], [1, 0, 1], [1, 30, 1], [16, 1, 0], [1, 1, 1], [12, 12, 12], [1, 1, 1], [1, 1, 1], [0, 0, 20]]


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("page", [16, 32])
def test_a_server_steps(B, dt, page):
    s = Server(B, dt, page)
    for i, new in enumerate(STEPS):
        s.load(new, 101 * i)
        s.step()
        s.check()


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_a_captured_step_serves_other_lengths(B, dt):
    s = Server(B, dt)
    s.load([5, 2, 0], 1)
    s.step()
    s.check()
    s.load([1, 1, 1], 2)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        s.step()
    for i, new in enumerate(STEPS):
        s.load(new, 1000 + 101 * i)
        graph.replay()
        s.check()
        before = [s.out.clone(), *(t.clone() for t in s.rows)]
        s.out.zero_()
        s.B.tr_paged_decode_attn_q8(s.gs, s.q_out[s.last.long()], s.pages, s.table, s.lens, 50, 3, s.out, s.ws)   # the same, not replayed
        s.B.tr_paged_read_q8(s.gs, s.pages, s.table, s.lens, s.starts, *s.rows)
        assert torch.equal(before[0], s.out) and all(torch.equal(a, b) for a, b in zip(before[1:], s.rows))


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_a_question_behind_documents_that_are_read_back(B, dt):
    """Chunks turned by their offsets into pages of 8 bits, the question's keys behind them, all read back for tr_prefill_attn; its last row is
    what decode says of the last token over the pages."""
    hq, hk, d, page, dtype = 8, 2, 128, 16, DT[dt]
    gs = B.make_shape(hq, hk, d, dt, 1e6, 1)
    lens, n_q = [70, 33, 100], 9
    n_doc, total = sum(lens), sum(lens) + n_q
    k, v = (randn(n_doc, hk, d, seed=s, dtype=dtype).cuda() for s in (1, 2))   # keys at chunk-local positions
    q, kq, vq = (randn(n_q, h, d, seed=9 + h, dtype=dtype).cuda() for h in (hq, hk, hk))
    n_blocks = -(-total // page)
    table = torch.randperm(n_blocks, generator=torch.Generator().manual_seed(3)).to(torch.int32).cuda().view(1, -1)
    slots = (table[0].repeat_interleave(page) * page + torch.arange(page, device="cuda", dtype=torch.int32).repeat(n_blocks))[:total].contiguous()
    codes = [torch.zeros(n_blocks, page, hk, d, dtype=torch.float8_e4m3fn, device="cuda") for _ in range(2)]
    scales = [torch.zeros(n_blocks, hk, 1, dtype=torch.uint8, device="cuda") for _ in range(2)]
    pages = B.make_pages_q8(*codes, *scales)
    at = 0
    for length in lens:   # a chunk's rows end within blocks, which the next one continues
        turn = torch.full((length,), at, dtype=torch.int32, device="cuda")
        B.tr_paged_append_q8(gs, None, None, k[at:at + length], v[at:at + length], None, None, EPS, turn, slots[at:at + length], None, pages)
        at += length
    pos, q_out = ints(np.arange(n_doc, total)), torch.empty_like(q)
    B.tr_paged_append_q8(gs, None, q, kq, vq, None, None, EPS, pos, slots[n_doc:], q_out, pages)
    ck, cv = (torch.empty(total, hk, d, dtype=dtype, device="cuda") for _ in range(2))
    B.tr_paged_read_q8(gs, pages, table, ints([total]), ints([0, total]), ck, cv)
    out, one = torch.empty_like(q), torch.empty(1, hq, d, dtype=dtype, device="cuda")
    B.tr_prefill_attn(gs, q, ck, cv, pos, total, out, B.workspace(B.tr_prefill_attn_workspace_size(gs, n_q, total)))
    B.tr_paged_decode_attn_q8(gs, q_out[-1:].contiguous(), pages, table, ints([total]), 0, 0, one,
                              B.workspace(B.tr_paged_decode_attn_q8_workspace_size(gs, 1, n_blocks, page)))
    torch.cuda.synchronize()
    rows = torch.arange(total)
    p = table[0].cpu().long()[rows // page]
    worth = [Q.values(c.cpu().view(torch.uint8), s.cpu())[p, rows % page] for c, s in zip(codes, scales)]
    assert torch.equal(ck.cpu().double(), worth[0]) and torch.equal(cv.cpu().double(), worth[1])
    # both attentions are within the tolerance of fp64 over the same rows; decode's query was rounded to the type once more
    assert (out[-1:].double() - one.double()).abs().max() <= 2 * (H.BF16_TOL if dt == "bf16" else 1e-4)
    # what 8 bits cost: a key or value is off by at most half a step, 2^-4 of it or 2^-10 of the block's scale
    want, _ = R.heads(torch.cat([k, kq]).cpu(), None, EPS, torch.cat([torch.full((n,), sum(lens[:i])) for i, n in enumerate(lens)] + [pos.cpu()]), R.frequencies(d, 1e6), 1)
    step = torch.ldexp(torch.ones((), dtype=torch.float64), scales[0].cpu().int() - 127)[p, :, 0][..., None]
    assert bool(((worth[0] - want).abs() <= 2.0 ** -4 * want.abs() * (1 + 2.0 ** -8) + 2.0 ** -9 * step).all())


@pytest.mark.parametrize("order", ["rows", "heads"])
def test_offsets_beyond_32_bits(B, order):
    """A pool of more than 4 GiB each for K and V, the pages in use at its end."""
    page, hk, d = 64, 8, 128
    n_pages = (5 << 30) // (page * hk * d)
    if order == "rows":
        kp, vp = (torch.empty(n_pages, page, hk, d, dtype=torch.uint8, device="cuda") for _ in range(2))
    else:
        kp, vp = (torch.empty(n_pages, hk, page, d, dtype=torch.uint8, device="cuda").transpose(1, 2) for _ in range(2))
    ks, vs = (torch.full((n_pages, hk, page // 16), 255, dtype=torch.uint8, device="cuda") for _ in range(2))
    lens, used = [190, 64], [n_pages - 1, 3, n_pages - 2, n_pages - 3]
    table = np.array([[used[0], used[1], used[2]], [used[3], -1, -1]])
    k, v = (randn(254, hk, d, seed=s, dtype=torch.bfloat16) for s in (1, 2))
    gs, pages = B.make_shape(16, hk, d, "bf16", 1e4), B.make_pages_q8(kp, vp, ks, vs)
    slots = [table[r, j // page] * page + j % page for r in (0, 1) for j in range(lens[r])]
    B.tr_paged_append_q8(gs, B.tr_rotary_init(0, 0, 1e4), None, k.cuda(), v.cuda(), None, None, EPS, None, ints(slots), None, pages)
    q = randn(2, 16, d, seed=2, dtype=torch.bfloat16)
    out, rows = torch.empty_like(q).cuda(), [torch.empty(254, hk, d, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    B.tr_paged_decode_attn_q8(gs, q.cuda(), pages, ints(table), ints(lens), 0, 0, out, B.workspace(B.tr_paged_decode_attn_q8_workspace_size(gs, 2, 3, page)))
    B.tr_paged_read_q8(gs, pages, ints(table), ints(lens), ints([0, 190, 254]), *rows)
    torch.cuda.synchronize()
    small = []
    for c, s, x, row in ((kp, ks, k, rows[0]), (vp, vs, v, rows[1])):
        codes, scale = torch.zeros(4, page, hk, d, dtype=torch.uint8), torch.full((4, hk, page // 16), 255, dtype=torch.uint8)
        got = torch.stack([c[p].cpu() for p in used]), torch.stack([s[p].cpu() for p in used])
        got[0][2, 62:] = 0   # rows that nobody wrote
        local = [used.index(int(i) // page) * page + int(i) % page for i in slots]
        Q.check_append(*got, codes, scale, x.double(), 0, local, "far pages")
        small.append(Q.values(*got))
        want = small[-1].reshape(-1, hk, d)[torch.tensor(local)]
        assert torch.equal(row.cpu().double(), want)
    want, bound = R.decode_batch(q, small[0], small[1], torch.tensor([[0, 1, 2], [3, -1, -1]]), lens, 0, 0, 2)
    R.assert_within(out, want, 2.0 ** -8 * want.abs() * 1.01 + bound, "far pages")


def test_calls_on_two_streams_at_once(B):
    """Two batches of one pool, each with its workspace: decodes, reads and appends to pages of their own overlap."""
    hq, hk, d, page = 8, 2, 128, 32
    gs, rot = B.make_shape(hq, hk, d, "bf16", 1e4), B.tr_rotary_init(1, 64, 1e4)
    lens = [[3000, 17, 900], [1500, 2500, 1]]
    pool = [x.cuda() for i in (1, 2) for x in Q.random_pool(500, page, hk, d, i)]
    pages = B.make_pages_q8(pool[0], pool[2], pool[1], pool[3])
    jobs, base = [], 0
    for i, ls in enumerate(lens):
        table, n = tables(np.random.default_rng(i), ls, page)
        table = np.where(table >= 0, table + base, -1)
        base += n
        new = np.concatenate([(490 + 3 * i) * page + np.arange(40)])
        jobs.append(dict(table=ints(table), lens=ints(ls), starts=ints(np.concatenate([[0], np.cumsum(ls)])), slots=ints(new), pos=ints(np.arange(40)),
                         q=randn(3, hq, d, seed=i, dtype=torch.bfloat16).cuda(), x=[randn(40, h, d, seed=10 * i + h, dtype=torch.bfloat16).cuda() for h in (hq, hk, hk)],
                         ws=B.workspace(B.tr_paged_decode_attn_q8_workspace_size(gs, 3, table.shape[1], page)), rows=sum(ls)))
    assert base < 490

    def work(j):
        out, q_out = torch.empty_like(j["q"]), torch.empty_like(j["x"][0])
        rows = [torch.empty(j["rows"], hk, d, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        B.tr_paged_append_q8(gs, rot, *j["x"], None, None, EPS, j["pos"], j["slots"], q_out, pages)
        B.tr_paged_decode_attn_q8(gs, j["q"], pages, j["table"], j["lens"], 0, 0, out, j["ws"])
        B.tr_paged_read_q8(gs, pages, j["table"], j["lens"], j["starts"], *rows)
        return [out, q_out, *rows]

    want = [work(j) for j in jobs]
    torch.cuda.synchronize()
    held = [t.clone() for t in pool]
    streams = [torch.cuda.Stream() for _ in jobs]
    torch.cuda.synchronize()
    for _ in range(10):
        got = []
        for s, j in zip(streams, jobs):
            with torch.cuda.stream(s):
                got.append(work(j))
        torch.cuda.synchronize()
        for a, b in zip(want, got):
            assert all(torch.equal(x, y) for x, y in zip(a, b))
        assert all(torch.equal(x, y) for x, y in zip(pool, held))
