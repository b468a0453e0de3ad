"""The answer's operators (cc_extend_segments, cc_append_attention, cc_sample) against the 64-bit oracle, through the binding."""
import math

import numpy as np
import pytest
import torch

from oracle import answer_oracle as A

pytestmark = pytest.mark.gpu
THETA = 5.0e5


def _ctx(dtype="bf16", hq=8, hkv=2, d=128, impl="auto"):
    import paper_2502_15734_amd as P
    ctx = P.Context(hq, hkv, d, THETA, P.CC_BF16 if dtype == "bf16" else P.CC_F32)
    ctx.set_impl({"auto": P.CC_IMPL_AUTO, "scalar": P.CC_IMPL_SCALAR}[impl])
    return ctx


def _i32(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()


def _np(t):
    return t.cpu().numpy()


# ---- cc_extend_segments --------------------------------------------------------------------------------------------------------
class Tables:
    """Random segments with room for growth on pages in random order."""

    def __init__(self, seed, n_req, max_segs, max_old, max_new, spare=0, room=2, grow_all=False, holes=False):
        rng = np.random.default_rng(seed)
        per = rng.integers(0 if n_req > 3 else 1, max_segs + 1, n_req)
        self.off = np.concatenate([[0], np.cumsum(per)])
        n = int(self.off[-1])
        last = np.zeros(n, bool)
        last[self.off[1:][per > 0] - 1] = True
        old = rng.integers(0, max_old + 1, n)
        new = np.where(last | grow_all, rng.integers(-1, max_new + 1, n), 0)
        if grow_all:
            old[:] = 0
        cap = (old + np.maximum(new, 0) + 15) // 16 + rng.integers(0, room + 1, n)
        if n > 4:
            cap[rng.integers(0, n)] = 0                                   # an owner of nothing
        start = np.concatenate([[0], np.cumsum(cap)[:-1]])
        self.segs = np.stack([np.repeat(np.arange(n_req), per), last, rng.integers(0, 9, n), old, start, rng.integers(0, 9, n),
                              rng.integers(0, 9, n), rng.integers(0, 9, n)], 1) if n else np.zeros((0, 8), int)
        held = np.minimum((old + 15) // 16, cap)
        need = int(((old + np.maximum(new, 0) + 15) // 16 - (old + 15) // 16).sum())
        n_held = int(held.sum())
        ids = rng.permutation(n_held + max(0, need + spare) + 3)
        self.tab = np.full(int(cap.sum()) + 1, -7)
        at = 0
        for s in range(n):
            self.tab[start[s]:start[s] + held[s]] = ids[at:at + held[s]]
            at += held[s]
        if holes and n_held:
            self.tab[rng.integers(0, len(self.tab), 3)] = (-1, 1 << 30, -5)
        self.free, self.n_blocks, self.new, self.cap = ids[at:at + max(0, need + spare)], len(ids), new, cap
        self.rows = int(np.maximum(new, 0).sum())


def _extend(ctx, t, max_rows, in_place=False, fill=-9):
    n_req = len(t.off) - 1
    segs_in = _i32(t.segs)
    o = dict(segs=segs_in if in_place else torch.full_like(segs_in, fill), block_tab=_i32(t.tab), cu_q=_i32(np.full(n_req + 1, fill)),
             q_pos=_i32(np.full(max_rows, fill)), slot_map=_i32(np.full(max_rows, fill)), row_req=_i32(np.full(max_rows, fill)),
             last_row=_i32(np.full(n_req, fill)), status=_i32(np.full(n_req, fill)), counts=_i32(np.full(4, fill)))
    ws = torch.full((max(256, ctx.extend_segments_workspace_bytes(len(t.segs), n_req)),), 255, dtype=torch.uint8, device="cuda")
    args = (segs_in, _i32(t.new), _i32(t.cap), _i32(t.off), _i32(t.free), o["block_tab"], t.n_blocks, o["segs"], o["cu_q"], o["q_pos"],
            o["slot_map"], o["row_req"], o["last_row"], o["status"], o["counts"], ws)
    ctx.extend_segments(*args)
    return o, args


def _check_extend(o, t, max_rows):
    want = A.extend_segments(t.segs, t.new, t.cap, t.off, t.free, t.tab, t.n_blocks, max_rows)
    for name, w in zip(("segs", "block_tab", "cu_q", "q_pos", "slot_map", "row_req", "last_row", "status", "counts"), want):
        np.testing.assert_array_equal(_np(o[name]).reshape(w.shape), w, err_msg=name)
    return want


EXTEND = [dict(seed=1, n_req=1, max_segs=1, max_old=0, max_new=1), dict(seed=2, n_req=1, max_segs=5, max_old=40, max_new=33),
          dict(seed=3, n_req=7, max_segs=4, max_old=100, max_new=1), dict(seed=4, n_req=64, max_segs=9, max_old=50, max_new=3),
          dict(seed=5, n_req=65, max_segs=6, max_old=0, max_new=70, grow_all=True), dict(seed=6, n_req=300, max_segs=12, max_old=30, max_new=2),
          dict(seed=7, n_req=1025, max_segs=3, max_old=20, max_new=40), dict(seed=8, n_req=2500, max_segs=2, max_old=17, max_new=5),
          dict(seed=9, n_req=40, max_segs=200, max_old=5, max_new=300), dict(seed=10, n_req=3, max_segs=2, max_old=0, max_new=5000, grow_all=True),
          dict(seed=11, n_req=2, max_segs=1000, max_old=3, max_new=9), dict(seed=12, n_req=1024, max_segs=5, max_old=64, max_new=1),
          dict(seed=13, n_req=2200, max_segs=25, max_old=40, max_new=1)]


@pytest.mark.parametrize("spare,lacking,holes", [(5, 0, False), (0, 3, True), (-4, 0, True), (-40, 9, False)])
@pytest.mark.parametrize("case", EXTEND, ids=lambda c: f"{c['n_req']}x{c['max_segs']}")
def test_extend_segments(case, spare, lacking, holes):
    t = Tables(**case, spare=spare, holes=holes)
    ctx = _ctx()
    max_rows = max(0, t.rows + 3 - 2 * lacking)
    o, _ = _extend(ctx, t, max_rows)
    _check_extend(o, t, max_rows)
    o, _ = _extend(ctx, t, max_rows, in_place=True)
    _check_extend(o, t, max_rows)


@pytest.mark.parametrize("max_rows", [0, 5, 30000])
def test_extend_segments_of_an_empty_batch(max_rows):
    """No request: counts of 0 and rows of nothing, whatever an earlier step left there."""
    t = Tables(1, 1, 1, 0, 1)
    t.segs, t.new, t.cap, t.off, t.tab = np.zeros((0, 8), int), np.zeros(0, int), np.zeros(0, int), np.zeros(1, int), np.arange(4)
    o, _ = _extend(_ctx(), t, max_rows)
    _check_extend(o, t, max_rows)


def test_extend_segments_many_rows():
    """Tables of prompts from nothing whose rows need many workgroups."""
    t = Tables(20, 90, 12, 0, 1500, grow_all=True)
    t.cap = np.maximum(t.cap, (np.maximum(t.new, 0) + 15) // 16)
    t.segs[:, 4] = np.concatenate([[0], np.cumsum(t.cap)[:-1]])
    t.tab = np.full(int(t.cap.sum()), -1)
    o, _ = _extend(_ctx(), t, t.rows)
    want = _check_extend(o, t, t.rows)
    assert want[8][2] == 0 and want[8][0] > 100000


def test_extend_segments_negative_and_huge_lengths():
    t = Tables(30, 4, 3, 20, 5)
    t.segs[:, 3] = np.where(np.arange(len(t.segs)) % 3 == 0, -5, t.segs[:, 3])
    t.new[-1] = 2 ** 31 - 1                                                      # more than any table holds
    t.new[:-1] = np.where(t.new[:-1] < 0, -2 ** 31, t.new[:-1])
    o, _ = _extend(_ctx(), t, 40)
    want = _check_extend(o, t, 40)
    assert want[7][np.nonzero(np.diff(t.off))[0][-1]] == A.TABLE_FULL


def test_extend_segments_in_a_graph():
    """Captured in place, every replay is the next step of the same answers; the eager call beside it says what it should be."""
    ctx = _ctx()
    t = Tables(40, 9, 4, 30, 1, room=9, spare=60)
    t.new = np.maximum(t.new, 0)
    t.cap = t.cap + 9
    t.segs[:, 4] = np.concatenate([[0], np.cumsum(t.cap)[:-1]])
    t.tab = np.concatenate([np.arange(1000, 1000 + int(t.cap.sum()))])
    t.n_blocks = 5000
    o, args = _extend(ctx, t, 12, in_place=True)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ctx.extend_segments(*args)
    args[0].copy_(_i32(t.segs)); args[5].copy_(_i32(t.tab))
    for _ in range(4):
        for name in ("q_pos", "slot_map", "row_req", "cu_q", "counts", "status", "last_row"):
            o[name].fill_(-9)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        want = _check_extend(o, t, 12)
        t.segs, t.tab = want[0].astype(np.int64), want[1].astype(np.int64)


# ---- cc_append_attention -------------------------------------------------------------------------------------------------------
class Batch:
    """Requests given as (lengths of their cached segments, tokens of the last segment, new ones among them)."""

    def __init__(self, seed, requests, hq, hkv, d, dtype, bad_pages=(), scale=1.0, spread=False):
        rng = np.random.default_rng(seed)
        self.dtype, self.hq, self.hkv, self.d = dtype, hq, hkv, d
        segs, off, cu, self.pos, tok, tab = [], [0], [0], [], [], 0
        for r, (chunks, tail, new) in enumerate(requests):
            start = 0
            for i, n in enumerate(list(chunks) + [tail]):
                segs.append([r, i == len(chunks), start, n, tab, new if i == len(chunks) else 0, 0, cu[-1]])
                start, tab = start + n, tab + (n + 15) // 16
            first = tail - new
            self.pos += list(range(start - new, start))
            tok += [(segs[-1][4], t) for t in range(first, tail)]
            off.append(len(segs)); cu.append(cu[-1] + new)
        self.segs, self.off, self.cu = np.array(segs), np.array(off), np.array(cu)
        self.n_blocks = tab + 4
        self.tab = rng.permutation(self.n_blocks)[:max(1, tab)]
        self.slot = np.array([self.tab[a + t // 16] * 16 + t % 16 for a, t in tok], dtype=np.int64)
        for i, p in bad_pages:                                             # (entry, page that does not exist); rows keep their slots
            self.tab[i] = p
        t = torch.bfloat16 if dtype == "bf16" else torch.float32
        g = torch.Generator().manual_seed(seed)
        mk = lambda *s: (torch.randn(*s, generator=g) * scale).to(t)
        n = len(self.pos)
        self.q, self.k_new, self.v_new = mk(n, hq, d), mk(n, hkv, d), mk(n, hkv, d)
        self.k_pool, self.v_pool = mk(self.n_blocks, hkv, 16, d), mk(self.n_blocks, hkv, d, 16)
        # what nobody may read: padding slots and pages of nobody
        used = torch.zeros(self.n_blocks, 16, dtype=torch.bool)
        for s in self.segs:
            for i in range(s[3]):
                if 0 <= self.tab[s[4] + i // 16] < self.n_blocks:
                    used[self.tab[s[4] + i // 16], i % 16] = True
        self.k_pool.permute(0, 2, 1, 3)[~used] = float("nan")
        self.v_pool.permute(0, 3, 1, 2)[~used] = float("nan")
        self.max_ctx = max(int(self.segs[self.off[r]:self.off[r + 1], 3].sum()) for r in range(len(requests)))
        self.max_segs = int(np.diff(self.off).max())
        self.n_req, self.most = len(requests), max(1, int(np.diff(self.cu).max()))

    def up(self, behind=0):
        """Device tensors; `behind` rows behind the last request's."""
        n = len(self.pos) + behind
        pad = lambda a, w: np.concatenate([np.asarray(a), np.full(behind, w)])
        more = lambda x: torch.cat([x, torch.zeros(behind, *x.shape[1:], dtype=x.dtype)]).cuda()
        t = dict(q=more(self.q), k_new=more(self.k_new), v_new=more(self.v_new), q_pos=_i32(pad(self.pos, 0)), slot_map=_i32(pad(self.slot, -1)),
                 cu_q=_i32(self.cu), k_pool=self.k_pool.cuda(), v_pool=self.v_pool.cuda(), block_tab=_i32(self.tab), segs=_i32(self.segs),
                 req_seg_off=_i32(self.off))
        t["out"] = torch.full((n, self.hq, self.d), float("nan"), dtype=self.q.dtype, device="cuda")
        t["lse"] = torch.full((n, self.hq), float("nan"), device="cuda")
        return t

    def workspace(self, ctx, n_rows=None):
        need = ctx.append_attention_workspace_bytes(len(self.pos) if n_rows is None else n_rows, self.most, self.n_req, self.max_ctx, self.max_segs)
        return torch.full((max(256, need),), 255, dtype=torch.uint8, device="cuda")

    def call(self, ctx, t, ws=None, lse=True, **more):
        ws = self.workspace(ctx, t["q_pos"].shape[0]) if ws is None else ws
        ctx.append_attention(t["q"], t["k_new"], t["v_new"], t["q_pos"], t["slot_map"], t["cu_q"], self.most, t["k_pool"], t["v_pool"], t["block_tab"],
                             t["segs"], t["req_seg_off"], self.n_req, self.max_ctx, self.max_segs, t["out"], t["lse"] if lse else None, ws, **more)

    def check(self, t, v_of=None, hidden=()):
        """Written keys and values, outputs and log-sum-exps against the oracle, which reads the pages as the call left them.  hidden: rows that
        take part in no comparison."""
        half = 2.0 ** -8 if self.dtype == "bf16" else 2.0 ** -24
        k, v = t["k_pool"].float().cpu().numpy(), t["v_pool"].float().cpu().numpy()
        if len(self.pos):
            want = A.rotate(self.k_new.double().numpy(), self.pos, THETA)
            got = k[self.slot // 16, :, self.slot % 16]
            fine = np.isfinite(want)                                      # (the turned pair of a value that is not finite is neither)
            near = np.abs(want[fine]).max() * 2
            assert (np.abs(got[fine] - want[fine]) <= half * np.abs(want[fine]) + (2e-6 if self.dtype == "bf16" else 2e-7) * near).all()
            assert np.array_equal(v[self.slot // 16, :, :, self.slot % 16], self.v_new.float().numpy(), equal_nan=True)
        out, lse = t["out"].double().cpu().numpy(), t["lse"].double().cpu().numpy()
        for r in range(self.n_req):
            a, b = int(self.cu[r]), int(self.cu[r + 1])
            ctx_r = A.paged_context(k, v, (lambda p: v[p]) if v_of is None else v_of, self.tab, self.segs, range(self.off[r], self.off[r + 1]))
            show = [i for i in range(a, b) if i not in hidden]
            if len(show) == 0:
                continue
            o, l, ob, lb = A.attend(self.q[show].double().numpy(), np.array(self.pos)[show], *ctx_r, THETA, half)
            off = np.abs(out[show] - o)
            assert (off <= ob).all(), f"request {r}: {np.nanmax(off / np.maximum(ob, 1e-300)):.3g} of the bound, or not a number"
            gone = np.isneginf(l)
            assert np.array_equal(np.isneginf(lse[show]), gone)
            assert (np.abs(lse[show][~gone] - l[~gone]) <= lb[~gone]).all(), f"request {r}: log-sum-exp"


HEADS = [(8, 2, 128, "bf16"), (4, 4, 128, "bf16"), (16, 1, 64, "bf16"), (6, 2, 64, "bf16"), (40, 2, 128, "bf16"), (10, 2, 128, "bf16"), (8, 2, 128, "f32"), (6, 2, 64, "f32"),
         (5, 1, 64, "f32"), (34, 2, 128, "f32")]
SHAPES = {
    "first token": [((), 1, 1)],
    "one each": [((16, 33), 5, 1), ((), 17, 1), ((100, 64, 31), 16, 1), ((500,), 1, 1)],
    "no rows": [((40,), 3, 0), ((7,), 3, 3), ((), 0, 0), ((90,), 9, 1)],
    "empty segments": [((0, 17, 0, 0, 15), 2, 2), ((0, 0), 1, 1)],
    "draft": [((61, 200), 20, 5), ((16,), 8, 8), ((300,), 31, 7)],
    "question": [((250, 333), 77, 70), ((31,), 130, 129)],
    "all at once": [((), 200, 200), ((), 33, 33)],
}


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("heads", HEADS, ids=lambda h: f"{h[0]}on{h[1]}x{h[2]}{h[3]}")
def test_append_attention(heads, shape):
    hq, hkv, d, dtype = heads
    b = Batch(sum(map(ord, shape)), SHAPES[shape], hq, hkv, d, dtype)
    ctx = _ctx(dtype, hq, hkv, d)
    t = b.up()
    b.call(ctx, t)
    torch.cuda.synchronize()
    b.check(t)


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
def test_append_attention_plain_kernel(dtype, d):
    b = Batch(3, SHAPES["draft"] + SHAPES["no rows"], 6, 2, d, dtype)
    t = b.up()
    b.call(_ctx(dtype, 6, 2, d, "scalar"), t)
    torch.cuda.synchronize()
    b.check(t)


@pytest.mark.parametrize("dtype,lengths,new", [("bf16", (700,) * 12, 1), ("bf16", (1000,) * 40, 3), ("bf16", (15,) * 300, 2), ("f32", (999,) * 9, 1),
                                               ("bf16", (300,) * 30, 90)])
def test_append_attention_over_long_contexts(dtype, lengths, new):
    """Keys divided over many workgroups, beside a request with next to nothing."""
    b = Batch(5, [(lengths, new + 9, new), ((), 1, 1), ((40,), 2, 1)], 8, 2, 128, dtype)
    t = b.up()
    b.call(_ctx(dtype), t)
    torch.cuda.synchronize()
    b.check(t)


@pytest.mark.parametrize("hq,d,new", [(8, 128, 1), (8, 64, 4), (8, 128, 5), (12, 128, 10), (8, 64, 16)])
def test_append_attention_few_columns_lose_nothing_inside(hq, d, new):
    """Up to 64 rows and heads on a KV head, bf16: queries and weights are sums of two bf16, off by 2^-15 (2^-7 of the value is left to the second, which is
    off by 2^-8 of that), not by 2^-8.  The angles' functions are off by 2e-6, so a logit by at most 4 e-6 max|q| sum|k| / sqrt d more.  Only the output's own
    rounding is one of bf16."""
    b = Batch(12, [((700, 33), 20, new), ((), 60, new), ((250,), 17, new)], hq, 2, d, "bf16")
    t = b.up()
    b.call(_ctx("bf16", hq, 2, d), t)
    torch.cuda.synchronize()
    k, v, out = t["k_pool"].float().cpu().numpy(), t["v_pool"].float().cpu().numpy(), t["out"].double().cpu().numpy()
    for r in range(b.n_req):
        rows = range(b.cu[r], b.cu[r + 1])
        context = A.paged_context(k, v, lambda p: v[p], b.tab, b.segs, range(b.off[r], b.off[r + 1]))
        q = b.q[rows].double().numpy()
        o, _, bound, _ = A.attend(q, np.array(b.pos)[rows], *context, THETA, 2.0 ** -15)
        turn = 4e-6 * np.abs(q).max() * np.abs(context[1]).sum(-1).max() / math.sqrt(d)
        bound += 2.0 ** -8 * np.abs(o) + math.expm1(2 * turn) * np.abs(context[2]).max()
        assert (np.abs(out[rows] - o) <= bound).all(), f"request {r}: {(np.abs(out[rows] - o) / bound).max():.3g} of the bound"


@pytest.mark.parametrize("scale", [1.0, 3.0])
@pytest.mark.parametrize("hq,d,new", [(8, 128, 17), (8, 64, 40), (12, 128, 45), (2, 128, 140), (16, 64, 33)])
def test_append_attention_many_columns_lose_nothing_inside(hq, d, new, scale):
    """As above for more than 64 rows and heads on a KV head; scale: with larger logits the reference of a row moves, and weights with it."""
    b = Batch(20, [((700, 33), new + 5, new), ((), new + 40, new), ((250,), new, new)], hq, 2, d, "bf16", scale=scale)
    t = b.up()
    b.call(_ctx("bf16", hq, 2, d), t)
    torch.cuda.synchronize()
    k, v, out = t["k_pool"].float().cpu().numpy(), t["v_pool"].float().cpu().numpy(), t["out"].double().cpu().numpy()
    for r in range(b.n_req):
        rows = range(b.cu[r], b.cu[r + 1])
        context = A.paged_context(k, v, lambda p: v[p], b.tab, b.segs, range(b.off[r], b.off[r + 1]))
        q = b.q[rows].double().numpy()
        o, _, bound, _ = A.attend(q, np.array(b.pos)[rows], *context, THETA, 2.0 ** -15)
        turn = 4e-6 * np.abs(q).max() * np.abs(context[1]).sum(-1).max() / math.sqrt(d)
        bound += 2.0 ** -8 * np.abs(o) + math.expm1(2 * turn) * np.abs(context[2]).max()
        assert (np.abs(out[rows] - o) <= bound).all(), f"request {r}: {(np.abs(out[rows] - o) / bound).max():.3g} of the bound"


@pytest.mark.parametrize("dtype,d,new", [("bf16", 128, 1), ("bf16", 64, 4), ("bf16", 128, 5), ("bf16", 64, 16), ("bf16", 128, 40), ("f32", 128, 3)])
def test_append_attention_infinite_values_that_every_row_sees(dtype, d, new):
    """An infinite value has a weight above 0 in every row: that dimension is infinite, the others are what they are without it.  One request has a
    cached key with nine times the others' logits, above or below them."""
    b = Batch(13, [((300,), 70, new), ((40,), 20 + new, new)], 8, 2, d, dtype)
    b.k_pool[b.tab[b.segs[2][4]]][:, 5] *= 9
    for s in (0, 2):
        page = b.tab[b.segs[s][4] + 1]
        b.v_pool[page, 0, 3, 4], b.v_pool[page, 0, 5, 9] = math.inf, -math.inf
    t = b.up()
    b.call(_ctx(dtype, 8, 2, d), t)
    torch.cuda.synchronize()
    out = t["out"].clone()
    assert (out[:, :4, 3] == math.inf).all() and (out[:, :4, 5] == -math.inf).all()
    finite = torch.isfinite(out)
    finite[:, :4, [3, 5]] = True
    assert finite.all()
    plain = t["v_pool"].clone()
    plain[torch.isinf(plain)] = 0.0
    k, v, half = t["k_pool"].float().cpu().numpy(), plain.float().cpu().numpy(), 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
    for r in range(2):
        rows = range(b.cu[r], b.cu[r + 1])
        o, _, bound, _ = A.attend(b.q[rows].double().numpy(), np.array(b.pos)[rows], *A.paged_context(k, v, lambda p: v[p], b.tab, b.segs, range(b.off[r], b.off[r + 1])),
                                  THETA, half)
        off = np.abs(out[rows].double().cpu().numpy() - o)
        off[:, :4, [3, 5]] = 0
        assert (off <= bound).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_append_attention_large_logits(dtype):
    """Logits of some hundred: the weights are those of one or two keys, and the running maximum moves."""
    b = Batch(6, [((300, 70), 30, 4), ((900,), 3, 1)], 8, 2, 128, dtype, scale=5.0)
    t = b.up()
    b.call(_ctx(dtype), t)
    torch.cuda.synchronize()
    b.check(t)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("impl", ["auto", "scalar"])
def test_append_attention_without_keys(dtype, impl):
    """Pages that do not exist hold no keys: a row of nothing else gets zeros and -inf, others what the rest gives."""
    b = Batch(7, [((), 3, 3), ((20, 40), 5, 2), ((64,), 16, 16)], 8, 2, 64, dtype, bad_pages=[(0, -1), (2, 1 << 30), (4, -7)])
    t = b.up()
    b.call(_ctx(dtype, 8, 2, 64, impl), t)
    torch.cuda.synchronize()
    assert (t["out"][:3] == 0).all() and torch.isneginf(t["lse"][:3]).all()
    b.check(t)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("value", [float("inf"), float("nan")])
def test_append_attention_values_a_row_does_not_see(dtype, value):
    """The last new token's key and value are not finite: rows in front of it do not see them; another request's neither."""
    b = Batch(8, [((30,), 40, 6), ((45,), 9, 1), ((), 21, 21)], 8, 2, 128, dtype)
    ends = [5, 27]
    for e in ends:
        b.v_new[e] = value
        b.k_new[e, :, 3] = value
    t = b.up()
    b.call(_ctx(dtype), t)
    torch.cuda.synchronize()
    b.check(t, hidden=ends)
    assert torch.isnan(t["out"][ends].float()).any(-1).all()


@pytest.mark.parametrize("dtype,d,new", [("bf16", 128, 3), ("bf16", 64, 4), ("bf16", 128, 6), ("bf16", 64, 16), ("bf16", 128, 16), ("bf16", 128, 21), ("bf16", 64, 30),
                                         ("f32", 128, 6), ("f32", 64, 21)])
def test_append_attention_largest_values_a_row_does_not_see(dtype, d, new):
    """The last new token's values are the type's largest, of either sign: nothing of them is in the rows in front of it (up to 16, up to 64 and more rows
    times heads of a group)."""
    b = Batch(14, [((30,), new + 34, new), ((), new, new), ((45,), 9, 1)], 8, 2, d, dtype)
    most = torch.finfo(b.v_new.dtype).max
    ends = [new - 1, 2 * new - 1]
    b.v_new[ends[0]], b.v_new[ends[1]] = most, -most
    t = b.up()
    b.call(_ctx(dtype, 8, 2, d), t)
    torch.cuda.synchronize()
    b.check(t, hidden=ends)


@pytest.mark.parametrize("dtype,d,new", [("bf16", 128, 1), ("bf16", 64, 9), ("bf16", 128, 21), ("f32", 128, 2)])
def test_append_attention_queries_of_zeros(dtype, d, new):
    """A pair of the queries is 0 (and -0), the keys' is the type's largest: their product is 0."""
    b = Batch(15, [((130,), 40, new), ((45,), new + 9, new)], 8, 2, d, dtype)
    for i in (5, 5 + d // 2):
        b.q[..., i] = 0.0
        b.q[:, ::2, i] = -0.0
        b.k_pool[..., i] = torch.where(torch.isnan(b.k_pool[..., i]), b.k_pool[..., i], torch.finfo(b.q.dtype).max * (1 if i == 5 else -1))
    t = b.up()
    b.call(_ctx(dtype, 8, 2, d), t)
    torch.cuda.synchronize()
    b.check(t)


def test_append_attention_rows_behind_and_no_lse():
    b = Batch(9, SHAPES["draft"], 8, 2, 128, "bf16")
    ctx = _ctx()
    t = b.up(behind=7)
    b.call(ctx, t, lse=False)
    torch.cuda.synchronize()
    n = len(b.pos)
    assert torch.isnan(t["out"][n:]).all() and torch.isnan(t["lse"]).all()
    first = t["out"][:n].clone()
    t = b.up()
    b.call(ctx, t)
    torch.cuda.synchronize()
    b.check(t)
    assert torch.equal(first, t["out"])                                       # (neither the rows behind nor lse change a bit)


def test_append_attention_source_rows():
    """q, k_new and v_new read through a row list."""
    b = Batch(10, SHAPES["one each"] + SHAPES["draft"], 8, 2, 128, "bf16")
    ctx = _ctx()
    t = b.up()
    b.call(ctx, t)
    n = len(b.pos)
    perm = torch.from_numpy(np.random.default_rng(1).permutation(n + 5)[:n].copy())
    t2 = b.up()
    for name in ("q", "k_new", "v_new"):
        wide = torch.full((n + 5, *t[name].shape[1:]), float("nan"), dtype=t[name].dtype, device="cuda")
        wide[perm.cuda()] = t[name]
        t2[name] = wide
    b.call(ctx, t2, src_rows=perm.int().cuda())
    torch.cuda.synchronize()
    b.check(t2)
    assert torch.equal(t["out"], t2["out"]) and torch.equal(t["lse"], t2["lse"])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_append_attention_values_in_the_store(dtype):
    """Copy-on-write pages: values stay where they are until a row of their page is written."""
    b = Batch(11, [((100, 50), 40, 3), ((64,), 5, 1)], 8, 2, 128, dtype)
    t = b.up()
    store = (torch.randn(b.n_blocks, 2, 128, 16, generator=torch.Generator().manual_seed(2))).to(b.q.dtype).cuda()
    v_map = torch.full((b.n_blocks,), -1, dtype=torch.int32)
    pages = [b.tab[i] for i in range(0, len(b.tab), 2)] + [b.tab[b.segs[2, 4] + 2]]       # the last: a page that gets a row
    rng = np.random.default_rng(3)
    for p in set(int(p) for p in pages):
        v_map[p] = int(rng.integers(0, b.n_blocks))
    before = v_map.clone()
    v_map = v_map.cuda()
    b.call(_ctx(dtype), t, shared=(store, v_map))
    torch.cuda.synchronize()
    written = set(int(s) // 16 for s in b.slot)
    after = v_map.cpu()
    assert all(int(after[p]) == (-1 if p in written else int(before[p])) for p in range(b.n_blocks))
    v, st = t["v_pool"].float().cpu().numpy(), store.float().cpu().numpy()
    for p in written:
        if int(before[p]) >= 0:
            for j in range(16):
                if p * 16 + j not in set(b.slot):
                    assert np.array_equal(v[p][..., j], st[int(before[p])][..., j])
    b.check(t, v_of=lambda p: st[int(after[p])] if int(after[p]) >= 0 else v[p])


@pytest.mark.parametrize("value", [None, float("inf"), float("nan")])
@pytest.mark.parametrize("d,new", [(128, 5), (64, 5), (128, 16), (128, 40), (64, 40)])
def test_append_attention_many_rows_with_values_in_the_store(d, new, value):
    """As above with 17 rows times heads of a group and more (up to 64, and more), bf16.  value: of the last new token, which only its own row sees."""
    b = Batch(17, [((100, 50), 40 + new, new), ((64, 400), 5 + new, new), ((33,), 9, 1)], 8, 2, d, "bf16")
    ends = [new - 1, 2 * new - 1] if value is not None else []
    b.v_new[ends] = 0.0 if value is None else value
    t = b.up()
    store = torch.randn(b.n_blocks, 2, d, 16, generator=torch.Generator().manual_seed(3)).to(b.q.dtype).cuda()
    rng = np.random.default_rng(4)
    v_map = np.full(b.n_blocks, -1)
    pages = set(int(p) for p in b.tab[::2]) | {int(b.slot[0]) // 16, int(b.slot[new]) // 16}            # (the first pages that get rows among them)
    for p in pages:
        v_map[p] = rng.integers(0, b.n_blocks)
    before = v_map.copy()
    dev_map = _i32(v_map)
    b.call(_ctx("bf16", 8, 2, d), t, shared=(store, dev_map))
    torch.cuda.synchronize()
    after, st = _np(dev_map), store.float().cpu().numpy()
    written = set(int(s) // 16 for s in b.slot)
    assert np.array_equal(after, [-1 if p in written else before[p] for p in range(b.n_blocks)])
    b.check(t, v_of=lambda p: st[after[p]] if after[p] >= 0 else t["v_pool"][p].float().cpu().numpy(), hidden=ends)


@pytest.mark.parametrize("dtype,d,new", [("bf16", 64, 1), ("bf16", 128, 8), ("bf16", 64, 32), ("bf16", 128, 20), ("bf16", 64, 40), ("bf16", 128, 64), ("f32", 64, 8), ("f32", 128, 20)])
def test_append_attention_over_more_pages_than_are_listed_at_a_time(dtype, d, new):
    """One range of keys of more than 256 pages per request (64 requests on 8 KV heads are not divided): new rows on both sides of the 256th page, behind it in
    a segment of its own, and behind two short ones; the last one's values are not finite and seen by its own row alone."""
    b = Batch(18, [((), 4096 + (new + 1) // 2, new), ((4096,), new, new), ((1500, 4, 0, 3000, 1), new + 20, new)] + [((), 1 + i % 5, 1) for i in range(61)], 16, 8, d, dtype)
    ctx = _ctx(dtype, 16, 8, d)
    rows = len(b.pos)
    assert ctx.append_attention_workspace_bytes(rows, b.most, b.n_req, b.max_ctx, b.max_segs) < 4 * rows * (16 * (d + 2) + 1) + 256          # (one part per row and head)
    ends = [new - 1, 2 * new - 1, 3 * new - 1] if new > 1 else []
    b.v_new[ends] = float("inf")
    t = b.up()
    b.call(ctx, t)
    torch.cuda.synchronize()
    b.check(t, hidden=ends)


@pytest.mark.parametrize("dtype,d,new", [("bf16", 128, 3), ("bf16", 64, 9), ("bf16", 128, 30), ("f32", 64, 2), ("f32", 128, 25)])
def test_append_attention_rows_that_are_attended_and_not_written(dtype, d, new):
    """Slots outside the pool, on either side: the row sees what its page holds already; the pages stay as they are but for the other rows' slots.  (Rows
    that are written and lie in one page follow each other, as lists have to.)"""
    b = Batch(19, [((61, 200), new + 20, new), ((), new, new), ((16,), 8, 1)], 8, 2, d, dtype)
    t = b.up()
    unwritten = b.slot // 16 % 2 == 0
    unwritten[b.cu[:-1]] = True
    t["slot_map"][torch.from_numpy(unwritten).cuda()] = _i32(np.resize([-1, b.n_blocks * 16, 2 ** 31 - 1, -2 ** 31], unwritten.sum()))
    k0, v0 = t["k_pool"].clone(), t["v_pool"].clone()
    ctx = _ctx(dtype, 8, 2, d)
    assert unwritten.any() and not unwritten.all() and ctx.check_query_list(t["slot_map"], b.n_blocks) == 0
    b.call(ctx, t)
    torch.cuda.synchronize()
    own = torch.zeros(b.n_blocks, 16, dtype=torch.bool, device="cuda")
    own.view(-1)[torch.from_numpy(b.slot[~unwritten]).cuda()] = True
    same = lambda x, y: torch.equal(torch.nan_to_num(x, nan=7.0), torch.nan_to_num(y, nan=7.0))
    assert same(t["k_pool"].transpose(1, 2)[~own], k0.transpose(1, 2)[~own]) and same(t["v_pool"].permute(0, 3, 1, 2)[~own], v0.permute(0, 3, 1, 2)[~own])
    assert torch.equal(t["v_pool"].permute(0, 3, 1, 2).reshape(-1, 2, d)[torch.from_numpy(b.slot[~unwritten]).cuda()].cpu(), b.v_new[torch.from_numpy(~unwritten)])
    k, v, out = t["k_pool"].float().cpu().numpy(), t["v_pool"].float().cpu().numpy(), t["out"].double().cpu().numpy()
    for r in range(b.n_req):
        rows = range(b.cu[r], b.cu[r + 1])
        o, _, bound, _ = A.attend(b.q[rows].double().numpy(), np.array(b.pos)[rows], *A.paged_context(k, v, lambda p: v[p], b.tab, b.segs, range(b.off[r], b.off[r + 1])),
                                  THETA, 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24)
        assert (np.abs(out[rows] - o) <= bound).all()


def test_append_attention_in_graphs_that_share_a_workspace():
    """Two captured calls over one workspace, replayed in turn beside eager work, on a stream of their own."""
    batches = [Batch(12, SHAPES["draft"] + [((3000,), 4, 1)], 8, 2, 128, "bf16"), Batch(13, SHAPES["one each"], 8, 2, 128, "bf16")]
    ctx = _ctx()
    ws = torch.empty(max(b.workspace(ctx).numel() for b in batches), dtype=torch.uint8, device="cuda")
    tensors = [b.up() for b in batches]
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graphs, want = [], []
    with torch.cuda.stream(stream):
        for b, t in zip(batches, tensors):
            b.call(ctx, t, ws=ws)
            stream.synchronize()
            want.append((t["out"].clone(), t["lse"].clone()))
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=stream):
                b.call(ctx, t, ws=ws)
            graphs.append(g)
    torch.cuda.synchronize()
    for _ in range(3):
        for g, t, w in zip(graphs, tensors, want):
            t["out"].fill_(float("nan")); t["lse"].fill_(float("nan")); ws.fill_(255)
            torch.cuda.synchronize()
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(t["out"], w[0]) and torch.equal(t["lse"], w[1])
    for b, t in zip(batches, tensors):
        b.check(t)


# ---- cc_sample -----------------------------------------------------------------------------------------------------------------
def _sample(ctx, z, vocab, u, **settings):
    n = z.shape[0]
    o = dict(token=_i32(np.full(n, -9)), logprob=torch.full((n,), 9.0, device="cuda"), n_kept=_i32(np.full(n, -9)))
    ws = torch.full((max(256, ctx.sample_workspace_bytes(n, vocab)),), 255, dtype=torch.uint8, device="cuda")
    dev = {k: (v if v is None else _i32(v) if k == "top_k" else torch.from_numpy(np.asarray(v, dtype=np.float32)).cuda()) for k, v in settings.items()}
    ctx.sample(z, vocab, torch.from_numpy(np.asarray(u, dtype=np.float32)).cuda(), o["token"], logprob=o["logprob"], n_kept=o["n_kept"], workspace=ws, **dev)
    return o


def _check_sample(o, z, vocab, u, temperature=None, top_k=None, top_p=None, min_p=None):
    """Tokens and counts equal; log-probabilities to a rounding to 32 bits (2^-24 of the value) and 2^-40 for the sums of whole multiples."""
    z, u = z[:, :vocab].double().cpu().numpy(), np.asarray(u, dtype=np.float32)
    token, logprob, kept = _np(o["token"]), _np(o["logprob"]).astype(np.float64), _np(o["n_kept"])
    get = lambda a, r, off: float(np.float32(a[r])) if a is not None else off
    for r in range(len(z)):
        w = A.sample(z[r], get(temperature, r, 1.0), int(top_k[r]) if top_k is not None else 0, get(top_p, r, 1.0), get(min_p, r, 0.0), float(u[r]))
        assert (token[r], kept[r]) == (w[0], w[2]), f"row {r}: {token[r]}, {kept[r]} kept, not {w}"
        assert logprob[r] == w[1] or abs(logprob[r] - w[1]) <= 2.0 ** -24 * abs(w[1]) + 2.0 ** -40, f"row {r}: {logprob[r]} not {w[1]}"


def _logits(seed, rows, vocab, dtype, pad=0):
    g = torch.Generator().manual_seed(seed)
    z = torch.randn(rows, vocab + pad, generator=g) * 2.0
    z[:, torch.randint(0, vocab, (1 + vocab // 50,), generator=g)] += 6
    if pad:
        z[:, vocab:] = 100.0                                              # not part of the vocabulary
    return z.to(torch.bfloat16 if dtype == "bf16" else torch.float32).cuda()


SETTINGS = {"plain": {}, "warm": dict(temperature=(0.3, 1.7)), "greedy": dict(temperature=(0.0, 0.0)), "k": dict(top_k=(1, 60)), "p": dict(top_p=(0.2, 0.999)),
            "min": dict(min_p=(0.001, 0.3)), "k p": dict(top_k=(2, 400), top_p=(0.5, 0.98)),
            "all": dict(temperature=(0.0, 1.5), top_k=(-1, 300), top_p=(0.3, 1.1), min_p=(-0.1, 0.1))}


@pytest.mark.parametrize("settings", SETTINGS)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,vocab,pad", [(1, 1, 0), (5, 2, 3), (7, 63, 0), (3, 64, 1), (33, 1000, 0), (4, 4097, 5), (9, 32000, 0), (3, 50257, 0), (2, 128256, 0), (300, 2049, 7)])
def test_sample(rows, vocab, pad, dtype, settings):
    rng = np.random.default_rng(rows + vocab)
    z = _logits(rows * vocab, rows, vocab, dtype, pad)
    s = {k: (rng.integers(lo, hi + 1, rows) if k == "top_k" else rng.uniform(lo, hi, rows)) for k, (lo, hi) in SETTINGS[settings].items()}
    u = rng.random(rows, dtype=np.float32)
    _check_sample(_sample(_ctx(), z, vocab, u, **s), z, vocab, u, **s)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("vocab,pad", [(1023, 1), (4088, 3), (4089, 0), (8176, 5), (8177, 1), (12280, 7), (12281, 1)])
def test_sample_where_rows_stop_fitting(vocab, pad, dtype):
    """Vocabularies on both sides of what is held at once, rows that begin inside a piece of 16 bytes."""
    rng = np.random.default_rng(vocab)
    z = _logits(vocab, 9, vocab, dtype, pad)
    for s in (dict(top_k=rng.integers(1, 80, 9)), dict(top_p=rng.uniform(0.3, 0.99, 9), temperature=rng.uniform(0.4, 1.4, 9)),
              dict(top_k=rng.integers(2, 900, 9), top_p=rng.uniform(0.3, 0.99, 9), min_p=rng.uniform(0.0, 0.02, 9)), dict(min_p=rng.uniform(0.0, 0.2, 9)), {}):
        u = rng.random(9, dtype=np.float32)
        _check_sample(_sample(_ctx(), z, vocab, u, **s), z, vocab, u, **s)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("vocab", [70, 5000, 40000])
def test_sample_ties(vocab, dtype):
    """Rows of few distinct logits: cuts fall among equals, and the lowest indexes stay."""
    rng = np.random.default_rng(vocab)
    z = torch.from_numpy(rng.integers(-2, 3, (12, vocab)).astype(np.float32) * 0.5)
    z[0] = 1.25
    z[1, ::3] = -0.0                                                          # equal to +0
    z[2] = torch.where(torch.arange(vocab) % 7 == 0, 3.0, -3.4e38)            # the rest masked with the type's lowest value
    z = z.to(torch.bfloat16 if dtype == "bf16" else torch.float32).cuda()
    for s in (dict(top_k=rng.integers(1, vocab, 12)), dict(top_p=rng.uniform(0.1, 0.95, 12)), dict(top_k=rng.integers(1, vocab, 12), top_p=rng.uniform(0.1, 0.95, 12)),
              dict(top_k=np.full(12, vocab + 5)), dict(top_k=np.full(12, 3), min_p=np.full(12, 0.9)), dict(min_p=np.full(12, 1.0)), dict(min_p=np.full(12, 1.5)),
              dict(top_p=np.zeros(12)), dict(top_p=np.full(12, -1.0), top_k=np.full(12, 9))):
        u = rng.random(12, dtype=np.float32)
        _check_sample(_sample(_ctx(), z, vocab, u, **s), z, vocab, u, **s)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("vocab", [900, 20000, 128256])
def test_sample_masked_by_the_lowest_value(vocab, dtype):
    """All but a few tokens at the type's lowest value, and top-k beyond the few: the masked ones count as kept, and are never drawn."""
    kind, rng, rows = torch.bfloat16 if dtype == "bf16" else torch.float32, np.random.default_rng(vocab), 10
    z = torch.full((rows, vocab), torch.finfo(kind).min)
    for r in range(rows):
        at = torch.from_numpy(rng.choice(vocab, 3 + 9 * r, replace=False))
        z[r, at] = torch.from_numpy(rng.standard_normal(len(at)).astype(np.float32)) * 3
    z = z.to(kind).cuda()
    k, full = np.full(rows, 50), np.ones(rows)
    heat = rng.uniform(0.2, 2.0, rows)
    for s in (dict(top_k=k), dict(top_k=k * 3, temperature=heat), dict(top_k=k, top_p=0.9 * full, temperature=heat), dict(top_k=k, min_p=0.01 * full),
              dict(top_k=k, top_p=0.9999999 * full), dict(top_k=k, min_p=1e-30 * full), dict(top_p=0.8 * full), dict(top_k=np.full(rows, vocab - 1), temperature=heat)):
        for u in (rng.random(rows, dtype=np.float32), np.full(rows, 1 - 2.0 ** -24, np.float32)):
            _check_sample(_sample(_ctx(), z, vocab, u, **s), z, vocab, u, **s)


@pytest.mark.parametrize("vocab", [200, 9000])
def test_sample_values_that_are_not_finite(vocab):
    rng = np.random.default_rng(vocab)
    z = torch.from_numpy(rng.standard_normal((8, vocab)).astype(np.float32))
    z[0] = -math.inf
    z[1] = math.nan
    z[2, ::2] = math.nan
    z[3, 1::2] = -math.inf
    z[4, [5, 17, 101]] = math.inf
    z[5, 7] = math.inf
    z[6] = torch.where(torch.arange(vocab) == vocab - 1, 0.5, -math.inf)
    z[7] = -3.0e38
    z = z.cuda()
    for s in (dict(), dict(top_k=np.full(8, 2)), dict(top_p=np.full(8, 0.6)), dict(temperature=np.zeros(8)), dict(min_p=np.full(8, 0.5)),
              dict(top_k=np.full(8, 150), top_p=np.full(8, 0.9), min_p=np.full(8, 0.01), temperature=np.full(8, 0.7))):
        for u in (rng.random(8, dtype=np.float32), np.full(8, 1 - 2.0 ** -24, np.float32), np.full(8, 1.0), np.full(8, np.nan), np.full(8, -0.5)):
            _check_sample(_sample(_ctx(), z, vocab, u, **s), z, vocab, u, **s)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("vocab", [12279, 40001, 128256])
def test_sample_values_that_are_not_finite_in_long_rows(vocab, dtype):
    """As above for the largest vocabulary that is held at once (an odd one) and for rows in parts; whole parts without a logit, too."""
    rng = np.random.default_rng(vocab)
    z = torch.from_numpy(rng.standard_normal((9, vocab)).astype(np.float32))
    z[0] = -math.inf
    z[1] = math.nan
    z[2, ::2] = math.nan
    z[3, 1::2] = -math.inf
    z[4, [5, 17, vocab - 2]] = math.inf
    z[5, 7] = math.inf
    z[6] = torch.where(torch.arange(vocab) == vocab - 1, 0.5, -math.inf)
    z[7, :vocab - 3000] = -math.inf
    z[8, 3000:] = math.nan
    z = z.to(torch.bfloat16 if dtype == "bf16" else torch.float32).cuda()
    full = np.ones(9)
    for s in (dict(), dict(top_k=2 * np.ones(9, int)), dict(top_p=0.6 * full), dict(temperature=0 * full), dict(min_p=0.5 * full),
              dict(top_k=150 * np.ones(9, int), top_p=0.9 * full, min_p=0.01 * full, temperature=0.7 * full)):
        for u in (rng.random(9, dtype=np.float32), np.full(9, 1 - 2.0 ** -24, np.float32), np.full(9, np.nan)):
            _check_sample(_sample(_ctx(), z, vocab, u, **s), z, vocab, u, **s)


@pytest.mark.parametrize("vocab", [333, 13001])
def test_sample_settings_at_their_ends(vocab):
    """Temperatures from the smallest number to infinity and NaN, cuts next to off and to nothing, whole numbers at their limits."""
    nan, inf, least = math.nan, math.inf, 2.0 ** -149
    rows = [(t, k, p, m) for t in (least, 1e-30, 1e-3, 1e4, 1e38, inf, nan) for k, p, m in ((0, 1.0, 0.0), (7, 1.0, 0.0), (0, 0.37, 0.0), (9, 0.61, 0.0), (0, 1.0, 0.53))]
    rows += [(1.0, 2 ** 31 - 1, 1.0, 0.0), (1.0, -2 ** 31, 1.0, 0.0), (1.0, 0, least, 0.0), (1.0, 0, nan, nan), (1.0, 0, inf, -inf), (1.0, 0, 1 - 2.0 ** -24, 0.0),
             (0.9, 0, 1.0, least), (0.9, 0, 1.0, 1.0), (0.9, 0, 1.0, inf), (-inf, 3, 1.0, 0.0), (0.9, vocab, 1.0, 0.0), (0.9, vocab - 1, 1.0, 0.0)]
    s = dict(zip(("temperature", "top_k", "top_p", "min_p"), (np.array(c) for c in zip(*rows))))
    z = _logits(vocab, len(rows), vocab, "f32", 2)
    for seed in range(3):
        u = np.random.default_rng(seed).random(len(rows), dtype=np.float32)
        _check_sample(_sample(_ctx(), z, vocab, u, **s), z, vocab, u, **s)


def test_sample_without_the_optional_outputs_on_a_stream():
    z = _logits(1, 20, 3000, "f32")
    u = np.random.default_rng(1).random(20, dtype=np.float32)
    ctx = _ctx()
    want = _sample(ctx, z, 3000, u)
    token = _i32(np.full(20, -9))
    ws = torch.empty(max(256, ctx.sample_workspace_bytes(20, 3000)), dtype=torch.uint8, device="cuda")
    ud = torch.from_numpy(u).cuda()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        ctx.sample(z, 3000, ud, token, workspace=ws)
    stream.synchronize()
    assert torch.equal(token, want["token"])


def test_sample_in_a_graph():
    rng = np.random.default_rng(2)
    z, ctx, vocab = _logits(2, 6, 70001, "bf16"), _ctx(), 70001
    settings = dict(temperature=np.array([0.7, 1, 0, 1.2, 1, 0.9]), top_k=np.array([0, 50, 3, 1000, 0, 7]), top_p=np.array([0.9, 1, 0.5, 0.95, 1, 0.7]))
    dev = {k: _i32(v) if k == "top_k" else torch.from_numpy(v.astype(np.float32)).cuda() for k, v in settings.items()}
    o = dict(token=_i32(np.zeros(6)), logprob=torch.zeros(6, device="cuda"), n_kept=_i32(np.zeros(6)))
    u = torch.zeros(6, device="cuda")
    ws = torch.empty(max(256, ctx.sample_workspace_bytes(6, vocab)), dtype=torch.uint8, device="cuda")
    run = lambda: ctx.sample(z, vocab, u, o["token"], logprob=o["logprob"], n_kept=o["n_kept"], workspace=ws, **dev)
    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for rep in range(4):
        draw = rng.random(6, dtype=np.float32)
        z.copy_(_logits(100 + rep, 6, vocab, "bf16"))
        u.copy_(torch.from_numpy(draw))
        for t in o.values():
            t.fill_(-9)
        ws.fill_(255)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        _check_sample(o, z, vocab, draw, **settings)


# ---- all of them: answers behind a prefill -------------------------------------------------------------------------------------
def _answer_setup(dtype, n_layers=2, answer=20, window=None, vocab=None, **settings):
    import workload as W
    from paper_2502_15734_amd.layers import AnswerLoop, DecoderLoop
    hq, hkv, d = (8, 2, 128) if dtype == "bf16" else (4, 2, 64)
    reqs = [W.RequestSpec([0, 1, 2], [0.3, 0.2, 0.25], 21), W.RequestSpec([2, 0], [0.5, 0.15], 16), W.RequestSpec([1], [0.2], 3)]
    w = W.custom("answer", dtype, hq, hkv, d, THETA, [100, 77, 64], [0, 5, 0], reqs, 1.0 / math.sqrt(d), seed=53, hidden=256)
    ffn, vocab = (640 if dtype == "bf16" else 160), vocab or (640 if dtype == "bf16" else 611)
    weights = [W.layer_weights(w.spec, 256, ffn, layer=l, qkv_scale=1.0 / 16) for l in range(n_layers)]
    rng = np.random.default_rng(7)
    rnd = W.round_to_bf16 if dtype == "bf16" else (lambda a: a)
    embed = rnd(rng.standard_normal((vocab, 256)).astype(np.float32))
    w_out = rnd((rng.standard_normal((vocab, 256)) / 4).astype(np.float32))
    gain = rnd(np.float32(1.0) + 0.1 * rng.standard_normal(256).astype(np.float32))
    loop = DecoderLoop(w, weights, window=window, answer_tokens=answer)
    loop.run()
    before = [(k.float().cpu().numpy(), v.float().cpu().numpy(), m.cpu().numpy()) for k, v, m in loop.pages]
    ans = AnswerLoop(loop, embed, gain, w_out, **settings)
    return w, weights, loop, ans, before, (embed, gain, w_out)


def _oracle_answer(w, weights, ans, before, model, tokens, eps=1.0e-5):
    """Logits in front of every token, in 64 bits, of answers that go `tokens` [steps, requests], from the pages and hidden states the prefill left."""
    from oracle import cachecraft_oracle as O
    embed, gain, w_out = (np.asarray(a, np.float64) for a in model)
    hq, hkv, d = w.spec.n_q_heads, w.spec.n_kv_heads, w.spec.head_dim
    store = ans.b.v_store.float().cpu().numpy()
    out = [[] for _ in tokens]
    last = ans.loop.h[ans.b.cu_q[1:].long() - 1].double().cpu().numpy()
    for r in range(w.n_requests):
        caches = []
        for k, v, m in before:
            caches.append(list(A.paged_context(k, v, lambda p: store[m[p]] if m[p] >= 0 else v[p], w.req_tab, w.segments, range(w.req_seg_off[r], w.req_seg_off[r + 1]))))
        h = last[r:r + 1]
        for step in range(len(tokens)):
            if step:
                h = embed[tokens[step - 1][r]][None]
                for lw, cache in zip(weights, caches):
                    x = O.rms_norm(h, lw.gain_attn, lw.eps)
                    qkv = x @ np.asarray(lw.w_qkv, np.float64).T
                    q, kn, vn = qkv[:, :hq * d].reshape(1, hq, d), qkv[:, hq * d:(hq + hkv) * d].reshape(1, hkv, d), qkv[:, (hq + hkv) * d:].reshape(1, hkv, d)
                    p = len(cache[0])
                    cache[0], cache[1], cache[2] = np.append(cache[0], p), np.concatenate([cache[1], A.rotate(kn, [p], THETA)]), np.concatenate([cache[2], vn])
                    o = A.attend(q, np.array([p]), *cache, THETA, 0.0)[0].reshape(1, -1)
                    h1 = h + O.linear(o, lw.w_o)
                    h = h1 + O.linear(O.gated_ffn_in(O.rms_norm(h1, lw.gain_ffn, lw.eps), lw.w_gate, lw.w_up), lw.w_down)
            out[step].append(O.linear(O.rms_norm(h, gain, eps), w_out)[0])
    return np.array(out)


@pytest.mark.parametrize("dtype,window", [("f32", None), ("bf16", None), ("bf16", 2)])
def test_answer_loop_matches_the_oracle(dtype, window):
    """Prefill, then 21 tokens of three requests (pages fill and new ones begin): logits in front of every token against the oracle that is fed the
    same tokens, tokens against the oracle's draw from the library's logits.  Tolerance: a layer's bar of relative error (each of its operators is inside
    it) per layer and one more for the logits, as a free-running loop inherits them."""
    steps = 21
    w, weights, loop, ans, before, model = _answer_setup(dtype, n_layers=2 if window is None else 3, window=window, temperature=[0.8, 0.0, 1.2], top_k=[0, 0, 40], top_p=[0.9, 1.0, 0.95], min_p=0.01)
    u = np.random.default_rng(3).random((steps, 3), dtype=np.float32)
    tokens, logprobs, logits = ans.run(u, keep=True)
    want = _oracle_answer(w, weights, ans, before, model, tokens)
    bar = (1e-2 if dtype == "bf16" else 2e-5) * (len(weights) + 1)
    for step in range(steps):
        for r in range(3):
            off = np.linalg.norm(logits[step][r] - want[step][r]) / np.linalg.norm(want[step][r])
            assert off <= bar, f"step {step} request {r}: logits {off:.3e} off"
            t = (0.8, 0.0, 1.2)[r], (0, 0, 40)[r], float(np.float32((0.9, 1.0, 0.95)[r])), float(np.float32(0.01))
            drawn = A.sample(logits[step][r], float(np.float32(t[0])), *t[1:], float(u[step, r]))
            assert tokens[step, r] == drawn[0] and abs(logprobs[step, r] - drawn[1]) <= 2.0 ** -24 * abs(drawn[1]) + 2.0 ** -40
    assert len(set(tokens[:, 0])) > 3
    seg = ans.segs.cpu().numpy()
    assert (seg[np.asarray(w.req_seg_off[1:]) - 1, 3] == [21 + 20, 16 + 20, 3 + 20]).all()
    with pytest.raises(ValueError):
        ans.run(u[:1])
    loop.close()


def test_answer_loop_in_a_graph_and_in_pieces():
    """Steps replayed from a graph, and a run in two pieces: the same bits as eager steps."""
    u = np.random.default_rng(4).random((18, 3), dtype=np.float32)
    runs = []
    for how in ("eager", "graph", "pieces"):
        _, _, loop, ans, _, _ = _answer_setup("bf16", temperature=1.0, top_p=0.95)
        if how == "pieces":
            parts = [ans.run(u[:5], keep=True), ans.run(u[5:], keep=True, graph=True)]
            runs.append([np.concatenate([a, b]) for a, b in zip(*(p[:2] for p in parts))] + [parts[0][2] + parts[1][2]])
        else:
            runs.append(ans.run(u, graph=how == "graph", keep=True))
        loop.close()
    for other in runs[1:]:
        assert np.array_equal(runs[0][0], other[0]) and np.array_equal(runs[0][1], other[1])
        assert all(np.array_equal(a, b) for a, b in zip(runs[0][2], other[2]))


@pytest.mark.parametrize("graph", [False, True])
def test_answer_loop_stops(graph):
    """A request that draws the stop token gets -1 from then on, the others go on as if it were not there."""
    u = np.random.default_rng(5).random((16, 3), dtype=np.float32)
    _, _, loop, ans, _, _ = _answer_setup("f32", temperature=1.0)
    free, _ = ans.run(u)
    loop.close()
    stop = int(free[6, 1])
    _, _, loop, ans, _, _ = _answer_setup("f32", temperature=1.0, stop=stop)
    got, _ = ans.run(u, graph=graph)
    for r in range(3):
        ends = np.nonzero(free[:, r] == stop)[0]
        n = int(ends[0]) + 1 if len(ends) else len(free)
        assert np.array_equal(got[:n, r], free[:n, r]) and (got[n:, r] == -1).all()
    assert (got[7:, 1] == -1).all()
    loop.close()


def _ended(got, logprobs, free, r, n):
    """Request r's tokens are those of the free run up to step n, and nothing from there on."""
    assert np.array_equal(got[:n, r], free[:n, r]) and (got[n:, r] == -1).all()
    assert np.isfinite(logprobs[:n, r]).all() and np.isneginf(logprobs[n:, r]).all()


def test_answer_loop_log_probabilities_of_stopped_requests():
    u = np.random.default_rng(5).random((16, 3), dtype=np.float32)
    _, _, loop, ans, _, _ = _answer_setup("f32", temperature=1.0)
    free, _ = ans.run(u)
    loop.close()
    stop = int(free[6, 1])
    _, _, loop, ans, _, _ = _answer_setup("f32", temperature=1.0, stop=stop)
    got, logprobs = ans.run(u)
    for r in range(3):
        at = np.nonzero(free[:, r] == stop)[0]
        _ended(got, logprobs, free, r, int(at[0]) + 1 if len(at) else len(free))
    loop.close()


@pytest.mark.parametrize("graph", [False, True])
def test_answer_loop_ends_where_nothing_can_be_drawn(graph):
    """A token whose embedding is NaN: the logits behind it are all NaN, and the request gets -1 and nothing more; the others go on."""
    u = np.random.default_rng(6).random((14, 3), dtype=np.float32)
    _, _, loop, ans, _, _ = _answer_setup("f32", temperature=1.0)
    free, _ = ans.run(u)
    loop.close()
    bad = int(free[4, 1])
    _, _, loop, ans, _, _ = _answer_setup("f32", temperature=1.0)
    ans.embed[bad] = math.nan
    got, logprobs = ans.run(u, graph=graph)
    for r in range(3):
        at = np.nonzero(free[:, r] == bad)[0]
        _ended(got, logprobs, free, r, int(at[0]) + 1 if len(at) else len(free))
    assert (got[5:, 1] == -1).all() and int(ans.n_kept[1]) == 0
    loop.close()
    _, _, loop, ans, _, _ = _answer_setup("f32", temperature=1.0)
    ans.logits[1] = -math.inf                                            # ... and a prompt that leaves nothing
    got, logprobs = ans.run(u, graph=graph)
    for r in range(3):
        _ended(got, logprobs, free, r, 0 if r == 1 else len(free))
    loop.close()


@pytest.mark.parametrize("graph", [False, True])
def test_answer_loop_ends_where_no_row_is_left(graph):
    """A request whose table is full gets nothing from then on, whatever logits an earlier step left."""
    u = np.random.default_rng(7).random((9, 3), dtype=np.float32)
    _, _, loop, ans, _, _ = _answer_setup("f32", temperature=1.0)
    free, _ = ans.run(u)
    loop.close()
    for r, n in ((1, 1), (2, 9)):                                       # (a question of 16 tokens fills its page, one of 3 has room for 13 more)
        _, _, loop, ans, _, _ = _answer_setup("f32", temperature=1.0)
        ans.tab_cap[ans.last_seg[r]] = 1
        got, logprobs = ans.run(u, graph=graph)
        for i in range(3):
            _ended(got, logprobs, free, i, n if i == r else 9)
        loop.close()


def test_answer_loops_one_behind_the_other():
    """A second answer from the same prefill is what it would be alone; the first cannot go on over its tokens, nor the second over another prefill's."""
    from paper_2502_15734_amd.layers import AnswerLoop
    u = np.random.default_rng(8).random((12, 3), dtype=np.float32)
    _, _, loop, first, _, model = _answer_setup("bf16", temperature=1.0)
    want, _ = first.run(u)
    _, _, loop, first, _, model = _answer_setup("bf16", temperature=1.0)
    first.run(np.flip(u)[:7])
    second = AnswerLoop(loop, *model, temperature=1.0)
    got, _ = second.run(u[:5])
    with pytest.raises(ValueError, match="taken the pages"):
        first.run(u[:1])
    more, _ = second.run(u[5:])
    assert np.array_equal(np.concatenate([got, more]), want)
    loop.run()
    with pytest.raises(ValueError, match="taken the pages"):
        second.run(u[:1])
    got, _ = AnswerLoop(loop, *model, temperature=1.0).run(u)
    assert np.array_equal(got, want)
    loop.close()


def test_answer_loop_of_no_steps():
    _, _, loop, ans, _, _ = _answer_setup("f32", answer=3, temperature=1.0)
    u = np.random.default_rng(9).random((4, 3), dtype=np.float32)
    first, then, behind = ans.run(u[:0]), ans.run(u, keep=True), ans.run(u[:0], keep=True)
    assert first[0].shape == first[1].shape == (0, 3) and behind[0].shape == (0, 3) and behind[2] == [] and then[0].shape == (4, 3)
    assert first[0].dtype == then[0].dtype and first[1].dtype == then[1].dtype
    loop.close()
