"""The operators of the answer that follows a selective prefill, at the sizes they are called with: their inputs, their plain form,
and the calls of paper_2502_15734_amd.Context that compute them.

  extend   cc_extend_segments: every segment of every request gets some tokens behind those its pages hold; pages come from a free
           list.  Writes the segment table, the page table, and position, cache slot and request of every new row.
  attend   cc_append_attention: the new rows' keys and values go into their slots, then each row attends causally over the whole
           paged context of its request (a row per request while an answer is written, several for a draft that is checked, hundreds
           for a further question).
  sample   cc_sample: one token per row of logits, with temperature, top-k, top-p and min-p, from given uniform numbers.

`own` False: the plain form, elementary torch operations.  True: the library's calls.
"""
import math
import random

import numpy as np
import torch

own = False

BLOCK = 16
DEVICE = "cuda"
THETA = 5.0e5
SEGMENT = 8            # int32 fields of a segment: request, kind, start, tokens, table offset, rows, token offset, row offset


# ---- the cases -----------------------------------------------------------------------------------------------------------------
def _extend(requests, chunks, length, question, new, reserve=64, short=False, layout=1, **name):
    """new: "one" (a token per request), "mixed" (most one, some a further question of up to 512 tokens, some none), "prompt" (all
    tokens of all segments: tables from nothing).  short: the free list lacks pages for the last requests."""
    return dict(op="extend", requests=requests, chunks_lo=chunks[0], chunks_hi=chunks[1], len_lo=length[0], len_hi=length[1],
                question_lo=question[0], question_hi=question[1], new=new, reserve=reserve, short=short, layout=layout, **name)


def _attend(requests, context, new, heads=(32, 8), dim=128, dtype="bf16", layout=1, **name):
    """context: the range of a request's tokens, the new ones included; new: new tokens of a request."""
    return dict(op="attend", requests=requests, ctx_lo=context[0], ctx_hi=context[1], new=new, q_heads=heads[0], kv_heads=heads[1],
                head_dim=dim, dtype=dtype, layout=layout, **name)


def _sample(rows, vocab, dtype, mode, pad=0, **name):
    """mode: "greedy", "k", "p", "min", "mixed" (each row its own settings), "plain" (temperature alone); pad: columns behind the vocabulary."""
    return dict(op="sample", rows=rows, vocab=vocab, dtype=dtype, mode=mode, pad=pad, **name)


def listed():
    return [
        # the tables of one step of a batch of 32 answers over 5 to 10 chunks each: all latency
        _extend(32, (5, 10), (256, 1024), (32, 128), "one", name="rows_32_answers"),
        # a step in which most requests answer, some bring a further question, and pages run out
        _extend(250, (1, 10), (100, 1024), (32, 128), "mixed", reserve=512, short=True, layout=2, name="rows_250_mixed"),
        # the tables of 500 whole prompts, from lengths alone
        _extend(500, (5, 12), (256, 1024), (32, 128), "prompt", layout=3, name="rows_500_prompts"),
        # one user, a short context, the next token: the smallest call
        _attend(1, (700, 700), 1, name="next_1x700"),
        # the batch of 32 requests of 1500 to 6700 tokens, a token each
        _attend(32, (1500, 6700), 1, layout=4, name="next_32_ragged"),
        # one very long context: few rows, everything is the split of the keys
        _attend(1, (130049, 130049), 1, layout=5, name="next_1x130k"),
        # five drafted tokens of 16 requests at once, 64 query heads on 8
        _attend(16, (1000, 8000), 5, heads=(64, 8), layout=6, name="draft_16x5_70b"),
        # a further question of 500 tokens over a context of 16000
        _attend(1, (16400, 16400), 500, layout=7, name="question_500_over_16k"),
        # fp32, small heads, an odd group
        _attend(6, (300, 3001), 2, heads=(6, 2), dim=64, dtype="f32", layout=8, name="next_6_f32"),
        # one answer's next token, fp32 logits, top-p
        _sample(1, 32000, "f32", "p", name="sample_1x32000"),
        # a batch of 32, bf16 logits (many equal ones), every request its own settings
        _sample(32, 128256, "bf16", "mixed", name="sample_32x128256"),
        # the largest batch, odd vocabulary, fp32 logits with padding columns
        _sample(256, 128001, "f32", "mixed", pad=255, name="sample_256x128001"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("extend", "attend", "attend", "sample"))
    layout = rng.randrange(1 << 20)
    if op == "extend":
        lo = rng.randint(1, 6)
        length = _log(rng, 16, 600)
        return _extend(_log(rng, 1, 500), (lo, lo + rng.randint(0, 5)), (length, length + rng.randint(0, 400)), (1, rng.randint(1, 128)),
                       rng.choice(("one", "mixed", "prompt")), reserve=rng.randint(0, 600), short=rng.random() < 0.3, layout=layout)
    if op == "attend":
        requests = _log(rng, 1, 64)
        heads, dim, dtype = rng.choice((((32, 8), 128, "bf16"), ((64, 8), 128, "bf16"), ((8, 8), 128, "bf16"), ((12, 4), 64, "bf16"), ((4, 2), 64, "f32"), ((8, 2), 128, "f32")))
        top = 130000 // requests
        hi = _log(rng, 2, top)
        lo = max(1, int(hi * rng.uniform(0.1, 1.0)))
        new = 1 if rng.random() < 0.5 else _log(rng, 1, 512)
        new = max(1, min(new, lo, 500 * 16400 * 32 // (requests * hi * heads[0])))
        return _attend(requests, (lo, hi), new, heads=heads, dim=dim, dtype=dtype, layout=layout)
    return _sample(_log(rng, 1, 256), _log(rng, 500, 128256), rng.choice(("bf16", "f32")), rng.choice(("greedy", "k", "p", "min", "mixed", "plain")),
                   pad=rng.choice((0, 0, 1, 64)))


def work(case):
    if case["op"] == "extend":
        s = _extend_tables(case)
        rows = int(s["n_new"].sum())
        pages = int(((s["segs"][:, 3] + s["n_new"] + BLOCK - 1) // BLOCK - (s["segs"][:, 3] + BLOCK - 1) // BLOCK).sum())
        n_segs, n_req = len(s["segs"]), case["requests"]
        # segment tables in and out, lengths and capacities, offsets; per row position, slot and request; per page its number in and out
        return {"bytes": n_segs * (2 * 4 * SEGMENT + 8) + n_req * 16 + rows * 12 + pages * 8, "flops": rows * 4.0}
    if case["op"] == "attend":
        lens, size = _contexts(case), 2 if case["dtype"] == "bf16" else 4
        hq, hkv, d, n = case["q_heads"], case["kv_heads"], case["head_dim"], case["new"]
        rows = n * case["requests"]
        keys = sum(int(v) for v in lens)
        seen = sum(n * int(v) - n * (n - 1) // 2 for v in lens)
        return {"bytes": (2 * keys * hkv * d + rows * (2 * hq + 2 * hkv) * d) * size + keys // BLOCK * 4, "flops": 4.0 * hq * d * seen}
    return {"bytes": case["rows"] * (case["vocab"] * (2 if case["dtype"] == "bf16" else 4) + 32.0), "flops": 4.0 * case["rows"] * case["vocab"]}


# ---- inputs --------------------------------------------------------------------------------------------------------------------
def _extend_tables(case):
    """The tables on the host (from the case alone): old lengths, new tokens, table offsets and room."""
    rs = np.random.RandomState(case["layout"])
    per = rs.randint(case["chunks_lo"], case["chunks_hi"] + 1, case["requests"]) + 1          # chunks and the question
    off = np.concatenate([[0], np.cumsum(per)])
    n = int(off[-1])
    req = np.repeat(np.arange(case["requests"]), per)
    last = np.zeros(n, bool)
    last[off[1:] - 1] = True
    tokens = np.where(last, rs.randint(case["question_lo"], case["question_hi"] + 1, n), rs.randint(case["len_lo"], case["len_hi"] + 1, n))
    new = np.zeros(n, np.int64)
    if case["new"] == "prompt":
        old, new = np.zeros(n, np.int64), tokens
    else:
        old = tokens + np.where(last, rs.randint(0, 64, n), 0)
        kind = rs.random_sample(n) if case["new"] == "mixed" else np.zeros(n)
        new[last] = np.where(kind < 0.8, 1, np.where(kind < 0.9, rs.randint(2, 513, n), 0))[last]
    cap = (old + new + np.where(last, case["reserve"], 0) + BLOCK - 1) // BLOCK
    segs = np.zeros((n, SEGMENT), np.int64)
    segs[:, 0], segs[:, 1], segs[:, 3] = req, last, old
    segs[:, 4] = np.concatenate([[0], np.cumsum(cap)[:-1]])
    return dict(segs=segs, n_new=new, cap=cap, req_seg_off=off)


def _contexts(case):
    return np.random.RandomState(case["layout"]).randint(case["ctx_lo"], case["ctx_hi"] + 1, case["requests"])


def _int(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).to(DEVICE)


def _prepare_extend(case, seed):
    t, rs = _extend_tables(case), np.random.RandomState(seed)
    held = (t["segs"][:, 3] + BLOCK - 1) // BLOCK
    need = int(((t["segs"][:, 3] + t["n_new"] + BLOCK - 1) // BLOCK - held).sum())
    n_held, n_tab = int(held.sum()), int(t["cap"].sum())
    n_free = need * 3 // 4 if case["short"] else need + 37
    ids = rs.permutation(n_held + n_free + 11)
    table = np.full(n_tab, -1, np.int64)
    at = np.repeat(t["segs"][:, 4] - np.concatenate([[0], np.cumsum(held)[:-1]]), held) + np.arange(n_held)
    table[at] = ids[:n_held]
    rows = int(t["n_new"].sum()) + 5
    n_req = case["requests"]
    return dict(case=case, segs_in=_int(t["segs"]), n_new=_int(t["n_new"]), tab_cap=_int(t["cap"]), req_seg_off=_int(t["req_seg_off"]),
                free_blocks=_int(ids[n_held:n_held + n_free]), block_tab=_int(table), n_blocks=len(ids),
                segs=_int(np.zeros_like(t["segs"])), cu_q=_int(np.zeros(n_req + 1)), q_pos=_int(np.zeros(rows)), slot_map=_int(np.zeros(rows)),
                row_req=_int(np.zeros(rows)), last_row=_int(np.zeros(n_req)), status=_int(np.zeros(n_req)), counts=_int(np.zeros(4)))


def _prepare_attend(case, seed):
    """Contexts of chunks of 256 to 1024 tokens and a question, on pages in random order; the last `new` tokens of each are the rows."""
    lens, new = _contexts(case), case["new"]
    n = np.random.RandomState(case["layout"] + 1).randint(256, 1025, (case["requests"], int(lens.max()) // 256 + 2))
    start = np.cumsum(n, 1) - n
    chunk = lens[:, None] - start - new > 1100                                               # what is left behind them is the question
    last = chunk.sum(1)
    req, nth = np.nonzero(np.arange(n.shape[1])[None] <= last[:, None])
    tail = nth == last[req]
    n = np.where(tail, lens[req] - start[req, nth], n[req, nth])
    pages = (n + BLOCK - 1) // BLOCK
    off, first = np.concatenate([[0], np.cumsum(last + 1)]), int(pages.sum())
    segs = np.stack([req, tail, start[req, nth], n, np.cumsum(pages) - pages, tail * new, np.cumsum(n) - n,
                     req * new], 1)
    table = np.random.RandomState(seed).permutation(first + 3)[:first]
    ends = segs[off[1:] - 1]
    tok = ends[:, 3][:, None] - new + np.arange(new)[None]                                    # index of each row in its last segment
    slots = table[ends[:, 4][:, None] + tok // BLOCK] * BLOCK + tok % BLOCK
    g = torch.Generator(device=DEVICE).manual_seed(seed)
    kind = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    hq, hkv, d, rows = case["q_heads"], case["kv_heads"], case["head_dim"], new * case["requests"]

    def normal(*shape):
        return torch.randn(shape, generator=g, device=DEVICE, dtype=torch.float32).to(kind)
    return dict(case=case, q=normal(rows, hq, d), k_new=normal(rows, hkv, d), v_new=normal(rows, hkv, d), k_pool=normal(first + 3, hkv, BLOCK, d),
                v_pool=normal(first + 3, hkv, d, BLOCK), segs=_int(segs), req_seg_off=_int(off), block_tab=_int(table),
                q_pos=_int((ends[:, 2][:, None] + tok).reshape(-1)), slot_map=_int(slots.reshape(-1)),
                cu_q=_int(np.arange(case["requests"] + 1) * new), out=torch.zeros(rows, hq, d, device=DEVICE, dtype=kind),
                max_ctx=int(lens.max()), max_segs=int(np.diff(off).max()))


def _prepare_sample(case, seed):
    """Logits as a model gives them: a broad bell, some hundred likely tokens, a few forbidden ones."""
    g = torch.Generator(device=DEVICE).manual_seed(seed)
    rows, vocab, mode = case["rows"], case["vocab"], case["mode"]
    z = torch.randn(rows, vocab + case["pad"], generator=g, device=DEVICE) * 2.0
    many = max(1, min(200, vocab // 4))
    z.scatter_add_(1, torch.randint(0, vocab, (rows, many), generator=g, device=DEVICE), torch.rand(rows, many, generator=g, device=DEVICE) * 14)
    z.scatter_(1, torch.randint(0, vocab, (rows, 3), generator=g, device=DEVICE), -math.inf)
    rs = np.random.RandomState(seed)
    pick = rs.randint(0, 6, rows) if mode == "mixed" else np.full(rows, {"greedy": 0, "k": 1, "p": 2, "min": 3, "plain": 4}[mode])
    heat = np.where(pick == 0, 0.0, rs.uniform(0.5, 1.3, rows))
    top_k = np.where((pick == 1) | (pick == 5), rs.randint(1, 101, rows), 0)
    top_p = np.where((pick == 2) | (pick == 5), rs.uniform(0.5, 0.99, rows), 1.0)
    min_p = np.where((pick == 3) | (pick == 5), rs.uniform(0.005, 0.2, rows), 0.0)

    def real(a):
        return torch.from_numpy(a.astype(np.float32)).to(DEVICE)
    return dict(case=case, logits=z.to(torch.bfloat16 if case["dtype"] == "bf16" else torch.float32), temperature=real(heat), top_k=_int(top_k),
                top_p=real(top_p), min_p=real(min_p), u=torch.rand(rows, generator=g, device=DEVICE), token=_int(np.zeros(rows)),
                n_kept=_int(np.zeros(rows)), logprob=torch.zeros(rows, device=DEVICE))


def prepare(case, seed):
    return {"extend": _prepare_extend, "attend": _prepare_attend, "sample": _prepare_sample}[case["op"]](case, seed)


# ---- the plain form ------------------------------------------------------------------------------------------------------------
def _before(a):
    return torch.cumsum(a, 0) - a


def _plain_extend(s):
    seg, off, tab = s["segs_in"].long(), s["req_seg_off"].long(), s["block_tab"]
    n_segs, n_req, n_tab, n_free, n_rows = seg.shape[0], off.shape[0] - 1, tab.shape[0], s["free_blocks"].shape[0], s["q_pos"].shape[0]
    req = torch.searchsorted(off[1:].contiguous(), torch.arange(n_segs, device=DEVICE), right=True)

    def per_request(a):
        return torch.zeros(n_req, dtype=torch.long, device=DEVICE).index_add_(0, req, a.long())
    old, add = seg[:, 3].clamp(min=0), s["n_new"].long().clamp(min=0)
    first = seg[:, 4]
    held = (old + BLOCK - 1) // BLOCK
    after = (old + add + BLOCK - 1) // BLOCK
    # what a request cannot have: table entries it does not own, tokens in front of ones whose positions are fixed, pages, rows
    full = (add > 0) & ((after > s["tab_cap"].long()) | (first < 0) | (first + after > n_tab))
    behind = torch.cumsum(old, 0)
    behind = behind[off[1:] - 1][req] - behind
    status = torch.where(per_request((add > 0) & (behind > 0)) > 0, 3, 0)
    status = torch.where((per_request(full) > 0) | (per_request(old + add) >= 2 ** 31), 2, status)
    ok = (status == 0).long()
    pages, rows = per_request(after - held) * ok, per_request(add) * ok
    status = torch.where((rows > 0) & (torch.cumsum(rows, 0) > n_rows), 4, status)
    status = torch.where((pages > 0) & (torch.cumsum(pages, 0) > n_free), 1, status)
    ok = (status == 0).long()
    add = add * ok[req]
    after = (old + add + BLOCK - 1) // BLOCK
    total = old + add
    row0, page0, tok0 = _before(add), _before(after - held), _before(total)
    start = tok0 - tok0[off[:-1]][req]
    n_added, n_pages = add.sum(), (after - held).sum()
    segs = torch.stack((seg[:, 0], seg[:, 1], start, total, first, add, tok0, row0), 1).int()
    # pages from the free list into the table
    p = torch.arange(n_free, device=DEVICE)
    of = torch.searchsorted(torch.cumsum(after - held, 0), p, right=True).clamp(max=n_segs - 1)
    to = torch.where(p < n_pages, first[of] + held[of] + p - page0[of], n_tab)
    tab = torch.cat((tab, tab.new_zeros(1))).index_copy_(0, to, s["free_blocks"])[:n_tab] if n_free else tab.clone()
    # rows
    j = torch.arange(n_rows, device=DEVICE)
    of = torch.searchsorted(torch.cumsum(add, 0), j, right=True).clamp(max=n_segs - 1)
    t = old[of] + j - row0[of]
    page = tab[(first[of] + t // BLOCK).clamp(0, n_tab - 1)].long()
    live = j < n_added
    slot = torch.where(live & (page >= 0) & (page < s["n_blocks"]), page * BLOCK + t % BLOCK, -1)
    n_r = per_request(add)
    cu = torch.cat((n_r.new_zeros(1), torch.cumsum(n_r, 0)))
    s["block_tab"].copy_(tab)
    counts = torch.stack((n_added, n_pages, n_req - ok.sum(), total.sum()))
    return [segs, s["block_tab"], cu.int(), torch.where(live, start[of] + t, 0).int(), slot.int(), torch.where(live, req[of], -1).int(),
            torch.where(n_r > 0, cu[1:] - 1, -1).int(), status.int(), counts.int()]


def _rotate(x, pos):
    """x [rows, heads, d] at positions pos, angles in 64 bits."""
    half = x.shape[-1] // 2
    a = pos.double()[:, None] * THETA ** (-torch.arange(half, device=DEVICE, dtype=torch.float64) / half)
    c, s = torch.cos(a).to(x.dtype)[:, None], torch.sin(a).to(x.dtype)[:, None]
    return torch.cat((x[..., :half] * c - x[..., half:] * s, x[..., half:] * c + x[..., :half] * s), -1)


def _plain_attend(s):
    c, kind = s["case"], s["q"].dtype
    hq, hkv, d, n_req = c["q_heads"], c["kv_heads"], c["head_dim"], c["requests"]
    pos, slot = s["q_pos"].long(), s["slot_map"].long()
    s["k_pool"][slot // BLOCK, :, slot % BLOCK] = _rotate(s["k_new"].float(), pos).to(kind)
    s["v_pool"][slot // BLOCK, :, :, slot % BLOCK] = s["v_new"]
    # the pages of every request, padded to the longest list
    seg, off = s["segs"].long(), s["req_seg_off"].long()
    pages = (seg[:, 3] + BLOCK - 1) // BLOCK
    ends = torch.cumsum(pages, 0)
    edge = torch.cat((ends.new_zeros(1), ends))[off]
    width = s["max_ctx"] // BLOCK + s["max_segs"]
    g = edge[:-1, None] + torch.arange(width, device=DEVICE)
    of = torch.searchsorted(ends, g.reshape(-1), right=True).clamp(max=seg.shape[0] - 1).view(n_req, width)
    nth = g - (ends - pages)[of]
    live = g < edge[1:, None]
    page = s["block_tab"].long()[torch.where(live, seg[:, 4][of] + nth, 0)]
    at = nth[..., None] * BLOCK + torch.arange(BLOCK, device=DEVICE)
    key_pos = torch.where(live[..., None] & (at < seg[:, 3][of][..., None]), seg[:, 2][of][..., None] + at, 1 << 40).reshape(n_req, 1, 1, -1)
    k = s["k_pool"][page].permute(0, 2, 1, 3, 4).reshape(n_req * hkv, width * BLOCK, d).float()
    v = s["v_pool"][page].permute(0, 2, 1, 4, 3).reshape(n_req * hkv, width * BLOCK, d).float()
    # rows [request, KV head, new token and head of the group]
    n, group = c["new"], hq // hkv
    q = _rotate(s["q"].float(), pos).view(n_req, n, hkv, group, d).permute(0, 2, 1, 3, 4).reshape(n_req * hkv, n * group, d)
    z = torch.bmm(q, k.transpose(1, 2)) / math.sqrt(d)
    z = z.view(n_req, hkv, n * group, -1).masked_fill_(key_pos > pos.view(n_req, 1, n, 1).expand(n_req, 1, n, group).reshape(n_req, 1, n * group, 1), -math.inf)
    p = torch.exp(z - z.amax(-1, keepdim=True))
    p /= p.sum(-1, keepdim=True)
    o = torch.bmm(p.view(n_req * hkv, n * group, -1), v)
    s["out"].copy_(o.view(n_req, hkv, n, group, d).permute(0, 2, 1, 3, 4).reshape(n_req * n, hq, d))
    return [s["out"], s["k_pool"], s["v_pool"]]


def _plain_sample(s):
    """In 64 bits: a token's number depends on sums next to a border."""
    vocab = s["case"]["vocab"]
    z = s["logits"][:, :vocab].double()
    heat = s["temperature"].double()[:, None]
    order, idx = torch.sort(z, dim=1, descending=True, stable=True)
    scale = torch.where(heat > 0, heat, 1.0)
    w = torch.exp((order - order[:, :1]) / scale)
    rank = torch.arange(vocab, device=DEVICE)[None]
    k = s["top_k"].long()[:, None]
    k = torch.where((k <= 0) | (k > vocab), vocab, k)
    k = torch.where(heat > 0, k, 1)
    sums = torch.cumsum(w, 1)
    before = torch.cat((torch.zeros_like(sums[:, :1]), sums[:, :-1]), 1)
    top_p = s["top_p"].double()[:, None]
    in_p = (before < top_p * sums.gather(1, k - 1)) | (top_p >= 1)
    kept = (rank < k) & in_p & (w >= s["min_p"].double()[:, None]) & (order > -math.inf)
    kept = kept | ((rank == 0) & (order > -math.inf))
    weight = torch.zeros_like(w).scatter_(1, idx, torch.where(kept, w, 0.0))
    sums = torch.cumsum(weight, 1)
    token = torch.searchsorted(sums, s["u"].double()[:, None] * sums[:, -1:], right=True)
    prob = weight.gather(1, token.clamp(max=vocab - 1)) / sums[:, -1:]
    return [token[:, 0].int(), torch.log(prob[:, 0]).float(), kept.sum(1).int()]


# ---- the library's calls -------------------------------------------------------------------------------------------------------
def _handle(s):
    """The context and workspace that a program keeps beside its buffers."""
    import paper_2502_15734_amd as P
    c = s["case"]
    bf16 = c.get("dtype", "bf16") == "bf16"
    s["ctx"] = ctx = P.Context(c.get("q_heads", 32), c.get("kv_heads", 8), c.get("head_dim", 128), THETA, P.CC_BF16 if bf16 else P.CC_F32)
    need = (ctx.extend_segments_workspace_bytes(s["segs_in"].shape[0], c["requests"]) if c["op"] == "extend" else
            ctx.append_attention_workspace_bytes(s["q"].shape[0], c["new"], c["requests"], s["max_ctx"], s["max_segs"]) if c["op"] == "attend" else
            ctx.sample_workspace_bytes(c["rows"], c["vocab"]))
    s["workspace"] = torch.empty(max(256, need), dtype=torch.uint8, device=DEVICE)


def _own(s):
    if "ctx" not in s:
        _handle(s)
    c, ctx = s["case"], s["ctx"]
    if c["op"] == "extend":
        ctx.extend_segments(s["segs_in"], s["n_new"], s["tab_cap"], s["req_seg_off"], s["free_blocks"], s["block_tab"], s["n_blocks"], s["segs"],
                            s["cu_q"], s["q_pos"], s["slot_map"], s["row_req"], s["last_row"], s["status"], s["counts"], s["workspace"])
        return [s["segs"], s["block_tab"], s["cu_q"], s["q_pos"], s["slot_map"], s["row_req"], s["last_row"], s["status"], s["counts"]]
    if c["op"] == "attend":
        ctx.append_attention(s["q"], s["k_new"], s["v_new"], s["q_pos"], s["slot_map"], s["cu_q"], c["new"], s["k_pool"], s["v_pool"],
                             s["block_tab"], s["segs"], s["req_seg_off"], c["requests"], s["max_ctx"], s["max_segs"], s["out"], None, s["workspace"])
        return [s["out"], s["k_pool"], s["v_pool"]]
    ctx.sample(s["logits"], c["vocab"], s["u"], s["token"], temperature=s["temperature"], top_k=s["top_k"], top_p=s["top_p"], min_p=s["min_p"],
               logprob=s["logprob"], n_kept=s["n_kept"], workspace=s["workspace"])
    return [s["token"], s["logprob"], s["n_kept"]]


def run(state):
    if own:
        return _own(state)
    return {"extend": _plain_extend, "attend": _plain_attend, "sample": _plain_sample}[state["case"]["op"]](state)


# ---- the definitions in 64 bits ------------------------------------------------------------------------------------------------
def exact(case, seed):
    if case["op"] == "extend":
        return None                                        # whole numbers throughout
    s = prepare(case, seed)
    if case["op"] == "sample":
        token, prob, count = [], [], []
        for r in range(case["rows"]):
            z = s["logits"][r, :case["vocab"]].double().cpu().numpy()
            heat, k, p, least, u = (float(s[n][r]) for n in ("temperature", "top_k", "top_p", "min_p", "u"))
            rank = np.lexsort((np.arange(len(z)), -z))
            rank = rank[z[rank] > -np.inf]
            w = np.exp((z[rank] - z[rank[0]]) / (heat if heat > 0 else 1.0))
            n = 1 if heat <= 0 else int(k) if 0 < k < len(w) else len(w)
            if p < 1:
                total, mass, m = math.fsum(w[:n]), np.cumsum(w[:n]), 1
                m = 1 + int(np.searchsorted(mass[:-1], p * total, side="left")) if n > 1 else 1
                n = min(n, m)
            n = max(1, min(n, int((w >= least).sum())))
            by_index = np.argsort(rank[:n])
            sums = np.cumsum(w[:n][by_index])
            i = int(np.searchsorted(sums, u * sums[-1], side="right"))
            token.append(int(rank[:n][by_index][i]))
            prob.append(math.log(w[:n][by_index][i] / sums[-1]))
            count.append(n)
        return [torch.tensor(token, dtype=torch.int32), torch.tensor(prob, dtype=torch.float64), torch.tensor(count, dtype=torch.int32)]
    hq, hkv, d, new = case["q_heads"], case["kv_heads"], case["head_dim"], case["new"]
    kind = s["q"].dtype
    inv = [THETA ** (-2.0 * i / d) for i in range(d // 2)]
    angle = s["q_pos"].double()[:, None] * torch.tensor(inv, dtype=torch.float64, device=DEVICE)

    def turned(x):
        z = torch.complex(x[..., : d // 2].double(), x[..., d // 2:].double()) * torch.polar(torch.ones_like(angle), angle)[:, None]
        return torch.cat((z.real, z.imag), -1)
    q, k_rows = turned(s["q"]), turned(s["k_new"])
    k_pool, v_pool = s["k_pool"].double(), s["v_pool"].double()
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEVICE)
    segs, off, table = s["segs"].tolist(), s["req_seg_off"].tolist(), s["block_tab"].long()
    for j, slot in enumerate(s["slot_map"].tolist()):
        k_pool[slot // BLOCK, :, slot % BLOCK] = k_rows[j]
        v_pool[slot // BLOCK, :, :, slot % BLOCK] = s["v_new"][j].double()
    for r in range(case["requests"]):
        keys, values = [], []
        for _, _, _, n, tab, _, _, _ in segs[off[r]:off[r + 1]]:
            blocks = table[tab:tab + (n + BLOCK - 1) // BLOCK]
            keys.append(k_pool[blocks].transpose(1, 2).reshape(-1, hkv, d)[:n].to(kind).double())        # (the cache holds them in its type)
            values.append(v_pool[blocks].permute(0, 3, 1, 2).reshape(-1, hkv, d)[:n])
        keys, values = torch.cat(keys), torch.cat(values)
        pos = s["q_pos"][r * new:(r + 1) * new].long()
        hidden = torch.arange(len(keys), device=DEVICE)[None] > pos[:, None]
        for h in range(hq):
            z = q[r * new:(r + 1) * new, h] @ keys[:, h // (hq // hkv)].T / math.sqrt(d)
            p = torch.softmax(z.masked_fill(hidden, -math.inf), -1)
            out[r * new:(r + 1) * new, h] = p @ values[:, h // (hq // hkv)]
    return [out, k_pool, v_pool]
