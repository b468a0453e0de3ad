"""The answer's operators without a GPU: the oracle on examples worked by hand, and what the calls refuse."""
import ctypes as C
import math

import numpy as np
import pytest

from oracle import answer_oracle as A


@pytest.fixture(scope="module")
def lib():
    import os
    import paper_2502_15734_amd as P
    if not os.path.exists(P.library_path()):
        from paper_2502_15734_amd import build
        build.build(verbose=False)
    return P.load_library()


def _segs(rows):
    """(request, kind, tokens, table offset) -> segment table"""
    return np.array([[r, k, 0, n, tab, 0, 0, 0] for r, k, n, tab in rows], dtype=np.int32)


def test_tables_of_two_prompts_by_hand():
    # request 0: 20 cached tokens, a question of 16 that gets 3 more; request 1: nothing yet, 5 tokens
    segs = _segs([(0, 0, 20, 0), (0, 1, 16, 2), (1, 1, 0, 5)])
    out = A.extend_segments(segs, [0, 3, 5], [2, 3, 1], [0, 2, 3], [50, 51, 52], [7, 8, 9, -1, -1, -1], 100, 10)
    segs2, tab, cu, pos, slot, req, last, status, counts = out
    assert tab.tolist() == [7, 8, 9, 50, -1, 51] and cu.tolist() == [0, 3, 8]
    assert pos.tolist() == [36, 37, 38, 0, 1, 2, 3, 4, 0, 0]
    assert slot.tolist() == [800, 801, 802, 816, 817, 818, 819, 820, -1, -1]
    assert req.tolist() == [0, 0, 0, 1, 1, 1, 1, 1, -1, -1] and last.tolist() == [2, 7]
    assert status.tolist() == [0, 0] and counts.tolist() == [8, 2, 0, 44]
    assert segs2[:, 2].tolist() == [0, 20, 0] and segs2[:, 3].tolist() == [20, 19, 5] and segs2[:, 5].tolist() == [0, 3, 5]
    assert segs2[:, 6].tolist() == [0, 20, 39] and segs2[:, 7].tolist() == [0, 0, 3]


def test_refusals_of_requests_by_hand():
    # 0: needs two pages of three; 1: table full; 2: grows in front of cached tokens; 3: needs two pages, none left; 4: needs no page; 5: rows
    segs = _segs([(0, 1, 0, 0), (1, 1, 16, 2), (2, 0, 4, 3), (2, 1, 4, 4), (3, 1, 0, 5), (4, 1, 3, 7), (5, 1, 3, 8)])
    out = A.extend_segments(segs, [17, 1, 1, 0, 32, 2, 9], [2, 1, 1, 1, 2, 1, 1], [0, 1, 2, 4, 5, 6, 7], [3, 4, 5], np.zeros(9, int), 9, 52)
    assert out[7].tolist() == [A.OK, A.TABLE_FULL, A.ORDER, A.NO_PAGES, A.OK, A.NO_ROWS]
    assert out[8].tolist() == [19, 2, 4, 49] and out[2].tolist() == [0, 17, 17, 17, 17, 19, 19] and out[6].tolist() == [16, -1, -1, -1, 18, -1]


def test_sampling_by_hand():
    z = [0.0, math.log(4), math.log(2), math.log(4), -math.inf]            # weights 1, 4, 2, 4 -> order 1, 3, 2, 0
    assert A.sample(z, 1, 0, 1, 0, 0.0) == (0, pytest.approx(math.log(1 / 11)), 4)
    assert [A.sample(z, 1, 0, 1, 0, u)[0] for u in (0.5 / 11, 1.5 / 11, 5.5 / 11, 7.5 / 11)] == [0, 1, 2, 3]
    assert A.sample(z, 1, 1, 1, 0, 0.99)[0] == 1 and A.sample(z, 0, 0, 1, 0, 0.99) == (1, 0.0, 1)
    assert A.sample(z, 1, 2, 1, 0, 0.99)[::2] == (3, 2) and A.sample(z, 1, 3, 1, 0, 0.99)[2] == 3
    assert A.sample(z, 1, 0, 4 / 11, 0, 0.99)[2] in (1, 2) and A.sample(z, 1, 0, 0.37, 0, 0.99)[2] == 2
    assert A.sample(z, 1, 0, 0.0, 0, 0.99)[2] == 1 and A.sample(z, 1, 0, 1, 0.51, 0.99)[2] == 2 and A.sample(z, 1, 0, 1, 2.0, 0.99)[2] == 1
    assert A.sample([-math.inf, math.nan], 1, 0, 1, 0, 0.5)[::2] == (-1, 0)
    assert A.sample([1.0, math.inf, math.inf], 1, 0, 1, 0, 0.6) == (2, pytest.approx(math.log(0.5)), 3)


def test_attention_by_hand():
    k = np.zeros((2, 1, 16, 64)); v = np.zeros((2, 1, 64, 16))
    k[1, 0, 0, 0], v[1, 0, :, 0] = 8 * math.log(3), 1.0                       # (1 / sqrt 64 = 1 / 8)
    v[1, 0, :, 1] = 5.0
    segs = np.array([[0, 1, 0, 2, 0, 0, 0, 0]])
    pos, keys, values = A.paged_context(k, v, lambda b: v[b], [1], segs, range(1))
    q = np.zeros((2, 1, 64)); q[:, 0, 0] = 1.0
    out, lse, *_ = A.attend(A.rotate(q, [0, -1], 1e4), [0, 1], pos, keys, values, 1e4, 0.0)
    assert np.allclose(out[0], 1.0) and np.allclose(out[1], (3 * 1 + 5) / 4) and np.allclose(lse[:, 0], [math.log(3), math.log(4)])


def test_refused_arguments(lib):
    import paper_2502_15734_amd as P
    ctx = P.Context(8, 2, 128, 5.0e5, P.CC_BF16)
    h, good, odd = ctx._h, C.c_void_p(4096), C.c_void_p(4100)
    assert lib.cc_extend_segments_workspace_bytes(None, 3, 2) == 0 and lib.cc_extend_segments_workspace_bytes(h, -1, 2) == 0
    ws = lib.cc_extend_segments_workspace_bytes(h, 3, 2)
    ok = dict(segs_in=good, n_new=good, tab_cap=good, n_segs=3, off=good, n_requests=2, free=good, n_free=4, tab=good, n_tab=9, n_blocks=8,
              segs=good, cu=good, pos=good, slot=good, req=good, max_rows=5, last=good, status=good, counts=good, ws=good, bytes=ws, stream=None)
    call = lambda **k: lib.cc_extend_segments(h, *{**ok, **k}.values())
    for bad, status in ((dict(n_segs=-1), -1), (dict(n_segs=65536), -1), (dict(max_rows=-1), -1), (dict(n_blocks=1 << 27), -1), (dict(segs_in=None), -1),
                        (dict(segs=None), -1), (dict(off=None), -1), (dict(free=None), -1), (dict(tab=None), -1), (dict(pos=None), -1),
                        (dict(counts=None), -1), (dict(segs=odd), -1), (dict(ws=None), -1), (dict(ws=odd), -1), (dict(bytes=ws - 1), -3)):
        assert call(**bad) == status, bad
        assert b"cc_extend_segments" in lib.cc_last_error(h)
    assert call(n_requests=0) == 0

    need = lib.cc_append_attention_workspace_bytes(h, 10, 2, 5, 4000, 7)
    ok2 = dict(q=good, k=good, v=good, rows=None, pos=good, slot=good, cu=good, n=10, most=2, kp=good, vp=good, nb=8, tab=good, segs=good, n_segs=9,
               off=good, n_requests=5, ctx=4000, per=7, shared=None, out=C.c_void_p(8192), lse=None, ws=good, bytes=max(need, 1), stream=None)
    call = lambda **k: lib.cc_append_attention(h, *{**ok2, **k}.values())
    from paper_2502_15734_amd.binding import SharedValues
    for bad, status in ((dict(n=-1), -1), (dict(most=11), -1), (dict(q=None), -1), (dict(k=None), -1), (dict(out=None), -1), (dict(cu=None), -1),
                        (dict(nb=0), -1), (dict(n_requests=0), -1), (dict(ctx=0), -1), (dict(per=0), -1), (dict(n_requests=65536), -1),
                        (dict(nb=1 << 27), -1), (dict(q=odd), -1), (dict(kp=odd), -1), (dict(out=good), -1),
                        (dict(shared=C.byref(SharedValues(4096, 8, None))), -1)):
        assert call(**bad) == status, bad
        assert len(lib.cc_last_error(h)) > 0
    assert call(n=0, most=0) == 0
    if need:
        assert call(bytes=need - 1) == -3 and call(ws=None) == -1 and call(ws=odd) == -1

    need = lib.cc_sample_workspace_bytes(h, 4, 1000)
    ok3 = dict(z=good, dtype=1, n=4, vocab=1000, stride=1000, t=None, k=None, p=None, m=None, u=good, token=good, lp=None, kept=None, ws=good,
               bytes=max(need, 1), stream=None)
    call = lambda **k: lib.cc_sample(h, *{**ok3, **k}.values())
    for bad, status in ((dict(n=-1), -1), (dict(n=65536), -1), (dict(vocab=0), -1), (dict(stride=999), -1), (dict(vocab=(1 << 22) + 1, stride=1 << 23), -1),
                        (dict(dtype=2), -2), (dict(z=None), -1), (dict(u=None), -1), (dict(token=None), -1), (dict(z=odd), -1)):
        assert call(**bad) == status, bad
        assert b"cc_sample" in lib.cc_last_error(h)
    assert call(n=0) == 0
    if need:
        assert call(bytes=need - 1) == -3 and call(ws=None) == -1 and call(ws=odd) == -1
    ctx.close()


def test_calls_beyond_the_grid_are_refused(lib):
    """Rows and workgroups that a launch could not count are refused, not cut off."""
    import paper_2502_15734_amd as P
    ctx = P.Context(8, 2, 128, 5.0e5, P.CC_BF16)
    h, good = ctx._h, C.c_void_p(4096)
    assert lib.cc_extend_segments(h, good, good, good, 1, good, 1, good, 4, good, 9, 8, good, good, good, good, good, (1 << 30) + 1, good, good, good,
                                  good, 1 << 30, None) == -1 and b"2^30 rows" in lib.cc_last_error(h)
    # 65535 requests of up to 2^17 rows: 2 KV heads x 2^17 x 4 / 128 column groups each
    assert lib.cc_append_attention(h, good, good, good, None, good, good, good, 1 << 18, 1 << 17, good, good, 8, good, good, 65535, good, 65535, 4000, 1,
                                   None, C.c_void_p(8192), None, good, 1 << 60, None) == -1 and b"2^24 - 1 workgroups" in lib.cc_last_error(h)
    ctx.close()


def test_refused_workspaces_of_rows_in_parts(lib):
    """cc_sample over a vocabulary whose rows are read in parts (those that one workgroup holds need no workspace)."""
    import paper_2502_15734_amd as P
    ctx = P.Context(8, 2, 128, 5.0e5, P.CC_BF16)
    h, good, odd = ctx._h, C.c_void_p(4096), C.c_void_p(4100)
    need = lib.cc_sample_workspace_bytes(h, 4, 32000)
    assert need > 0 and 2 * need - 256 <= lib.cc_sample_workspace_bytes(h, 8, 32000) <= 2 * need and lib.cc_sample_workspace_bytes(None, 4, 32000) == 0
    call = lambda ws, n: lib.cc_sample(h, good, 0, 4, 32000, 32000, None, None, None, None, good, good, None, None, ws, n, None)
    for ws, n, status in ((None, need, -1), (odd, need, -1), (good, need - 1, -3), (good, 0, -3)):
        assert call(ws, n) == status and b"cc_sample" in lib.cc_last_error(h)
    ctx.close()


def test_refused_arguments_of_an_empty_batch(lib):
    import paper_2502_15734_amd as P
    ctx = P.Context(8, 2, 128, 5.0e5, P.CC_BF16)
    h, good = ctx._h, C.c_void_p(4096)
    assert lib.cc_extend_segments_workspace_bytes(h, 0, 0) == 0
    for lacking in ("cu", "counts", "pos", "slot", "req"):
        p = {k: None if k == lacking else good for k in ("cu", "pos", "slot", "req", "counts")}
        assert lib.cc_extend_segments(h, None, None, None, 0, None, 0, None, 0, None, 0, 8, None, p["cu"], p["pos"], p["slot"], p["req"], 5, None, None,
                                      p["counts"], None, 0, None) == -1 and b"cc_extend_segments" in lib.cc_last_error(h)
    ctx.close()


def test_row_lists_beyond_the_grid_are_refused(lib):
    """Lists whose rows, or whose parts to join, a launch could not count."""
    import paper_2502_15734_amd as P
    ctx = P.Context(8, 2, 128, 5.0e5, P.CC_BF16)
    h, good = ctx._h, C.c_void_p(4096)
    call = lambda n, tokens: lib.cc_append_attention(h, good, good, good, None, good, good, good, n, 1, good, good, 8, good, good, 1, good, 1, tokens, 1, None,
                                                     C.c_void_p(8192), None, good, (1 << 63) - 1, None)
    for impl, n, tokens in ((P.CC_IMPL_AUTO, 1 << 21, 16000),         # 2^24 rows and heads in 125 ranges: a workgroup each
                            (P.CC_IMPL_AUTO, 1 << 24, 300),           # 2^27 in two or three: one for eight
                            (P.CC_IMPL_AUTO, 1 << 26, 100),           # 2^26 rows to write: one for four
                            (P.CC_IMPL_SCALAR, 1 << 26, 100)):
        ctx.set_impl(impl)
        assert call(n, tokens) == -1 and b"2^24 - 1 workgroups" in lib.cc_last_error(h), (impl, n)
    ctx.close()
    one = P.Context(1, 1, 128, 5.0e5, P.CC_BF16)
    assert lib.cc_append_attention(one._h, good, good, good, None, good, good, good, (1 << 31) - 1, 1, good, good, 8, good, good, 1, good, 1, 100, 1, None,
                                   C.c_void_p(8192), None, good, (1 << 63) - 1, None) == -1 and b"2^24 - 1 workgroups" in lib.cc_last_error(one._h)
    one.close()


def test_sample_refuses_tensors_of_other_types(lib):
    """Numbers of 64 bits, numpy's own, would be read as others."""
    import torch
    import paper_2502_15734_amd as P
    ctx = P.Context(8, 2, 128, 5.0e5, P.CC_BF16)
    f, i = torch.zeros(4), torch.zeros(4, dtype=torch.int32)
    ok = dict(u=f, token=i, temperature=f, top_k=i, top_p=f, min_p=f, logprob=f, n_kept=i)
    for name, t in ok.items():
        for bad in (t.double(), t.long(), t[:3]):
            with pytest.raises(ValueError, match="fewer entries"):
                ctx.sample(torch.zeros(4, 8), 8, **{**ok, name: bad})
    ctx.close()
