"""Host side of the paged cache: descriptions and arguments that are refused before anything is enqueued (no GPU needed)."""
import ctypes
import os

import pytest
import torch


@pytest.fixture(scope="module")
def rk():
    import paper_2605_08840_amd as r
    if not os.path.exists(r.LIB_PATH):
        import __graft_entry__
        __graft_entry__.build()
    return r


def good(rk, **kw):
    base = dict(n_seqs=3, n_q_heads=4, n_kv_heads=2, head_dim=64, page_size=32, n_pages=20, max_pages=6, dtype="bf16")
    base.update(kw)
    c = rk.make_cache(**{k: v for k, v in base.items() if not k.startswith("_")})
    for k, v in base.items():
        if k.startswith("_"):
            setattr(c, k[1:], v)
    return c


ONE = ctypes.c_void_p(256)            # never dereferenced on the host


def append(rk, c, **over):
    a = dict(k=ONE, v=ONE, kp=ONE, vp=ONE, ks=ONE, vs=ONE, table=ONE, lens=ONE, new_start=None, positions=None, cos=None, sin=None,
             q=None, q_out=None)
    a.update(over)
    return rk.lib().restkv_append(ctypes.byref(c), *a.values(), None)


def attend(rk, c, ws=ONE, ws_n=1 << 40, **over):
    a = dict(q=ONE, kp=ONE, vp=ONE, ks=ONE, vs=ONE, table=ONE, lens=ONE, new_start=None, out=ONE, lse=None)
    a.update(over)
    return rk.lib().restkv_attend(ctypes.byref(c), *a.values(), ws, ws_n, None)


def fetch(rk, c, first=0, n=8, **over):
    a = dict(kp=ONE, vp=ONE, ks=ONE, vs=ONE, table=ONE, lens=ONE, idx=None)
    a.update({k: v for k, v in over.items() if k in a})
    return rk.lib().restkv_fetch(ctypes.byref(c), *a.values(), first, n, over.get("k_out", ONE), over.get("v_out", ONE), None)


def test_description_layout_matches_header(rk):
    assert ctypes.sizeof(rk.RestkvCache) == 18 * 4 + 15 * 8


BAD = [
    (dict(n_seqs=-1), -1), (dict(n_q_heads=3), -1), (dict(n_q_heads=0), -1), (dict(n_kv_heads=0), -1), (dict(n_pages=0), -1),
    (dict(max_pages=0), -1), (dict(max_new=0), -1), (dict(n_tokens=-1), -1), (dict(max_len=-1), -1),
    (dict(max_len=6 * 32 + 1), -1),            # more than the table names
    (dict(scale=-1.0), -1), (dict(scale=float("inf")), -1), (dict(scale=float("nan")), -1),
    (dict(rotary_dim=80), -1), (dict(rotary_dim=-16), -1), (dict(rotary_dim=24), -2),
    (dict(head_dim=96), -2), (dict(dtype=7), -2), (dict(format="f32"), -2), (dict(dtype="f32", format="bf16"), -2),
    (dict(dtype="f32", out_dtype="bf16"), -2),
    (dict(page_size=8), -2), (dict(page_size=48), -2), (dict(page_size=1 << 17), -2), (dict(max_pages=1 << 26), -2),
    (dict(n_seqs=16385), -2), (dict(max_new=1 << 29), -2),
    (dict(page_strides=(64, 32, -1)), -1), (dict(page_strides=(0, 32, 1)), -1), (dict(page_strides=(64, -1, 1)), -1),
    (dict(page_strides=(1 << 20, 1, 65537)), -2),
    (dict(_token_stride=0), -1),               # the default layout with strides beside it
    (dict(_q_stride_t=63), -1), (dict(_kv_stride_h=-64), -1), (dict(_out_stride_h=8), -1), (dict(_lse_stride_t=-1), -1),
    (dict(_table_stride_s=-1), -1), (dict(_lens_stride_h=-1), -1),
]


@pytest.mark.parametrize("over,code", BAD, ids=lambda x: str(x))
def test_descriptions_that_are_refused(rk, over, code):
    c = good(rk, **over)
    assert append(rk, c) == code
    assert attend(rk, c) == code
    assert fetch(rk, c) == code
    assert rk.restkv_attend_workspace_bytes(c) == 0


def test_arguments_that_are_refused(rk):
    c, q4, turn = good(rk), good(rk, format="q4"), good(rk, rotary_dim=64, n_positions=10)
    odd = ctypes.c_void_p(264)
    for name in ("k", "v", "kp", "vp", "table", "lens"):
        assert append(rk, c, **{name: None}) == -1, name
    for name in ("q", "kp", "vp", "table", "lens", "out"):
        assert attend(rk, c, **{name: None}) == -1, name
    for name in ("kp", "vp", "table", "lens", "k_out", "v_out"):
        assert fetch(rk, c, **{name: None}) == -1, name
    for call in (append, attend, fetch):
        assert call(rk, q4, ks=None) == -1 and call(rk, q4, vs=None) == -1
        assert call(rk, c, kp=odd) == -1 and call(rk, q4, vs=odd) == -1
    assert append(rk, c, q=ONE) == -1 and append(rk, c, q_out=ONE) == -1
    assert append(rk, turn) == -1 and append(rk, turn, cos=ONE) == -1 and append(rk, good(rk, rotary_dim=64), cos=ONE, sin=ONE) == -1
    # cache positions are no positions where every head has its own
    assert append(rk, good(rk, rotary_dim=64, n_positions=10, head_lens=True), cos=ONE, sin=ONE) == -1
    # without new_start every sequence has max_new tokens
    short = good(rk, n_tokens=5, max_new=2)
    assert append(rk, short) == -1 and attend(rk, short) == -1
    assert fetch(rk, c, k_out=odd) == -1 and fetch(rk, c, first=-1) == -1 and fetch(rk, c, n=-1) == -1
    assert fetch(rk, c, n=(1 << 30) + 1) == -2
    # workspace: missing, too small, misaligned
    need = rk.restkv_attend_workspace_bytes(good(rk, max_pages=600, n_pages=900))
    long = good(rk, max_pages=600, n_pages=900)
    assert need > 0
    assert attend(rk, long, ws=None) == -3 and attend(rk, long, ws_n=need - 1) == -3 and attend(rk, long, ws=odd, ws_n=need) == -3


def test_nothing_to_do_is_no_error(rk):
    for c in (good(rk, n_seqs=0), good(rk, n_tokens=0, n_seqs=0)):
        assert append(rk, c) == 0 and attend(rk, c, ws=None, ws_n=0) == 0 and fetch(rk, c) == 0
    assert append(rk, good(rk, n_tokens=0), new_start=ONE) == 0 and attend(rk, good(rk, n_tokens=0), new_start=ONE) == 0
    assert fetch(rk, good(rk), n=0) == 0


def test_short_caches_need_no_workspace(rk):
    assert rk.restkv_attend_workspace_bytes(good(rk, page_size=64, max_pages=100, n_pages=400, max_len=128)) == 0
    assert rk.alloc_attend_workspace(good(rk, max_len=100), device="cpu") is None
    # bounded however large the batch of row blocks is
    big = good(rk, n_seqs=48, n_q_heads=64, n_kv_heads=8, head_dim=128, max_pages=4096, n_pages=1 << 17, max_new=64)
    assert 0 < rk.restkv_attend_workspace_bytes(big) < 1 << 28


def test_binding_refuses_tensors_that_are_not_what_they_are_said_to_be(rk):
    c = good(rk)
    pages = rk.alloc_cache_pages(c, device="cpu")
    assert pages.k.shape == (20, 2, 32, 64) and rk.alloc_cache_pages(good(rk, token_major=True), device="cpu").k.shape == (20, 32, 2, 64)
    assert rk.alloc_cache_pages(good(rk, head_tables=True), device="cpu").k.shape == (20, 1, 32, 64)
    q4 = rk.alloc_cache_pages(good(rk, format="q4"), device="cpu")
    assert q4.k.shape == (20, 2, 32, 32) and q4.k_scale.shape == (20, 2, 32, 2, 2)
    x = torch.zeros(3, 2, 64, dtype=torch.bfloat16)
    table, lens = torch.zeros(3, 6, dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    with pytest.raises(rk.RestkvError, match="not on a GPU"):
        rk.restkv_append(c, x, x, pages, table, lens)
    for other in (dict(n_kv_heads=1), dict(page_size=64), dict(n_pages=21), dict(head_dim=128), dict(format="q4"),
                  dict(dtype="f32"), dict(token_major=True), dict(head_tables=True), dict(page_strides=(128, 32, 1))):
        with pytest.raises(rk.RestkvError, match="are not the described ones"):
            rk.restkv_append(good(rk, **other), x, x, pages, table, lens)
    k, s = q4.k, q4.k_scale
    for bad in ((k, k), (k, k, s, None), (k, k[..., :16], s, s), (k, k, s[..., :1], s[..., :1]), (k, k.transpose(1, 2), s, s),
                (k[0], k[0], s, s), (k, k, s.float(), s.float()), (pages.k, pages.v, s, s), (pages.k, pages.v.float()),
                (pages.k[..., ::2], pages.v[..., ::2]), (k, k, s.transpose(3, 4), s)):
        with pytest.raises(rk.RestkvError):
            rk.CachePages(*bad)


def test_an_empty_call_needs_no_arrays(rk):
    """No sequence, no token or no row: tensors without an element have no address."""
    none = dict(kp=None, vp=None, ks=None, vs=None, table=None, lens=None)
    for c in (good(rk, n_seqs=0), good(rk, n_seqs=0, n_tokens=0, format="q4"), good(rk, n_seqs=0, rotary_dim=64)):
        assert append(rk, c, k=None, v=None, **none) == 0
        assert attend(rk, c, ws=None, ws_n=0, q=None, out=None, **none) == 0
        assert fetch(rk, c, k_out=None, v_out=None, **none) == 0
    c = good(rk, n_tokens=0)
    assert append(rk, c, k=None, v=None, new_start=ONE) == 0 and attend(rk, c, ws=None, ws_n=0, q=None, out=None, new_start=ONE) == 0
    assert fetch(rk, good(rk), n=0, k_out=None, v_out=None) == 0
    assert fetch(rk, good(rk, n_seqs=0), n=-1) == -1 and append(rk, good(rk, n_seqs=0, head_dim=96)) == -2


def test_scales_whose_logits_pass_float32_are_refused(rk):
    assert attend(rk, good(rk, scale=3e38)) == -1


def test_binding_asks_for_all_entries_that_are_read(rk):
    told = rk.binding._Told
    assert told(good(rk)).n_table == 3 * 6 and told(good(rk)).n_lens == 3
    assert told(good(rk, head_tables=True, head_lens=True)).n_table == 3 * 2 * 6
    assert told(good(rk, head_tables=True, head_lens=True)).n_lens == 3 * 2
    assert told(good(rk, _table_stride_s=0, _lens_stride_s=0)).n_table == 3 * 6                     # the library's defaults
    assert told(good(rk, _table_stride_s=0, _lens_stride_s=0)).n_lens == 3
    assert told(good(rk, _table_stride_s=1)).n_table == 2 + 6                                       # rows that overlap
    assert told(good(rk, _table_stride_s=6, _table_stride_h=18)).n_table == 12 + 18 + 6              # heads outermost
    assert told(good(rk, _lens_stride_s=1, _lens_stride_h=3)).n_lens == 2 + 3 + 1
    assert told(good(rk, n_seqs=0)).n_table == 0 and told(good(rk, n_seqs=0)).n_lens == 0


def test_binding_knows_pages_by_their_head_stride(rk):
    x, table, lens = torch.zeros(3, 2, 64, dtype=torch.bfloat16), torch.zeros(3, 2, 6, dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    one, both = (rk.alloc_cache_pages(good(rk, head_tables=h), device="cpu") for h in (True, False))
    # tables per head over pages of one head that are said to be a head apart: rows behind the array
    apart = good(rk, head_tables=True, page_strides=(64, 32, 1))
    with pytest.raises(rk.RestkvError, match="are not the described ones"):
        rk.restkv_append(apart, x, x, one, table, lens)
    for c, pages in ((apart, both), (good(rk, head_tables=True), one),
                     (good(rk, _page_stride=0, _head_stride=0, _token_stride=0), both)):
        with pytest.raises(rk.RestkvError, match="not on a GPU"):
            rk.restkv_append(c, x, x, pages, table, lens)


def test_queries_of_more_threads_than_a_launch_takes_are_refused(rk):
    for n, fmt in ((1 << 28, None), (1 << 28, "q4"), (1 << 30, None)):
        assert attend(rk, good(rk, n_seqs=1, n_q_heads=1, n_kv_heads=1, max_new=n, n_tokens=n, format=fmt)) == -2


def test_a_call_without_a_token_does_nothing_with_or_without_new_start(rk):
    none = dict(kp=None, vp=None, ks=None, vs=None, table=None, lens=None)
    for c in (good(rk, n_tokens=0), good(rk, n_tokens=0, format="q4", max_new=7), good(rk, n_tokens=0, rotary_dim=64)):
        for start in (None, ONE):
            assert append(rk, c, k=None, v=None, new_start=start, **none) == 0
            assert attend(rk, c, ws=None, ws_n=0, q=None, out=None, new_start=start, **none) == 0
    assert append(rk, good(rk, n_tokens=2)) == -1 and attend(rk, good(rk, n_tokens=2)) == -1


@pytest.fixture
def checks_only(rk, monkeypatch):
    """The binding's checks of CPU tensors, with nothing behind them."""
    monkeypatch.setattr(rk.binding, "_check_pages", lambda *a: -1)
    monkeypatch.setattr(rk.binding, "_on_gpu", lambda *a: None)
    return rk


def i32(*shape):
    return torch.zeros(shape, dtype=torch.int32)


def calls_of(rk, c):
    """The three calls with tensors as described, of which a case exchanges some."""
    pages = rk.CachePages(*(torch.zeros(20, 2, 32, 64, dtype=torch.bfloat16) for _ in range(2)))
    n = c.n_tokens
    q, kv = torch.zeros(n, 4, 64, dtype=torch.bfloat16), torch.zeros(n, 2, 64, dtype=torch.bfloat16)
    rows = torch.zeros(c.n_seqs, 2, 5, 64, dtype=torch.bfloat16)

    def go(**over):
        t = dict(table=i32(c.n_seqs, 6), lens=i32(c.n_seqs), new_start=None, positions=None, cos=torch.zeros(40, 16), sin=torch.zeros(40, 16), idx=None)
        t.update(over)
        turns = {x: t[x] for x in ("positions", "cos", "sin")}
        rk.restkv_append(c, kv, kv, pages, t["table"], t["lens"], new_start=t["new_start"], q=q, q_out=q, **turns)
        if not {"positions", "cos", "sin", "idx"} & set(over):
            rk.restkv_attend(c, q, pages, t["table"], t["lens"], q.clone(), new_start=t["new_start"])
        if not {"positions", "cos", "sin", "new_start"} & set(over):
            rk.restkv_fetch(c, pages, t["table"], t["lens"], rows, rows.clone(), idx=t["idx"])
    return go


def test_binding_takes_arrays_of_the_described_shape(checks_only):
    rk = checks_only
    c = good(rk, rotary_dim=32, n_positions=40, max_new=2)
    go = calls_of(rk, c)
    go()
    # what is read of these is what is meant: more rows than are used, dimensions of one, one row after the other
    for fine in (dict(table=i32(9, 6)), dict(table=i32(3, 1, 6)), dict(table=i32(18)), dict(lens=i32(7)), dict(lens=i32(3, 1)),
                 dict(new_start=i32(4)), dict(new_start=i32(9)), dict(positions=i32(6)), dict(positions=i32(1, 6)), dict(positions=i32(3, 2)),
                 dict(cos=torch.zeros(99, 16), sin=torch.zeros(40, 1, 16)), dict(idx=i32(3, 2, 5)), dict(idx=i32(30))):
        go(**fine)
    for wrong in (dict(table=i32(3, 8)), dict(table=i32(6, 6).t()), dict(table=i32(6, 3)), dict(table=i32(3, 2, 6)), dict(table=i32(19)),
                  dict(lens=i32(3, 2)), dict(lens=i32(2, 3)), dict(new_start=i32(2, 2)), dict(positions=i32(7)), dict(positions=i32(2, 3)),
                  dict(positions=i32(3, 2), new_start=i32(4)), dict(cos=torch.zeros(40, 32)), dict(sin=torch.zeros(40, 32)), dict(cos=torch.zeros(16, 40)),
                  dict(idx=i32(3, 2, 6)), dict(idx=i32(2, 3, 5)), dict(idx=i32(4, 2, 5)), dict(idx=i32(31))):
        with pytest.raises(rk.RestkvError, match="has to be"):
            go(**wrong)


def test_binding_takes_arrays_of_one_sequence_and_by_head(checks_only):
    rk = checks_only
    go = calls_of(rk, good(rk, n_seqs=1, rotary_dim=32, n_positions=40))
    for fine in (dict(table=i32(6)), dict(table=i32(4, 6)), dict(lens=i32(1)), dict(lens=i32(1, 1)), dict(idx=i32(2, 5)), dict(positions=i32(1, 1))):
        go(**fine)
    for wrong in (dict(table=i32(1, 8)), dict(lens=i32(1, 2)), dict(idx=i32(2, 6)), dict(idx=i32(5, 2))):
        with pytest.raises(rk.RestkvError, match="has to be"):
            go(**wrong)
    c = good(rk, rotary_dim=32, n_positions=40, head_lens=True, head_tables=True)
    go = calls_of(rk, c)
    go(table=i32(3, 2, 6), lens=i32(3, 2))
    go(table=i32(5, 2, 6), lens=i32(4, 2))
    for wrong in (dict(table=i32(3, 6)), dict(table=i32(2, 3, 6)), dict(table=i32(3, 2, 8)), dict(lens=i32(6, 3)), dict(lens=i32(2, 3))):
        with pytest.raises(rk.RestkvError, match="has to be"):
            go(**{**dict(table=i32(3, 2, 6), lens=i32(3, 2)), **wrong})
    # strides set by hand: as many entries as are read
    c = good(rk, rotary_dim=32, n_positions=40, _table_stride_s=8, _lens_stride_s=2)
    go = calls_of(rk, c)
    go(table=i32(3, 8), lens=i32(3, 2))
    go(table=i32(22), lens=i32(5))
    for wrong in (dict(table=i32(21)), dict(lens=i32(4))):
        with pytest.raises(rk.RestkvError, match="has to be"):
            go(**{**dict(table=i32(3, 8), lens=i32(3, 2)), **wrong})


def test_outputs_whose_rows_overlap_are_refused(rk):
    """Rows of different tokens and heads at the same place: each would hold what was written last."""
    def out(t, h, **kw):          # past the strides a call without its workspace is refused for that
        c = good(rk, max_pages=600, n_pages=900, _out_stride_t=t, _out_stride_h=h, **kw)
        return attend(rk, c, ws=None)

    def lse(t, h):
        return attend(rk, good(rk, max_pages=600, n_pages=900, _lse_stride_t=t, _lse_stride_h=h), ws=None, lse=ONE)

    # 3 tokens, 4 heads: tokens outermost, heads outermost, gaps, rows that interleave
    for t, h in ((256, 64), (300, 70), (64, 192), (70, 300), (128, 384), (512, 128), (64, 200), (448, 128)):
        assert out(t, h) == -3, (t, h)
    for t, h in ((128, 64), (192, 64), (64, 64), (64, 128), (255, 64), (64, 191), (100, 130), (65, 66), (384, 192)):
        assert out(t, h) == -1, (t, h)
    assert out(64, 100, n_q_heads=2) == -1 and out(64, 200, n_q_heads=2) == -3
    for t, h in ((4, 1), (1, 3), (7, 2), (2, 7)):
        assert lse(t, h) == -3, (t, h)
    for t, h in ((3, 1), (1, 2), (1, 1), (2, 4)):
        assert lse(t, h) == -1, (t, h)
    # a single token or head; strides of a log-sum-exp that is not asked for
    assert out(64, 64, n_seqs=1) == -3 and out(64, 64, n_q_heads=1, n_kv_heads=1) == -3
    assert attend(rk, good(rk, max_pages=600, n_pages=900, _lse_stride_t=1), ws=None) == -3
    # rotated queries; queries that are only read may overlap
    assert append(rk, good(rk, _q_stride_t=128), q=ONE, q_out=ONE) == -1
    assert attend(rk, good(rk, max_pages=600, n_pages=900, _q_stride_t=128), ws=None) == -3
