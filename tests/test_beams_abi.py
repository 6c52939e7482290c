"""Host side of the beams: descriptions and arguments that are refused before anything is enqueued (no GPU needed)."""
import ctypes

import pytest
import torch

from test_pages_abi import ONE, good, rk  # noqa: F401

ODD = ctypes.c_void_p(257)


def beams(rk, **kw):
    base = dict(n_groups=3, n_beams=4, n_vocab=1000, n_out=8, dtype="f32")
    base.update(kw)
    return rk.make_beams(**base)


def select(rk, b, ws=ONE, ws_n=1 << 40, **over):
    a = dict(logits=ONE, scores=ONE, finished=None, new_scores=ctypes.c_void_p(512), parents=ONE, tokens=ONE, new_finished=None)
    a.update(over)
    return rk.lib().restkv_beam_select(ctypes.byref(b), *a.values(), ws, ws_n, None)


def layers(rk, n=2, k=256, v=256, ks=256, vs=256):
    return (rk.binding.RestkvLayerPages * max(n, 1))(*[(k, v, ks, vs)] * n)


def reorder(rk, c, n_beams=3, stride=0, n_layers=2, **over):
    a = dict(lens=ONE, table=ONE, table_out=ONE, layers=layers(rk))
    parents = over.pop("parents", ONE)
    a.update(over)
    return rk.lib().restkv_beam_reorder(ctypes.byref(c), n_beams, parents, stride, *a.values(), n_layers, None)


def attend(rk, c, n_beams=3, ws=ONE, ws_n=1 << 40, **over):
    a = dict(shared=ONE, q=ONE, kp=ONE, vp=ONE, ks=ONE, vs=ONE, table=ONE, lens=ONE, new_start=None, out=ONE, lse=None)
    a.update(over)
    return rk.lib().restkv_attend_beams(ctypes.byref(c), n_beams, *a.values(), ws, ws_n, None)


def test_layouts_match_header(rk):  # noqa: F811
    assert ctypes.sizeof(rk.RestkvBeams) == 6 * 4 + 8
    assert ctypes.sizeof(rk.binding.RestkvLayerPages) == 32


@pytest.mark.parametrize("kw,code", [
    (dict(n_groups=-1), -1), (dict(n_beams=0), -1), (dict(n_vocab=0), -1), (dict(n_out=0), -1), (dict(logit_stride=999), -1),
    (dict(logit_stride=-5), -1), (dict(n_groups=16385), -2), (dict(n_beams=65), -2), (dict(n_out=65), -2), (dict(n_vocab=(1 << 24) + 1), -2),
    (dict(dtype=4), -2), (dict(dtype=7), -2), (dict(logit_stride=(1 << 40) + 1), -2),
])
def test_select_descriptions_that_are_refused(rk, kw, code):  # noqa: F811
    b = beams(rk, **kw)
    assert select(rk, b) == code
    assert rk.restkv_beam_workspace_bytes(b) == 0


def test_select_arguments_that_are_refused(rk):  # noqa: F811
    b = beams(rk)
    for name in ("logits", "scores", "new_scores", "parents", "tokens"):
        assert select(rk, b, **{name: None}) == -1, name
    assert select(rk, b, logits=ctypes.c_void_p(258)) == -1            # float32 at an address that is none
    assert select(rk, beams(rk, dtype="bf16"), logits=ODD) == -1
    assert select(rk, b, new_scores=ONE) == -1                         # in place, but 8 of 4 beams
    assert select(rk, b, finished=ONE, new_finished=ONE) == -1
    need = rk.restkv_beam_workspace_bytes(b)
    assert need > 0
    assert select(rk, b, ws=None) == -3 and select(rk, b, ws_n=need - 1) == -3 and select(rk, b, ws=ctypes.c_void_p(264)) == -3
    none = beams(rk, n_groups=0)
    assert rk.restkv_beam_workspace_bytes(none) == 0
    assert select(rk, none, logits=None, scores=None, ws=None) == 0    # looks at no array
    assert rk.lib().restkv_beam_select(None, *[ONE] * 8, 0, None) == -1


def test_reorder_refusals(rk):  # noqa: F811
    c = good(rk)
    for n, code in ((0, -1), (-1, -1), (2, -1), (65, -2)):             # 3 sequences
        assert reorder(rk, c, n_beams=n) == code
        assert attend(rk, c, n_beams=n) == code
    for name in ("parents", "lens", "table", "table_out"):
        assert reorder(rk, c, **{name: None}) == -1, name
    assert reorder(rk, c, layers=None) == -1
    assert reorder(rk, c, stride=2) == -1 and reorder(rk, c, stride=-1) == -1
    assert reorder(rk, c, n_layers=-1) == -1 and reorder(rk, c, n_layers=257) == -2
    assert reorder(rk, c, layers=layers(rk, k=None)) == -1 and reorder(rk, c, layers=layers(rk, v=264)) == -1
    assert reorder(rk, good(rk, format="q4"), layers=layers(rk, ks=None)) == -1
    assert reorder(rk, good(rk, _table_stride_s=5)) == -1              # tables that overlap: 6 entries each
    assert reorder(rk, good(rk, _table_stride_s=6, _table_stride_h=6)) == -1
    assert reorder(rk, good(rk, _table_stride_s=12, _table_stride_h=5)) == -1
    assert reorder(rk, good(rk, head_dim=96)) == -2
    assert reorder(rk, good(rk, n_seqs=0), parents=None, lens=None, table=None, layers=None) == 0


def test_attend_beams_refusals(rk):  # noqa: F811
    c = good(rk)
    for name in ("shared", "q", "kp", "vp", "table", "lens", "out"):
        assert attend(rk, c, **{name: None}) == -1, name
    assert attend(rk, good(rk, format="q4"), ks=None) == -1
    assert attend(rk, good(rk, _out_stride_t=64)) == -1                # rows of out overlap
    assert rk.restkv_attend_beams_workspace_bytes(c, 2) == 0 and rk.restkv_attend_beams_workspace_bytes(c, 0) == 0
    big = good(rk, max_pages=600, n_pages=4000)
    need = rk.restkv_attend_beams_workspace_bytes(big, 3)
    assert need > 0
    assert attend(rk, big, ws=None) == -3 and attend(rk, big, ws_n=need - 1) == -3 and attend(rk, big, ws=ctypes.c_void_p(264)) == -3
    # short caches need what restkv_attend does, others (or all, where told so) more
    assert need == rk.restkv_attend_workspace_bytes(big)
    rk.restkv_debug_force_shared(True)
    more = rk.restkv_attend_beams_workspace_bytes(big, 3)
    assert more > need and attend(rk, big, ws_n=need) == -3
    rk.restkv_debug_force_shared(False)
    large = good(rk, max_pages=6000, n_pages=4000)
    assert rk.restkv_attend_beams_workspace_bytes(large, 3) != rk.restkv_attend_workspace_bytes(large)
    assert rk.restkv_attend_beams_workspace_bytes(large, 1) == rk.restkv_attend_workspace_bytes(large)
    assert attend(rk, good(rk, n_seqs=0), shared=None, q=None) == 0
    assert attend(rk, good(rk, n_tokens=0), new_start=ONE, shared=None, q=None) == 0


def test_binding_refuses_tensors_that_are_not_on_a_gpu(rk):  # noqa: F811
    b = beams(rk)
    f, i = torch.zeros(3, 8), torch.zeros(3, 8, dtype=torch.int32)
    with pytest.raises(rk.RestkvError):
        rk.restkv_beam_select(b, torch.zeros(12, 1000), torch.zeros(3, 4), f, i, i, None)
    c = good(rk, n_pages=2)
    k = torch.zeros(2, 2, 32, 64, dtype=torch.bfloat16)
    pages = rk.CachePages(k, k)
    table, lens = torch.zeros(3, 6, dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    with pytest.raises(rk.RestkvError):
        rk.restkv_beam_reorder(c, 3, torch.zeros(1, 3, dtype=torch.int32), table, lens, [pages])
    with pytest.raises(rk.RestkvError):
        rk.restkv_beam_reorder(c, 3, torch.zeros(1, 3, dtype=torch.int32), table, lens, [])
    q = torch.zeros(3, 4, 64, dtype=torch.bfloat16)
    with pytest.raises(rk.RestkvError):
        rk.restkv_attend_beams(c, 3, torch.zeros(1, dtype=torch.int32), q, pages, table, lens, torch.empty_like(q))
    with pytest.raises(rk.RestkvError):                                # layers of two layouts
        rk.CacheLayers([pages, rk.CachePages(k[:, :, :16], k[:, :, :16])])
