"""Descriptions that a program makes and drops, one for each batch or step, are freed with what the binding has worked out from them (no GPU needed)."""
import gc
import weakref

import torch

from test_pages_abi import good, rk  # noqa: F401


def refused(rk, f, *args, **kw):  # noqa: F811
    try:
        f(*args, **kw)
    except rk.RestkvError:
        return
    raise AssertionError("not refused")


def freed(rk, make, use):  # noqa: F811
    left = []
    for _ in range(50):
        x = make()
        use(x)
        assert "told" in x.__dict__
        left.append(weakref.ref(x))
        del x
    gc.collect()
    return all(r() is None for r in left)


def test_descriptions_of_a_cache_are_freed(rk):  # noqa: F811
    k = torch.zeros(20, 2, 32, 64, dtype=torch.bfloat16)
    pages = rk.CachePages(k, k)
    table, lens, q = torch.zeros(3, 6, dtype=torch.int32), torch.zeros(3, dtype=torch.int32), torch.zeros(3, 4, 64, dtype=torch.bfloat16)
    kv, shared = q[:, :2], torch.zeros(1, dtype=torch.int32)
    for use in (lambda c: refused(rk, rk.restkv_attend, c, q, pages, table, lens, q),
                lambda c: refused(rk, rk.restkv_append, c, kv, kv, pages, table, lens),
                lambda c: refused(rk, rk.restkv_fetch, c, pages, table, lens, k, k),
                lambda c: refused(rk, rk.restkv_beam_reorder, c, 3, shared.view(1, 1), table, lens, [pages]),
                lambda c: refused(rk, rk.restkv_attend_beams, c, 3, shared, q, pages, table, lens, q)):
        assert freed(rk, lambda: good(rk), use)


def test_descriptions_of_beams_are_freed(rk):  # noqa: F811
    f, i = torch.zeros(3, 8), torch.zeros(3, 8, dtype=torch.int32)
    assert freed(rk, lambda: rk.make_beams(n_groups=3, n_beams=4, n_vocab=1000, n_out=8, dtype="f32"),
                 lambda b: refused(rk, rk.restkv_beam_select, b, torch.zeros(12, 1000), torch.zeros(3, 4), f, i, i, None))


def test_descriptions_of_beams_are_freed_without_a_collection(rk):  # noqa: F811
    """At once, not when the collector comes by: nothing refers to itself."""
    gc.collect()
    gc.disable()
    try:
        f, i = torch.zeros(3, 8), torch.zeros(3, 8, dtype=torch.int32)
        b = rk.make_beams(n_groups=3, n_beams=4, n_vocab=1000, n_out=8, dtype="f32")
        refused(rk, rk.restkv_beam_select, b, torch.zeros(12, 1000), torch.zeros(3, 4), f, i, i, None)
        r = weakref.ref(b)
        del b
        assert r() is None
    finally:
        gc.enable()
