"""How restkv_attend_beams sizes its list of chunks, on the host (no GPU needed): whatever the lengths, the chunks fit the workspace."""
import random

import pytest

from test_pages_abi import rk  # noqa: F401

MOST = 1 << 24            # tiles of 64 positions of the longest cache there may be


def cache(rk, n_seqs, fmt="f32", **kw):  # noqa: F811
    base = dict(n_seqs=n_seqs, n_q_heads=1, n_kv_heads=1, head_dim=64, page_size=65536, n_pages=100, max_pages=16384,
                dtype="bf16" if fmt == "q4" else fmt, format=fmt)
    base.update(kw)
    return rk.make_cache(**base)


def check(rk, c, n_beams, tiles):  # noqa: F811
    fronts, room, own, own_room = rk.restkv_debug_beams_list(c, n_beams, tiles)
    at = len(tiles) * n_beams // (n_beams + 1)             # (so many entries of sequences behind those of groups)
    used = [sum(t > 0 for t in x) for x in (tiles[:len(tiles) - at], tiles[len(tiles) - at:])]
    assert used[0] <= fronts <= room and used[1] <= own <= own_room, (n_beams, fronts, room, own, own_room)
    return fronts, own


FORMATS = ["f32", "bf16", "q4"]


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("groups", [40, 550, 2000, 8192])
def test_longest_caches(rk, groups, fmt):  # noqa: F811
    """2^30 positions each (pages may be shared, so memory does not rule that out)."""
    c = cache(rk, 2 * groups, fmt)
    check(rk, c, 2, [MOST] * groups + [0] * (2 * groups))
    check(rk, c, 2, [0] * groups + [MOST] * (2 * groups))
    check(rk, c, 2, [MOST - 7] * groups + [7] * (2 * groups))
    check(rk, c, 2, [MOST // 2 + 1] * groups + [MOST // 2 - 1] * (2 * groups))
    check(rk, c, 2, [0] * groups + [1] * (2 * groups - 1) + [MOST])
    check(rk, c, 2, [0] * (3 * groups))


@pytest.mark.parametrize("fmt", FORMATS)
def test_lengths_of_all_sizes(rk, fmt):  # noqa: F811
    r = random.Random(5)
    for _ in range(150):
        n_beams, new, hq, heads = r.choice([2, 3, 8, 33, 64]), r.choice([1, 2, 17]), r.choice([1, 4]), r.choice([1, 2, 8, 600])
        per_head = r.random() < 0.3 and heads <= 8
        groups = r.randint(33, min(700, 16384 // n_beams))
        c = cache(rk, groups * n_beams, fmt, n_q_heads=hq * heads, n_kv_heads=heads, max_new=new, head_lens=per_head)
        by = heads if per_head else 1
        top = r.choice([1, 20, 4000, 1 << 20, MOST])
        front = [r.randint(0, top) if r.random() < 0.8 else 0 for _ in range(groups * by)]
        check(rk, c, n_beams, front + [r.choice([0, 1, r.randint(0, MOST - f), min(top, MOST - f)]) for f in front for _ in range(n_beams)])


def test_an_even_share_where_lengths_are_ordinary(rk):  # noqa: F811
    """64 groups of four beams behind 2048 positions: no more chunks than run at a time, and no fewer than half as many."""
    c = cache(rk, 256, "bf16", n_q_heads=32, n_kv_heads=8, head_dim=128)
    assert check(rk, c, 4, [32] * 64 + [1] * 256) == (64, 256)
    c = cache(rk, 160, "bf16", n_q_heads=1)
    fronts, own = check(rk, c, 2, [3000] * 80 + [1] * 160)
    assert 256 <= fronts + own <= 512


def test_refusals(rk):  # noqa: F811
    c = cache(rk, 256)
    for n_beams, tiles in ((2, [1] * 383), (0, []), (3, [1] * 341), (65, [1] * 259), (2, [MOST + 1] * 384), (2, [-1] * 384)):
        with pytest.raises(rk.RestkvError):
            rk.restkv_debug_beams_list(c, n_beams, tiles)
    with pytest.raises(rk.RestkvError):
        rk.restkv_debug_beams_list(cache(rk, 4), 2, [1] * 6)           # parts cut evenly
    with pytest.raises(rk.RestkvError):
        rk.restkv_debug_beams_list(cache(rk, 256, max_len=64), 2, [1] * 384)       # as if each were alone
    assert rk.lib().restkv_debug_beams_list(rk.binding.ctypes.byref(c), 2, None, None) == -1


@pytest.mark.parametrize("fmt", FORMATS)
def test_sizes_of_the_longest_caches_are_worked_out_in_64_bits(rk, fmt):  # noqa: F811
    """Parts cut evenly, with room for 2^30 positions a sequence: what 64 parts cost passes 2^31 (an overflow shows under the sanitizer)."""
    for groups, n_beams, hq in ((1, 2, 1), (2, 2, 8), (1, 40, 8), (3, 20, 2)):
        c = cache(rk, groups * n_beams, fmt, n_q_heads=hq)
        assert rk.restkv_attend_beams_workspace_bytes(c, n_beams) > 0
        c.max_len = (1 << 30) - 1
        assert rk.restkv_attend_beams_workspace_bytes(c, n_beams) > 0
