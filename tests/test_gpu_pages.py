"""Paged cache on the GPU: append, attention and fetch against a plain implementation in 64 bits (tests/pages_ref.py), at the
lengths, page boundaries, masks, strides and values where they can go wrong, and the calls together as they are used."""
import math

import pytest
import torch

import pages_ref as ref
import paper_2605_08840_amd as rk

pytestmark = pytest.mark.gpu

Plain = ref.Plain


def turns(p, n_pos, seed=1):
    """Tables of cosines and sines (from 64 bits) and a position for every token."""
    half = max(p.c.rotary_dim // 2, 1)
    a = torch.arange(n_pos, dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(half, dtype=torch.float64) / half)
    return a.cos().float(), a.sin().float(), torch.randint(0, n_pos, (p.tokens,), generator=torch.Generator().manual_seed(seed),
                                                           dtype=torch.int32)


# ---- append -------------------------------------------------------------------------------------

APPENDS = [
    # lens (new tokens included), new, what
    ([1], [1], dict()),
    ([16, 17, 31, 32, 33], [1, 1, 1, 1, 1], dict(rotary_dim=64)),
    ([40, 5, 0, 100], [40, 5, 0, 3], dict(rotary_dim=32, d=128, hq=8, hkv=8)),
    ([33, 64], [20, 64], dict(rotary_dim=128, d=128, ps=32, interleaved=True, token_major=True)),
    ([7, 70], [7, 13], dict(rotary_dim=16, hq=7, hkv=1, ps=64)),
    ([[9, 40], [33, 20]], [2, 5], dict(rotary_dim=64, head_lens=True)),
    ([[9, 40, 3], [33, 20, 50]], [2, 3], dict(hq=6, hkv=3, d=128, head_lens=True, head_tables=True, rotary_dim=128)),
    ([3] * 70, [3, 0] * 35, dict(rotary_dim=64, hq=2, hkv=2)),          # more sequences than a wavefront has lanes
    ([2] * 130, [2] * 130, dict(hq=2, hkv=1)),
    ([50], [50], dict(max_new=80, extra_tokens=9)),                     # rows behind the last sequence
    ([90], [50], dict(max_new=30)),                                     # only the first 30 take part
]


@pytest.mark.parametrize("dtype,fmt", [("f32", None), ("bf16", None), ("bf16", "q4"), ("f32", "q4")])
@pytest.mark.parametrize("lens,new,more", APPENDS)
@pytest.mark.parametrize("odd", [False, True])
def test_append(lens, new, more, dtype, fmt, odd):
    p = Plain(rk, lens=lens, new=new, dtype=dtype, fmt=fmt, seed=len(lens) + 7 * odd, n_positions=200, **more)
    cos, sin, pos = turns(p, 200)
    hkv, hq, d, rot, c = p.hkv, p.hq, p.d, p.c.rotary_dim, p.c
    # odd: columns of one wider tensor, at an address that no vector load takes
    wide = p.normal(p.tokens, 1 + (hq + 2 * hkv) * d).to(p.type)
    cut = lambda w, a, n: w[:, 1 + a * d:1 + (a + n) * d].unflatten(1, (n, d))  # noqa: E731
    q, k, v = cut(wide, 0, hq), cut(wide, hq, hkv), cut(wide, hq + hkv, hkv)
    if odd:
        w = wide.cuda()
        qd, kd, vd = cut(w, 0, hq), cut(w, hq, hkv), cut(w, hq + hkv, hkv)
        q_out = qd                                                          # in place
    else:
        qd, kd, vd = (x.contiguous().cuda() for x in (q, k, v))
        q_out = torch.full_like(qd, 3.0)
    before = p.down()
    rk.restkv_append(c, kd, vd, p.pages, p.tensors["table"], p.tensors["lens"], new_start=p.tensors["new_start"],
                     positions=pos.cuda(), cos=cos.cuda(), sin=sin.cuda(), q=qd, q_out=q_out)
    got, got_q = p.down(), q_out.cpu()
    want_q = (q if odd else torch.full_like(q, 3.0)).clone()
    want = {n: x.clone() for n, x in before.items()}
    for s, n in enumerate(new):
        n = min(n, c.max_new)
        for i in range(n):
            t = p.start[s] + i
            ct, st = cos[pos[t].long()], sin[pos[t].long()]
            want_q[t] = ref.rotate(q[t].float(), ct, st, rot, c.rotary_pairs).to(p.type)
            for h in range(hkv):
                at = p.lens[s][h] - n + i
                if at < 0:
                    continue
                w = p.where(s, h, at)
                for name, x in (("k", ref.rotate(k[t, h].float(), ct, st, rot, c.rotary_pairs)), ("v", v[t, h].float())):
                    if p.q4:
                        want[name][w], want[name + "_scale"][w] = ref.to_q4(x)
                    else:
                        want[name][w] = x.to(p.type)
    assert torch.equal(got_q, want_q)
    for name in want:
        assert torch.equal(torch.nan_to_num(got[name].float(), 12345.0), torch.nan_to_num(want[name].float(), 12345.0)), name


def test_append_leaves_out_what_has_no_place():
    """A position outside the tables, a page that is not there, a length beyond the room or short of the new tokens."""
    p = Plain(rk, lens=[20, 40, 30, 2], new=[4, 4, 4, 4], rotary_dim=64, n_positions=50, max_len=38)
    cos, sin, pos = turns(p, 50)
    pos[1], pos[2] = -1, 50
    p.table[2, 0, 1] = -1                                  # cache positions 16 .. of sequence 2
    p.tensors["table"] = p.table[:, 0].contiguous().cuda()
    k, v, q = p.normal(16, 2, 64).bfloat16().cuda(), p.normal(16, 2, 64).bfloat16().cuda(), p.normal(16, 4, 64).bfloat16().cuda()
    q_out, before = torch.zeros_like(q), p.down()
    rk.restkv_append(p.c, k, v, p.pages, p.tensors["table"], p.tensors["lens"], new_start=p.tensors["new_start"], positions=pos.cuda(),
                     cos=cos.cuda(), sin=sin.cuda(), q=q, q_out=q_out)
    got = p.down()
    written = torch.zeros(before["k"].shape[:3], dtype=torch.bool)
    for s, at, i in [(0, 16, 0), (0, 19, 3), (1, 36, 0), (1, 37, 1), (3, 0, 2), (3, 1, 3)]:
        for h in range(2):
            written[p.where(s, h, at)] = True
            assert torch.equal(got["v"][p.where(s, h, at)], v[4 * s + i, h].cpu())
    for name in ("k", "v"):
        same = (got[name] == before[name]) | (torch.isnan(got[name]) & torch.isnan(before[name]))
        assert torch.equal(same.all(-1), ~written)
    assert torch.equal(q_out.any(-1).any(-1).cpu(), torch.tensor([i not in (1, 2) for i in range(16)]))


@pytest.mark.parametrize("d", [64, 128])
def test_four_bits_of_unusual_values(d):
    """Equal values, single large ones, the range's ends, subnormals, infinities and NaN: codes, steps and zeros."""
    n = 24
    p = Plain(rk, lens=[n], new=[n], dtype="f32", fmt="q4", d=d, hq=2, hkv=1)
    x = p.normal(n, 1, d)
    x[0], x[1], x[2] = 0.0, 2.5, -1.0 / 3
    x[3] *= 1e30
    x[4], x[5] = x[4] * 1e38, x[5] * 1e-40
    x[6] *= 1e-30
    x[7, 0, 5], x[8, 0, 9], x[9, 0, 3] = math.inf, -math.inf, math.nan
    x[10, 0, ::2], x[11, 0, 17] = 1e-3, 3e4
    x[12] = torch.finfo(torch.float32).max
    x[13] = torch.finfo(torch.float32).max * torch.sign(x[13])
    x[14], x[15] = x[14] + 1000.0, -0.0
    x[16] = torch.arange(d).float() / 32
    x[17] = x[17].sign()
    rk.restkv_append(p.c, x.cuda(), (-x).cuda(), p.pages, p.tensors["table"], p.tensors["lens"])
    got = p.down()
    for name, y in (("k", x), ("v", -x)):
        codes, scale = ref.to_q4(y[:, 0])
        for t in range(n):
            w = p.where(0, 0, t)
            assert torch.equal(got[name][w], codes[t]), (name, t)
            assert torch.equal(torch.nan_to_num(got[name + "_scale"][w].float(), 777.0), torch.nan_to_num(scale[t].float(), 777.0)), (name, t)
        # within half a step, wherever the group is finite
        val, f = ref.from_q4(codes, scale), torch.arange(d) % (d // 16) // 2
        fine = torch.isfinite(val)
        half = scale[..., 0].double()[:, f] * (0.5 + 2.0 ** -20)
        assert ((val - y[:, 0].double()).abs() <= half)[fine].all()
        assert not fine[7:10].all() and fine[:3].all()


# ---- fetch --------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype,fmt", [("f32", None), ("bf16", None), ("bf16", "q4"), ("f32", "q4")])
@pytest.mark.parametrize("d,more", [(64, {}), (128, dict(token_major=True, ps=32)), (128, dict(head_lens=True, hkv=3, hq=3)),
                                    (64, dict(head_lens=True, head_tables=True))])
def test_fetch(dtype, fmt, d, more):
    hkv = more.get("hkv", 2)
    lens = [[5 + 37 * s + 11 * h for h in range(hkv)] for s in range(3)] if more.get("head_lens") else [0, 45, 16]
    p = Plain(rk, lens=lens, new=[1, 1, 1], dtype=dtype, fmt=fmt, d=d, **more)
    if not more.get("head_tables"):
        p.table[1, 0, 1] = -7                              # a page that is not there
        p.tensors["table"] = p.table[:, 0].contiguous().cuda()
    for first, n in ((0, 50), (13, 1), (44, 17)):
        idx = torch.randint(-3, 60, (3, hkv, n), generator=p.g, dtype=torch.int32)
        for ix in (None, idx):
            k, v = (torch.full((3, hkv, n, d), 9.0, dtype=p.type, device="cuda") for _ in range(2))
            rk.restkv_fetch(p.c, p.pages, p.tensors["table"], p.tensors["lens"], k, v, idx=None if ix is None else ix.cuda(), first=first)
            for name, got in (("k", k.cpu()), ("v", v.cpu())):
                want = torch.zeros(got.shape, dtype=torch.float64)
                for s in range(3):
                    for h in range(hkv):
                        rows, there = p.rows(s, h, name)
                        for j in range(n):
                            t = first + j if ix is None else int(ix[s, h, j])
                            if 0 <= t < len(rows) and there[t]:
                                want[s, h, j] = rows[t]
                assert torch.equal(got, want.float().to(p.type)), (first, n, ix is None)


# ---- attention ----------------------------------------------------------------------------------

FORMATS = [("f32", None, None), ("bf16", None, None), ("bf16", None, "f32"), ("bf16", "q4", None), ("bf16", "q4", "f32"), ("f32", "q4", None)]

ATTENDS = [
    ([1], [1], dict()),
    ([15, 16, 17, 63, 64, 65], [1] * 6, dict()),
    ([0, 1, 130], [1, 1, 1], dict(hq=2, hkv=2)),                              # a sequence without a position
    ([129, 300, 700], [1, 1, 1], dict(d=128, hq=8, hkv=2, ps=64)),            # several chunks
    ([260, 2, 31], [3, 2, 1], dict(d=128, hq=14, hkv=2, ps=32)),              # group of 7; 21 rows
    ([40, 333], [40, 17], dict(hq=6, hkv=2, token_major=True)),               # 120 rows, row blocks of several tokens
    ([40, 333], [40, 17], dict(hq=6, hkv=2, causal=False)),
    ([[9, 140], [333, 20], [5, 0]], [2, 5, 1], dict(head_lens=True)),
    ([[90, 40, 3], [33, 200, 50]], [2, 3], dict(hq=6, hkv=3, d=128, head_lens=True, head_tables=True)),
    ([200], [1], dict(scale=0.31, max_len=150)),                              # longer than the room: the first 150
    ([200], [90], dict(max_new=33, room=3)),                                  # the first 33 of 90
    ([70, 500], [0, 4], dict(extra_tokens=3, hq=40, hkv=1)),                  # no new tokens; rows behind the last
    ([3] * 67 + [400], [1] * 68, dict(hq=2, hkv=1)),                          # more sequences than lanes, one of them long
    ([2, 5], [4, 9], dict()),                                                 # more new tokens than positions
]


ATTENDS += [
    # 1 to 16 rows: copies of the rows that divide the keys (4 bits), with and without a tile cut short
    ([64, 129, 200], [1, 1, 1], dict(hq=3, hkv=3, d=128)),                    # 1 row
    ([64, 127, 333], [1, 1, 1], dict(hq=10, hkv=2, d=128, ps=32)),            # 5 rows
    ([70, 128, 385], [2, 1, 2], dict(hq=8, hkv=2, d=128)),                    # 8
    ([70, 128, 385], [3, 1, 2], dict(hq=6, hkv=2, d=64)),                     # 9
    ([100, 17], [2, 2], dict(hq=16, hkv=2, d=128, causal=False)),             # 16
    # rows of a window: one and two blocks of a wavefront, several workgroups, some without rows
    ([300, 65], [11, 3], dict(hq=6, hkv=2, d=128, ps=64)),                    # 33 rows
    ([700, 90], [16, 16], dict(hq=8, hkv=2, d=128, ps=32, token_major=True)),  # 64
    ([129, 400, 33], [33, 20, 33], dict(hq=4, hkv=2, d=128)),                 # 66
    ([260, 1000], [70, 65], dict(hq=8, hkv=2, d=64, ps=64)),                  # 280
    ([[30, 400], [500, 3]], [24, 2], dict(hq=12, hkv=2, d=128, head_lens=True)),
    ([200, 190], [40, 40], dict(hq=2, hkv=2, d=128, causal=False)),
]


def test_attention_of_many_sequences_and_heads():
    """More entries than a workgroup has threads, lengths of 0 to 2000 among them."""
    for head_lens in (True, False):
        n = 150 if head_lens else 300
        g = torch.Generator().manual_seed(7)
        lens = torch.randint(0, 9, (n, 2), generator=g)
        lens[torch.randint(0, n, (6,), generator=g), 0] = torch.tensor([2000, 700, 130, 65, 64, 1])
        lens = lens.tolist() if head_lens else lens[:, 0].tolist()
        p = Plain(rk, lens=lens, new=[(s % 5 > 0) * 1 for s in range(n)], hq=2, hkv=2, head_lens=head_lens, out_dtype="f32")
        check_attend(p, p.normal(p.tokens, 2, 64).bfloat16(), torch.float32)


def run_attend(p, q, out_type, lse=True, **more):
    out = torch.full((p.tokens, p.hq, p.d), 5.0, dtype=out_type, device="cuda")
    l = torch.full((p.tokens, p.hq), 5.0, dtype=torch.float32, device="cuda") if lse else None
    ws = rk.alloc_attend_workspace(p.c)
    if ws is not None:
        ws.fill_(255)                                      # whatever it holds
    rk.restkv_attend(p.c, q.cuda(), p.pages, p.tensors["table"], p.tensors["lens"], out, l, ws, new_start=p.tensors["new_start"], **more)
    return out.cpu(), None if l is None else l.cpu()


def used_rows(p):
    return [t for s, n in enumerate(p.new) for t in range(p.start[s], p.start[s] + min(n, p.c.max_new))]


def check_attend(p, q, out_type, causal=True, scale=None):
    got, lse = run_attend(p, q, out_type)
    rows = used_rows(p)
    want = ref.attention(p, q, scale=scale, causal=causal)
    ref.assert_attention(got, lse, want, out_type, rows)
    rest = [t for t in range(p.tokens) if t not in set(rows)]
    assert (got[rest] == 5.0).all() and (lse[rest] == 5.0).all()
    return got, lse


@pytest.mark.parametrize("dtype,fmt,out", FORMATS)
@pytest.mark.parametrize("lens,new,more", ATTENDS)
def test_attention(lens, new, more, dtype, fmt, out):
    p = Plain(rk, lens=lens, new=new, dtype=dtype, fmt=fmt, out_dtype=out, seed=sum(new), **more)
    out_type = torch.float32 if "f32" in (dtype, out) else torch.bfloat16
    q = (p.normal(p.tokens, p.hq, p.d) * 2).to(p.type)
    check_attend(p, q, out_type, causal=more.get("causal", True), scale=more.get("scale"))


@pytest.mark.parametrize("dtype,fmt,out", FORMATS)
def test_attention_far_apart_logits(dtype, fmt, out):
    """Weights that are 0 but for one key, references that move by hundreds, and equal logits."""
    out_type = torch.float32 if "f32" in (dtype, out) else torch.bfloat16
    for spread in (0.0, 12.0):
        p = Plain(rk, lens=[300, 90], new=[2, 1], dtype=dtype, fmt=fmt, out_dtype=out, d=128, hq=4, hkv=1, spread=spread)
        q = (p.normal(p.tokens, p.hq, p.d) * 5).to(p.type)
        check_attend(p, q, out_type)


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("dtype,fmt", [("f32", None), ("bf16", None), ("bf16", "q4")])
def test_what_a_query_does_not_see_has_no_influence(dtype, fmt, bad):
    """Later tokens of the same call whose keys and values are not finite; the queries that see them get what they ask for."""
    for d, hq, n in ((64, 2, 6), (128, 8, 40)):
        p = Plain(rk, lens=[100, 70], new=[n, n], dtype=dtype, fmt=fmt, d=d, hq=hq, hkv=2, out_dtype="f32")
        first = [100 - n // 2, 70 - 1]                     # the first bad position of each sequence
        q = p.normal(p.tokens, p.hq, d).to(p.type)
        clean = run_attend(p, q, torch.float32)
        for s in range(2):
            for h in range(2):
                for t in range(first[s], p.lens[s][h], 3):
                    for name in ("k", "v"):
                        x = p.pool[name + "_scale"][p.where(s, h, t)] if p.q4 else p.pool[name][p.where(s, h, t)]
                        x.view(-1)[1::2] = bad
        p.up()
        got = run_attend(p, q, torch.float32)
        for s in range(2):
            for i in range(n):
                t, sees = p.start[s] + i, p.lens[s][0] - n + i + 1
                if sees <= first[s]:
                    assert torch.equal(got[0][t], clean[0][t]) and torch.equal(got[1][t], clean[1][t]), (d, s, i)
                elif math.isnan(bad):
                    assert torch.isnan(got[0][t]).all()


@pytest.mark.parametrize("dtype,fmt", [("f32", None), ("bf16", None), ("bf16", "q4")])
def test_values_that_are_not_finite_and_seen(dtype, fmt):
    """An infinity among the values of a key that all see: what the sum gives, channel by channel."""
    p = Plain(rk, lens=[90], new=[2], dtype=dtype, fmt=fmt, d=64, hq=2, hkv=1, out_dtype="f32")
    q = p.normal(2, 2, 64).to(p.type)
    if p.q4:
        p.pool["v_scale"][p.where(0, 0, 70)][1] = torch.tensor([0.5, math.inf])
    else:
        p.pool["v"][p.where(0, 0, 70)][7] = math.inf
        p.pool["v"][p.where(0, 0, 88)][9] = -math.inf       # the first query's own position, in a tile with a mask
    p.up()
    got, _ = run_attend(p, q, torch.float32)
    want = ref.attention(p, q)[0]
    inf = torch.isinf(want)
    assert inf.any() and torch.equal(got.double()[inf], want[inf]) and torch.isfinite(got[~inf]).all()


@pytest.mark.parametrize("dtype,fmt", [("f32", None), ("bf16", None), ("bf16", "q4")])
def test_missing_pages_and_keys_of_minus_infinity(dtype, fmt):
    p = Plain(rk, lens=[100, 40, 50], new=[2, 1, 3], dtype=dtype, fmt=fmt, d=128, hq=4, hkv=2, out_dtype="f32")
    p.table[0, 0, 2], p.table[0, 0, 6] = -1, p.c.n_pages         # positions 32 .. 47 and the last ones
    p.table[1, 0, :] = -1                                        # nothing is left of sequence 1
    p.tensors["table"] = p.table[:, 0].contiguous().cuda()
    q = p.normal(p.tokens, 4, 128).to(p.type)
    got, lse = check_attend(p, q, torch.float32)
    assert (got[2] == 0).all() and torch.isneginf(lse[2]).all()
    if not p.q4:          # every logit of sequence 2 is -inf
        q = q.abs() + 1
        for h in range(2):
            for t in range(50):
                p.pool["k"][p.where(2, h, t)] = -math.inf
        p.up()
        got, lse = run_attend(p, q, torch.float32)
        assert (got[3:] == 0).all() and torch.isneginf(lse[3:]).all()
        # all but one
        p.pool["k"][p.where(2, 0, 13)] = 0.25
        p.up()
        got, lse = run_attend(p, q, torch.float32)
        v = p.rows(2, 0, "v")[0][13].float()
        # one weight w = 2^x, |x| the rounding of the logit: w v (in up to three parts, a rounding each), 1 / w and their product
        # are five roundings, and what three bf16 parts leave of w is below a sixth
        assert ((got[3:, :2] - v).abs() <= 6 * ref.F32 * v.abs()).all() and torch.isfinite(lse[3:, :2]).all()


@pytest.mark.parametrize("dtype,fmt", [("bf16", None), ("f32", None), ("bf16", "q4"), ("f32", "q4")])
def test_strided_unaligned_queries_and_outputs_and_no_lse(dtype, fmt):
    p = Plain(rk, lens=[77, 200], new=[3, 2], dtype=dtype, fmt=fmt, d=64, hq=6, hkv=3)
    wide = p.normal(p.tokens, 11 * 64 + 1).to(p.type).cuda()
    q = wide[:, 65:65 + 6 * 64].unflatten(1, (6, 64))
    store = torch.full((6 * (p.tokens + 1) * 64 + 1,), 5.0, dtype=p.type, device="cuda")
    out = store[1:].view(6, p.tokens + 1, 64)[:, :p.tokens].transpose(0, 1)
    rk.restkv_attend(p.c, q, p.pages, p.tensors["table"], p.tensors["lens"], out, None, rk.alloc_attend_workspace(p.c), new_start=p.tensors["new_start"])
    ref.assert_attention(out.cpu(), None, ref.attention(p, q.cpu()), p.type, used_rows(p))
    assert (store[1:].view(6, p.tokens + 1, 64)[:, p.tokens] == 5.0).all() and store[0] == 5.0


@pytest.mark.parametrize("dtype,fmt", [("bf16", None), ("f32", None), ("bf16", "q4")])
def test_long_cache_many_chunks(dtype, fmt):
    """20011 positions: many chunks, against 64 bits on the GPU; twice the same bits."""
    n, d, hq, hkv, ps = 20011, 128, 8, 2, 64
    g = torch.Generator(device="cuda").manual_seed(3)
    pages = (n + ps - 1) // ps
    c = rk.make_cache(n_seqs=1, n_q_heads=hq, n_kv_heads=hkv, head_dim=d, page_size=ps, n_pages=pages, max_pages=pages, dtype=dtype,
                      format=fmt, max_new=n, out_dtype="f32")
    vt = torch.float32 if dtype == "f32" else torch.bfloat16
    k, v = (torch.randn((n, hkv, d), generator=g, device="cuda").to(vt) for _ in range(2))
    k[5] *= 6
    pool, table = rk.alloc_cache_pages(c), torch.randperm(pages, generator=g, device="cuda").int()[None]
    lens = torch.tensor([n], dtype=torch.int32, device="cuda")
    rk.restkv_append(c, k, v, pool, table, lens)
    ko, vo = (torch.empty((1, hkv, n, d), dtype=torch.float32 if fmt else vt, device="cuda") for _ in range(2))
    f = rk.make_cache(n_seqs=1, n_q_heads=hq, n_kv_heads=hkv, head_dim=d, page_size=ps, n_pages=pages, max_pages=pages,
                      dtype="f32" if fmt else dtype, format=fmt)
    rk.restkv_fetch(f, pool, table, lens, ko, vo)
    for new in (1, 2, 5, 20, 64):
        c = rk.make_cache(n_seqs=1, n_q_heads=hq, n_kv_heads=hkv, head_dim=d, page_size=ps, n_pages=pages, max_pages=pages,
                          dtype=dtype, format=fmt, max_new=new, out_dtype="f32")
        q = torch.randn((new, hq, d), generator=g, device="cuda").to(vt)
        ws = rk.alloc_attend_workspace(c)
        runs = []
        for _ in range(2):
            out, lse = torch.empty((new, hq, d), device="cuda"), torch.empty((new, hq), device="cuda")
            rk.restkv_attend(c, q, pool, table, lens, out, lse, ws)
            runs.append((out, lse))
        assert torch.equal(runs[0][0], runs[1][0]) and torch.equal(runs[0][1], runs[1][1])
        for h in range(hkv):
            kk, vv = ko[0, h].double(), vo[0, h].double()
            x = q[:, h * 4:h * 4 + 4].double().reshape(-1, d)
            s = torch.matmul(x, kk.t().contiguous()) * d ** -0.5
            mask = torch.arange(n, device="cuda")[None] > (n - new + torch.arange(new, device="cuda")).repeat_interleave(4)[:, None]
            s[mask] = -math.inf
            w = torch.softmax(s, -1)
            # as in pages_ref.attention: logits of magnitude sums up to 6 |k| of 128 terms (the heavy key), 47/15 of that in 4 bits
            e_logit = 2.0 ** -24 * (136 * float((x.abs() @ kk.abs().t().contiguous()).max()) * d ** -0.5 * (4 if fmt else 1) + 4 * float(s[~mask].abs().max()) + 4)
            bound = (2 * e_logit + (n / 64 + 85) * 2.0 ** -24) * (w @ vv.abs()) * (4 if fmt else 1)
            off = (runs[0][0][:, h * 4:h * 4 + 4].double().reshape(-1, d) - w @ vv).abs()
            assert (off <= bound).all(), (off / bound).max()
            e = (runs[0][1][:, h * 4:h * 4 + 4].double().reshape(-1) - torch.logsumexp(s, -1)).abs()
            assert (e <= e_logit + (n / 64 + 120) * 2.0 ** -24).all()


# ---- the calls together -------------------------------------------------------------------------

@pytest.mark.parametrize("fmt", [None, "q4"])
def test_evict_decode_and_evict_again(fmt):
    """A layer's cache is evicted into pages, 16 tokens are decoded, and the grown cache is evicted again through the
    statistics of the paged attention: the same rows, and the scores of the library's own attention pass."""
    hq, hkv, d, L, W, B, ps, steps = 8, 2, 128, 700, 16, 160, 32, 16
    g = torch.Generator(device="cuda").manual_seed(5)
    rnd = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    bf = torch.bfloat16
    q, k, v = rnd(hq, W, d).to(bf), rnd(hkv, L, d).to(bf), rnd(hkv, L, d).to(bf)
    gram = rnd(hq, d, d) / d ** 0.5
    gram = torch.matmul(gram, gram.transpose(1, 2).contiguous())
    p = rk.make_params(n_q_heads=hq, n_kv_heads=hkv, head_dim=d, seq_len=L, window=W, budget=B, dtype="bf16")
    buf = rk.alloc_layer_buffers(p, bf)
    rk.evict_layer(p, q, k, v, gram, buf)
    pages = (B + steps + ps - 1) // ps
    common = dict(n_seqs=1, n_q_heads=hq, n_kv_heads=hkv, head_dim=d, page_size=ps, n_pages=pages + 2, max_pages=pages, dtype=bf, format=fmt)
    fill = rk.make_cache(**common, max_new=B)
    pool, table = rk.alloc_cache_pages(fill), torch.randperm(pages + 2, generator=g, device="cuda")[:pages].int()[None]
    lens = torch.full((1,), B, dtype=torch.int32, device="cuda")
    rk.restkv_append(fill, buf.k_out.transpose(0, 1), buf.v_out.transpose(0, 1), pool, table, lens)
    # decode: rotation at the true positions
    ang = torch.arange(L + steps, dtype=torch.float64, device="cuda")[:, None] * 10000.0 ** (-torch.arange(d // 2, dtype=torch.float64, device="cuda") / (d // 2))
    cos, sin = ang.cos().float(), ang.sin().float()
    step = rk.make_cache(**common, rotary_dim=d, n_positions=L + steps)
    ws, out = rk.alloc_attend_workspace(step), torch.empty((1, hq, d), dtype=bf, device="cuda")
    queries, outs, new_k, new_v = [], [], [], []
    for i in range(steps):
        kn, vn, qn = rnd(1, hkv, d).to(bf), rnd(1, hkv, d).to(bf), rnd(1, hq, d).to(bf)
        lens += 1
        rk.restkv_append(step, kn, vn, pool, table, lens, positions=torch.tensor([L + i], dtype=torch.int32, device="cuda"), cos=cos, sin=sin, q=qn, q_out=qn)
        rk.restkv_attend(step, qn, pool, table, lens, out, None, ws)
        queries.append(qn[0])
        outs.append(out[0].float())
        new_k.append(kn)
        new_v.append(vn)
    # the window's queries again, all at once: output and log-sum-exp as the score takes them
    n = B + steps
    win = rk.make_cache(**common, max_new=steps, out_dtype="f32", out_head_major=True)
    qs = torch.stack(queries)
    o = torch.empty((hq, steps, d), device="cuda")
    lse = torch.empty((hq, steps), device="cuda")
    rk.restkv_attend(win, qs, pool, table, lens, o.transpose(0, 1), lse.transpose(0, 1), rk.alloc_attend_workspace(win))
    # (a step's output is the window's, rounded once; both sums within 2^-15 of the exact one here)
    assert ((torch.stack(outs) - o.transpose(0, 1)).abs() <= 2.0 ** -8 * o.transpose(0, 1).abs() + 2.0 ** -14 * 4).all()
    kd, vd = (torch.empty((1, hkv, n, d), dtype=bf, device="cuda") for _ in range(2))
    rk.restkv_fetch(win, pool, table, lens, kd, vd)
    if fmt is None:
        assert torch.equal(kd[0, :, :B], buf.k_out) and torch.equal(vd[0, :, :B], buf.v_out)
        assert torch.equal(vd[0, :, B:], torch.cat(new_v).transpose(0, 1))
        a, b = torch.cat(new_k).float().chunk(2, -1)
        c, s = cos[L:, None], sin[L:, None]
        assert torch.equal(kd[0, :, B:], torch.cat((a * c - b * s, b * c + a * s), -1).to(bf).transpose(0, 1))
    p2 = rk.make_params(n_q_heads=hq, n_kv_heads=hkv, head_dim=d, seq_len=n, window=steps, budget=B, dtype="bf16")
    buf2 = rk.alloc_layer_buffers(p2, bf)
    qh = qs.transpose(0, 1).contiguous()
    own = torch.empty_like(buf2.score)
    rk.restkv_score(p2, qh, kd[0], vd[0], gram, own, buf2.workspace)
    rk.restkv_score_from_attention(p2, qh, kd[0], vd[0], gram, o, lse, buf2.score, buf2.workspace)
    # 16-bit pages: the scores' own bound on both sides; 4 bits: the dense rows are rounded to bf16 once more, 2^-8 of a value
    tol = 2e-3 if fmt is None else 2e-2
    assert ((buf2.score - own).abs() <= tol * own + 1e-6).all()
    rk.restkv_smooth(p2, buf2.score, buf2.ema, buf2.final, buf2.aws_info, buf2.aws_d, buf2.workspace)
    rk.restkv_select(p2, buf2.final, buf2.idx, buf2.workspace)
    # the kept rows, straight from the pages
    kk, vv = torch.empty_like(buf2.k_out)[None], torch.empty_like(buf2.v_out)[None]
    rk.restkv_fetch(win, pool, table, lens, kk, vv, idx=buf2.idx)
    rk.restkv_compact(p2, kd[0], vd[0], buf2.idx, buf2.k_out, buf2.v_out)
    assert torch.equal(kk[0], buf2.k_out) and torch.equal(vv[0], buf2.v_out)


@pytest.mark.parametrize("fmt", [None, "q4"])
def test_decode_step_replayed_from_a_hip_graph(fmt):
    """Append and attention captured once, replayed with lengths that grow between the replays; two graphs share a workspace."""
    hq, hkv, d, ps, cap = 8, 2, 64, 16, 640
    g = torch.Generator(device="cuda").manual_seed(9)
    c = rk.make_cache(n_seqs=2, n_q_heads=hq, n_kv_heads=hkv, head_dim=d, page_size=ps, n_pages=2 * cap // ps, max_pages=cap // ps,
                      dtype="bf16", format=fmt, rotary_dim=d, n_positions=cap)
    table = torch.randperm(2 * cap // ps, generator=g, device="cuda").int().view(2, -1)
    ang = torch.arange(cap, dtype=torch.float64, device="cuda")[:, None] * 10000.0 ** (-torch.arange(d // 2, dtype=torch.float64, device="cuda") / 32)
    cos, sin = ang.cos().float(), ang.sin().float()
    k, v, q = (torch.empty((2, n, d), dtype=torch.bfloat16, device="cuda") for n in (hkv, hkv, hq))
    ws = rk.alloc_attend_workspace(c)
    assert ws is not None
    sides = []
    for graphed in (True, False):
        pool, lens = rk.alloc_cache_pages(c), torch.tensor([600, 3], dtype=torch.int32, device="cuda")
        pool.k.view(torch.uint8).random_(0, 60, generator=torch.Generator(device="cuda").manual_seed(1))
        pool.v.view(torch.uint8).random_(0, 60, generator=torch.Generator(device="cuda").manual_seed(2))
        q_out, out, lse = torch.empty_like(q), torch.empty_like(q), torch.empty((2, hq), device="cuda")

        def step(pool=pool, lens=lens, q_out=q_out, out=out, lse=lse):
            lens.add_(1)
            rk.restkv_append(c, k, v, pool, table, lens, cos=cos, sin=sin, q=q, q_out=q_out)
            rk.restkv_attend(c, q_out, pool, table, lens, out, lse, ws)

        if graphed:
            for x in (k, v, q):
                x.normal_(generator=g)
            s = torch.cuda.Stream()
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                step()
            torch.cuda.current_stream().wait_stream(s)
            lens.copy_(torch.tensor([600, 3], dtype=torch.int32))
            graphs = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()]
            for gr in graphs:
                with torch.cuda.graph(gr):
                    step()
            lens.copy_(torch.tensor([600, 3], dtype=torch.int32))
        sides.append((step, pool, lens, out, lse))
    for i in range(6):
        for x in (k, v, q):
            x.normal_(generator=g)
        graphs[i & 1].replay()
        torch.cuda.synchronize()
        sides[1][0]()
        torch.cuda.synchronize()
        assert torch.equal(sides[0][2], sides[1][2]) and torch.equal(sides[0][3], sides[1][3]) and torch.equal(sides[0][4], sides[1][4])
        assert torch.equal(sides[0][1].v.view(torch.uint8), sides[1][1].v.view(torch.uint8))
    assert sides[0][2].tolist() == [606, 9]


def test_two_calls_at_once():
    """Two streams, a workspace each: the results of the calls one after the other."""
    p = Plain(rk, lens=[1500, 700], new=[2, 1], d=128, hq=8, hkv=2)
    q = p.normal(p.tokens, 8, 128).bfloat16().cuda()
    streams, outs, ws = [torch.cuda.Stream() for _ in range(2)], [torch.empty_like(q) for _ in range(3)], [rk.alloc_attend_workspace(p.c) for _ in range(2)]
    t = p.tensors
    rk.restkv_attend(p.c, q, p.pages, t["table"], t["lens"], outs[2], None, ws[0], new_start=t["new_start"])
    torch.cuda.synchronize()
    for _ in range(20):
        for i, s in enumerate(streams):
            rk.restkv_attend(p.c, q, p.pages, t["table"], t["lens"], outs[i], None, ws[i], new_start=t["new_start"], stream=s)
    torch.cuda.synchronize()
    assert torch.equal(outs[0], outs[2]) and torch.equal(outs[1], outs[2])


def test_calls_on_another_stream():
    p = Plain(rk, lens=[500, 33], new=[1, 1], d=128, hq=8, hkv=2)
    q = p.normal(2, 8, 128).bfloat16()
    want = run_attend(p, q, torch.bfloat16)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = run_attend(p, q, torch.bfloat16)
    also = run_attend(p, q, torch.bfloat16, stream=torch.cuda.current_stream())
    assert all(torch.equal(a, b) and torch.equal(a, c) for a, b, c in zip(want, got, also))


def test_binding_refuses_wrong_tensors_on_the_gpu():
    p = Plain(rk, lens=[50, 3], new=[1, 1])
    t, q = p.tensors, p.normal(2, 4, 64).bfloat16().cuda()
    kv, out, lse = p.normal(2, 2, 64).bfloat16().cuda(), torch.empty_like(q), torch.empty((2, 4), device="cuda")

    def refused(f, *a, **kw):
        with pytest.raises(rk.RestkvError):
            f(*a, **kw)

    A = (p.c, q, p.pages, t["table"], t["lens"])
    refused(rk.restkv_attend, *A, out.float())
    refused(rk.restkv_attend, *A, out[:1])
    refused(rk.restkv_attend, *A, out, lse.double())
    refused(rk.restkv_attend, *A, out.cpu())
    refused(rk.restkv_attend, p.c, q[..., ::2], p.pages, t["table"], t["lens"], out)
    refused(rk.restkv_attend, p.c, q[:1].expand(2, 4, 64), p.pages, t["table"], t["lens"], out)
    refused(rk.restkv_attend, p.c, q, p.pages, t["table"].long(), t["lens"], out)
    refused(rk.restkv_attend, p.c, q, p.pages, t["table"][:, :1], t["lens"], out)
    refused(rk.restkv_attend, p.c, q, p.pages, t["table"], t["lens"][:1], out)
    refused(rk.restkv_attend, *A, out, new_start=t["new_start"][:2])
    refused(rk.restkv_append, p.c, kv, kv[:, :1], p.pages, t["table"], t["lens"])
    refused(rk.restkv_append, p.c, kv, kv.float(), p.pages, t["table"], t["lens"])
    refused(rk.restkv_append, p.c, kv, kv.transpose(0, 1).contiguous().transpose(0, 1), p.pages, t["table"], t["lens"])
    refused(rk.restkv_append, p.c, kv, kv, p.pages, t["table"], t["lens"], q=q)
    refused(rk.restkv_append, p.c, kv, kv, p.pages, t["table"], t["lens"], positions=t["lens"].long())
    ko = torch.empty((2, 2, 8, 64), dtype=torch.bfloat16, device="cuda")
    refused(rk.restkv_fetch, p.c, p.pages, t["table"], t["lens"], ko, ko[:, :, :4])
    refused(rk.restkv_fetch, p.c, p.pages, t["table"], t["lens"], ko.float(), ko.float())
    refused(rk.restkv_fetch, p.c, p.pages, t["table"], t["lens"], ko, ko.clone(), idx=t["lens"])


@pytest.mark.parametrize("dtype,fmt,new", [("bf16", None, 5), ("bf16", None, 20), ("bf16", "q4", 1), ("bf16", "q4", 6), ("f32", None, 5)])
def test_attention_of_more_rows_replayed_from_a_hip_graph(dtype, fmt, new):
    """20, 80, 4 and 24 rows: the kernels of several row blocks and of many rows, captured, with lengths that change."""
    lens = [[2000, 77], [40, 2047], [1, 900]]
    p = Plain(rk, lens=[2048, 2048], new=[new, new], dtype=dtype, fmt=fmt, d=128, hq=8, hkv=2, ps=64)
    t, q = p.tensors, p.normal(2 * new, 8, 128).to(p.type).cuda()
    ws, told = rk.alloc_attend_workspace(p.c), torch.tensor([2048, 2048], dtype=torch.int32, device="cuda")
    assert ws is not None
    outs, lses = [torch.empty_like(q) for _ in range(2)], [torch.empty(q.shape[:2], device="cuda") for _ in range(2)]

    def step(i):
        rk.restkv_attend(p.c, q, p.pages, t["table"], told, outs[i], lses[i], ws, new_start=t["new_start"])

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(0)
    for l in lens + lens:
        told.copy_(torch.tensor(l, dtype=torch.int32))
        q.mul_(0.9)
        graph.replay()
        torch.cuda.synchronize()
        step(1)
        torch.cuda.synchronize()
        assert torch.equal(outs[0], outs[1]) and torch.equal(lses[0], lses[1])


@pytest.mark.parametrize("fmt", [None, "q4"])
def test_pages_that_pass_four_gigabytes(fmt):
    """Pages of 65536 positions, the last of an array of more than 2^32 bytes: the results of a small array."""
    ps, d, hq, hkv, n, new = 65536, 64, 4, 1, 65700, 65600
    row = d // 2 if fmt else 2 * d
    many = (1 << 32) // (ps * row) + 3
    assert many * ps * row > 1 << 32
    g = torch.Generator(device="cuda").manual_seed(4)
    k, v = (torch.randn((n, hkv, d), generator=g, device="cuda").bfloat16() for _ in range(2))
    q = torch.randn((n, hq, d), generator=g, device="cuda").bfloat16()
    start, lens = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([0, new, n], [new, n - new]))
    got = []
    for pages, table in ((4, [[2, 0], [3, 1]]), (many, [[many - 1, 1], [0, many - 2]])):
        args = dict(n_seqs=2, n_q_heads=hq, n_kv_heads=hkv, head_dim=d, page_size=ps, n_pages=pages, max_pages=2, dtype="bf16", format=fmt)
        c = rk.make_cache(max_new=new, n_tokens=n, **args)
        pool, tb = rk.alloc_cache_pages(c), torch.tensor(table, dtype=torch.int32, device="cuda")
        rk.restkv_append(c, k, v, pool, tb, lens, new_start=start)
        ko, vo = (torch.zeros((2, hkv, new, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        rk.restkv_fetch(c, pool, tb, lens, ko, vo)
        if not fmt:
            assert torch.equal(ko[0, 0], k[:new, 0]) and torch.equal(vo[1, 0, :n - new], v[new:, 0])
        res = [ko, vo]
        for m in (1, 12):
            cd = rk.make_cache(max_new=m, **args)
            out, lse = torch.empty((2 * m, hq, d), dtype=torch.bfloat16, device="cuda"), torch.empty((2 * m, hq), device="cuda")
            rk.restkv_attend(cd, q[:2 * m], pool, tb, lens, out, lse, rk.alloc_attend_workspace(cd))
            assert torch.isfinite(lse).all()
            res += [out, lse]
        got.append(res)
        del pool
    assert all(torch.equal(a, b) for a, b in zip(*got))


@pytest.mark.parametrize("out", [None, "f32"])
@pytest.mark.parametrize("lens,new,more", [
    ([300, 65, 40], [40, 3, 33], dict(hq=8, hkv=2, d=128)),                   # 160 rows: eight wavefronts, five of them with rows
    ([700, 90], [100, 90], dict(hq=8, hkv=2, d=64, ps=32)),                   # 400 and 360
    ([700, 31], [64, 64], dict(hq=8, hkv=2, d=128, causal=False)),            # 256, more of them than positions
    ([[200, 400], [500, 3]], [40, 22], dict(hq=12, hkv=2, d=128, head_lens=True)),
    ([60] * 70 + [900], [34, 0, 3] * 23 + [5, 34], dict(hq=4, hkv=1, d=64)),  # 136, of more sequences than lanes
])
def test_attention_of_many_rows(lens, new, more, out):
    p = Plain(rk, lens=lens, new=new, dtype="bf16", out_dtype=out, seed=sum(new), **more)
    check_attend(p, p.normal(p.tokens, p.hq, p.d).bfloat16(), torch.float32 if out else torch.bfloat16, causal=more.get("causal", True))


@pytest.mark.parametrize("dtype,fmt", [("f32", "q4"), ("bf16", "q4"), ("f32", None), ("bf16", None)])
@pytest.mark.parametrize("n,d", [(75, 64), (120, 128), (3000, 128)])
def test_float32_output_is_as_near_as_plain_float32(dtype, fmt, n, d):
    """Norm of the output's error against 64 bits: at most twice that of the same attention in float32 on the CPU (codes put
    together with an offset, whose sums are several times what they stand for, are further off: 5 to 8 times at 75 and 120)."""
    p = Plain(rk, lens=[n, n // 2], new=[1, 1], dtype=dtype, fmt=fmt, out_dtype="f32", hq=8, hkv=2, d=d, ps=32, seed=n)
    q = p.normal(2, 8, d).to(p.type)
    got, _ = run_attend(p, q, torch.float32)
    off, plain = 0.0, 0.0
    for s in range(2):
        for h in range(2):
            k, v = p.rows(s, h, "k")[0], p.rows(s, h, "v")[0]
            x = q[s, h * 4:h * 4 + 4]
            want = torch.softmax(x.double() @ k.t() * d ** -0.5, -1) @ v
            near = torch.softmax(x.float() @ k.float().t() * d ** -0.5, -1) @ v.float()
            off += float((got[s, h * 4:h * 4 + 4].double() - want).square().sum())
            plain += float((near.double() - want).square().sum())
    assert off <= 4 * plain, (off / plain) ** 0.5


@pytest.mark.parametrize("dtype,fmt,d,rot,pairs", [
    ("bf16", None, 128, 128, False), ("bf16", None, 128, 64, False), ("bf16", "q4", 128, 128, True), ("bf16", None, 64, 64, True),
    ("f32", None, 64, 64, False), ("f32", "q4", 128, 128, False), ("f32", None, 128, 0, False), ("bf16", "q4", 64, 32, False)])
def test_large_calls_are_many_small_ones(dtype, fmt, d, rot, pairs):
    """70000 tokens, queries in place: the bits that calls of 600 leave; fetched at once and in parts."""
    n, step, hq, hkv, ps, cap = 70000, 600, 8, 8, 64, 70016
    g = torch.Generator(device="cuda").manual_seed(d + rot)
    t = torch.float32 if dtype == "f32" else torch.bfloat16
    k, v, q = (torch.randn((n, h, d), generator=g, device="cuda").to(t) for h in (hkv, hkv, hq))
    table = torch.randperm(cap // ps, generator=g, device="cuda").int()[None]
    ang = torch.randn((n, max(rot // 2, 1)), generator=g, device="cuda")
    cos, sin = ang.cos(), ang.sin()
    args = dict(n_seqs=1, n_q_heads=hq, n_kv_heads=hkv, head_dim=d, page_size=ps, n_pages=cap // ps, max_pages=cap // ps, dtype=dtype,
                format=fmt, rotary_dim=rot, interleaved=pairs, n_positions=n)
    pools, qs = [], []
    for size in (n, step):
        pool, x = rk.alloc_cache_pages(rk.make_cache(**args)), q.clone()
        for a in range(0, n, size):
            b = min(a + size, n)
            lens = torch.tensor([b], dtype=torch.int32, device="cuda")
            rk.restkv_append(rk.make_cache(max_new=b - a, **args), k[a:b], v[a:b], pool, table, lens, cos=cos, sin=sin, q=x[a:b], q_out=x[a:b])
        pools.append(pool)
        qs.append(x)
    assert torch.equal(qs[0], qs[1]) and (rot == 0) == torch.equal(qs[0], q)
    bits = lambda x: x.view(torch.uint8 if x.dtype == torch.uint8 else torch.int16 if x.element_size() == 2 else torch.int32)  # noqa: E731
    for name in ("k", "v") + (("k_scale", "v_scale") if fmt else ()):
        assert torch.equal(*(bits(getattr(p, name)) for p in pools)), name
    c, out = rk.make_cache(**args), []
    for size in (n, 20000):
        parts = []
        for a in range(0, n, size):
            ko, vo = (torch.empty((1, hkv, min(size, n - a), d), dtype=t, device="cuda") for _ in range(2))
            rk.restkv_fetch(c, pools[0], table, lens, ko, vo, first=a)
            parts.append((ko, vo))
        out.append([torch.cat(x, 2) for x in zip(*parts)])
    assert torch.equal(out[0][0], out[1][0]) and torch.equal(out[0][1], out[1][1])
    if not fmt:
        assert torch.equal(out[0][1][0].transpose(0, 1), v)


# ---- what is not seen, finite but as large as its type holds ---------------------------------------

def page_zero_unused(p):
    """Page 0 (whose rows stand in for those of absent pages) free of every sequence: its place is taken by a spare page."""
    held = set(p.table.flatten().tolist())
    if 0 in held:
        spare = min(set(range(p.c.n_pages)) - held)
        for x in p.pool.values():
            x[[0, spare]] = x[[spare, 0]]
        p.table[p.table == 0] = spare


@pytest.mark.parametrize("dtype,fmt,out", FORMATS)
@pytest.mark.parametrize("junk", [3e38, -3e38])
def test_finite_junk_in_slots_that_nobody_sees(dtype, fmt, out, junk):
    """Slots behind the last position and rows of page 0 (4 bits: their steps and zeros) that hold the largest finite values."""
    out_type = torch.float32 if "f32" in (dtype, out) else torch.bfloat16
    for hq, new, d in ((1, 1, 64), (4, 1, 128), (8, 1, 64), (8, 2, 128), (8, 4, 64), (16, 5, 128)):
        p = Plain(rk, lens=[70, 129, 5, 17 * 16 - 3], new=[new] * 4, dtype=dtype, fmt=fmt, d=d, hq=hq, hkv=1, out_dtype=out, junk=junk,
                  seed=hq + new)
        page_zero_unused(p)
        p.table[1, 0, 2], p.table[3, 0, 0] = -1, p.c.n_pages      # positions 32 .. 47 and the first ones
        p.tensors["table"] = p.table[:, 0].contiguous().cuda()
        p.up()
        check_attend(p, p.normal(p.tokens, hq, d).to(p.type), out_type)


@pytest.mark.parametrize("dtype,fmt,out", FORMATS)
@pytest.mark.parametrize("bad", [3e38, -3e38])
def test_finite_extremes_that_later_queries_see(dtype, fmt, out, bad):
    """Tokens of the same call as large as their type holds (4 bits: steps, zeros, both): queries before them go by the rest."""
    out_type = torch.float32 if "f32" in (dtype, out) else torch.bfloat16
    for d, hq, n, names, at in ((64, 2, 6, "v", 0), (128, 8, 40, "v", 0), (128, 8, 3, "vk", 0), (64, 4, 2, "v", None), (64, 8, 9, "kv", None)):
        p = Plain(rk, lens=[100, 70], new=[n, n], dtype=dtype, fmt=fmt, d=d, hq=hq, hkv=2, out_dtype=out)
        first = [100 - n // 2, 70 - 1]                     # the first such position of each sequence
        q = p.normal(p.tokens, p.hq, d).to(p.type)
        for s in range(2):
            for h in range(2):
                for t in range(first[s], p.lens[s][h]):
                    for name in names:
                        x = p.pool[name + "_scale"][p.where(s, h, t)] if p.q4 else p.pool[name][p.where(s, h, t)]
                        if at is None:
                            x[:] = bad
                        else:
                            x.view(-1)[at::2] = bad
        p.up()
        got, lse = run_attend(p, q, out_type)
        rows = [p.start[s] + i for s in range(2) for i in range(n) if p.lens[s][0] - n + i + 1 <= first[s]]
        ref.assert_attention(got, lse, ref.attention(p, q), out_type, rows)


def test_four_bits_of_every_kind_of_nan():
    """Quiet and signalling NaN of both signs, at even and odd channels, among finite values: the group is NaN, its neighbours are not."""
    patterns = [0xFFFFFFFF, 0xFFFF0001, 0x7FFFFFFF, 0x7F800001, 0xFF800001, 0xFFC00000, 0x7FC00000, 0xFFFF0000]
    for d in (64, 128):
        n = 2 * len(patterns)
        p = Plain(rk, lens=[n], new=[n], dtype="f32", fmt="q4", d=d, hq=2, hkv=1)
        sides = dict(k=p.normal(n, 1, d), v=p.normal(n, 1, d))
        for x in sides.values():
            for i in range(n):
                bits = patterns[i // 2]
                x.view(torch.int32)[i, 0, d // 2 + 2 + i % 2] = bits - (1 << 32) if bits >> 31 else bits
        rk.restkv_append(p.c, sides["k"].cuda(), sides["v"].cuda(), p.pages, p.tensors["table"], p.tensors["lens"])
        got, group = p.down(), torch.arange(d) % (d // 16) // 2
        ko, vo = (torch.empty((1, 1, n, d), device="cuda") for _ in range(2))
        rk.restkv_fetch(p.c, p.pages, p.tensors["table"], p.tensors["lens"], ko, vo)
        for name, x, back in (("k", sides["k"], ko), ("v", sides["v"], vo)):
            codes, scale = ref.to_q4(x[:, 0])
            for t in range(n):
                w, what = p.where(0, 0, t), (name, d, hex(patterns[t // 2]), t % 2)
                assert torch.equal(got[name][w], codes[t]), what
                assert torch.equal(torch.nan_to_num(got[name + "_scale"][w].float(), 777.0), torch.nan_to_num(scale[t].float(), 777.0)), what
                assert torch.equal(torch.isnan(back[0, 0, t]).cpu(), group == group[d // 2 + 2]), what
