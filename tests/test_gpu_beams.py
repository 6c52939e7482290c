"""Beams over the paged cache on the GPU: selection, reordering and shared attention against plain implementations in 64 bits
(tests/beams_ref.py, tests/pages_ref.py), at the sizes, masks, ties and page boundaries where they can go wrong, and the calls
together as they are used."""
import math

import pytest
import torch

import beams_ref as ref
import pages_ref
import paper_2605_08840_amd as rk

pytestmark = pytest.mark.gpu

Plain = pages_ref.Plain


# ---- selection ----------------------------------------------------------------------------------


def run_select(logits, scores, finished, n_out, end=2, in_place=False, stream=None):
    """logits [rows, vocab] on the GPU, any row stride; scores, finished on the CPU."""
    groups, beams = scores.shape
    b = rk.make_beams(n_groups=groups, n_beams=beams, n_vocab=logits.shape[1], n_out=n_out, dtype=logits.dtype, end_token=end,
                      logit_stride=logits.stride(0) if logits.shape[0] > 1 else 0)
    ws = rk.alloc_beam_workspace(b)
    ws.fill_(255)                                          # whatever it holds
    sc, fn = scores.cuda(), None if finished is None else finished.int().cuda()
    ns = sc if in_place else torch.full((groups, n_out), 7.0, device="cuda")
    nf = fn if in_place and fn is not None else torch.full((groups, n_out), 7, dtype=torch.int32, device="cuda")
    parents, tokens = (torch.full((groups, n_out), 7, dtype=torch.int32, device="cuda") for _ in range(2))
    rk.restkv_beam_select(b, logits, sc, ns, parents, tokens, ws, finished=fn, new_finished=nf, stream=stream)
    return tuple(x.cpu() for x in (ns, parents, tokens, nf))


def check_select(logits, scores, finished, n_out, end=2, **more):
    got = run_select(logits.cuda() if not logits.is_cuda else logits, scores, finished, n_out, end, **more)
    ref.assert_select(got, ref.select(logits.cpu(), scores, finished, n_out, end), logits.shape[1])
    return got


SELECTS = [
    # groups, beams, vocab, n_out
    (1, 1, 1, 1), (1, 1, 1, 4), (2, 3, 5, 8), (3, 2, 63, 2), (1, 4, 1000, 8), (2, 5, 4095, 5), (2, 3, 4096, 64), (1, 2, 4097, 3),
    (1, 3, 8191, 6), (2, 2, 8200, 33), (1, 4, 20011, 16), (2, 64, 700, 64), (70, 1, 300, 1), (1, 16, 50257, 32), (1, 1, 200000, 64),
    (300, 2, 40, 7),
]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("groups,beams,vocab,n_out", SELECTS)
def test_select(groups, beams, vocab, n_out, dtype):
    g = torch.Generator().manual_seed(groups + beams + vocab)
    logits = (3 * torch.randn((groups * beams, vocab), generator=g)).to(dtype)
    scores = -10 * torch.rand((groups, beams), generator=g)
    check_select(logits, scores, None, n_out)
    ended = torch.rand((groups, beams), generator=g) < 0.4
    check_select(logits, scores, ended, n_out, end=vocab - 1)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("shift,pad", [(1, 0), (3, 5), (0, 1), (2, 2), (7, 9)])
def test_select_rows_at_any_address(dtype, shift, pad):
    """Rows that begin at no 16-byte address; large logits before, between and behind them."""
    vocab, rows = 5003, 6
    g = torch.Generator().manual_seed(shift)
    flat = torch.full((shift + rows * (vocab + pad) + 16,), 1e4, dtype=dtype)
    view = flat[shift:shift + rows * (vocab + pad)].view(rows, vocab + pad)[:, :vocab]
    view.copy_(torch.randn((rows, vocab), generator=g))
    d = flat.cuda()
    check_select(d[shift:shift + rows * (vocab + pad)].view(rows, vocab + pad)[:, :vocab], torch.rand((2, 3), generator=g), None, 9)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_select_ties(dtype):
    """Equal logits: the lower token; equal beams: the lower beam; -0 and 0 are equal; any number of them."""
    for vocab, n_out in ((9000, 64), (40, 64), (30000, 5)):
        x = torch.zeros((4, vocab), dtype=dtype)
        x[1, ::2] = -0.0
        got = check_select(x, torch.zeros((2, 2)), None, n_out)
        assert got[2][0].tolist() == (list(range(min(n_out, vocab))) + list(range(n_out - min(n_out, vocab))))[:n_out]
        x = torch.randint(-3, 4, (4, vocab), generator=torch.Generator().manual_seed(1)).to(dtype)     # few different values
        x[1] = x[0]
        check_select(x, torch.full((2, 2), -1.5), None, n_out)
        x = torch.arange(vocab).to(dtype).expand(4, -1).contiguous() / 64                              # all large ones together
        check_select(x, torch.tensor([[0.0, 0.0], [-1.0, 0.0]]), None, n_out)
        check_select(x.flip(1).contiguous(), torch.zeros((2, 2)), None, n_out)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_select_beams_far_apart(dtype):
    """One beam far ahead of many others, over many pieces of its row: nearly all is its own; and two that overlap."""
    g = torch.Generator().manual_seed(11)
    x = torch.randn((32, 60000), generator=g).to(dtype)
    scores = -50 - 10 * torch.rand((2, 16), generator=g)
    scores[0, 3], scores[1, 5], scores[1, 9] = 0, 0, -0.5
    for n_out in (5, 64):
        got = check_select(x, scores, None, n_out)
        assert (got[1][0] == 3).all() and set(got[1][1].tolist()) <= {5, 9}


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_select_masks_and_unusual_values(dtype):
    g = torch.Generator().manual_seed(3)
    vocab, low = 6000, torch.finfo(dtype).min
    x = torch.randn((14, vocab), generator=g).to(dtype)
    x[0] = -math.inf                                       # nothing is allowed
    x[1, torch.randperm(vocab, generator=g)[3:]] = -math.inf      # three tokens are
    x[2, 1:] = -math.inf
    x[3, :-1] = low                                        # masked with the lowest value: still candidates
    x[4] = low
    x[5, 77] = math.nan
    x[6, 78] = math.inf
    x[7, 5], x[7, 6] = 1e30, 9e29
    x[8] *= 1e-30
    x[9, 4000:] = -math.inf
    scores = torch.tensor([[0.0, -1.0], [-2.0, -3.0], [-0.5, -0.25], [-1.0, -1.0], [-4.0, -1.0], [-math.inf, -2.0], [math.nan, math.inf]])
    for n_out in (2, 6, 64):
        got = check_select(x, scores, None, n_out)
        assert 1 not in got[1][2] and 0 not in got[1][3] and (got[1][6] == -1).all()      # (rows 5 and 6)
    # all ended, some without a score
    ended = torch.ones((7, 2), dtype=torch.int32)
    got = check_select(x, scores, ended, 4)
    assert got[1][0].tolist() == [0, 1, -1, -1] and got[2][0].tolist() == [2, 2, -1, -1] and got[3][0].tolist() == [1, 1, 1, 1]
    assert got[1][5].tolist() == [1, -1, -1, -1] and (got[1][6] == -1).all()
    # the first step: one beam stands for all
    first = torch.full((7, 2), -math.inf)
    first[:, 0] = 0
    check_select(x, first, None, 8)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_select_scores_that_float32_does_not_hold(dtype):
    """Logits so far apart that a score is finite in 64 bits, and none as it is given out: such a token is not taken."""
    low, top = torch.finfo(dtype).min, torch.finfo(dtype).max
    x = torch.full((4, 100), low, dtype=dtype)
    x[0, 5], x[1, 50], x[2, 7], x[3, 99] = top, top / 2, 0.0, top
    scores = torch.tensor([[0.0, -1.0], [-2.0, -3e38]])
    got = check_select(x, scores, None, 6)
    assert got[2][0].tolist() == [5, 50, -1, -1, -1, -1] and got[1][0].tolist() == [0, 1, -1, -1, -1, -1]


def test_select_largest_vocabulary_and_two_calls_at_once():
    vocab = 1 << 24
    g = torch.Generator(device="cuda").manual_seed(2)
    x = torch.randn((3, vocab), generator=g, device="cuda").bfloat16()
    x[2, vocab - 1] = 40.0
    check_select(x[:1], torch.zeros((1, 1)), None, 64)
    got = check_select(x[1:], torch.tensor([[-0.5, -0.25]]), None, 64, end=vocab - 1)
    assert got[2][0, 0] == vocab - 1 and got[3][0, 0] == 1
    rows = [torch.randn((8, 5000), generator=g, device="cuda") for _ in range(2)]
    scores = -torch.rand((2, 4), generator=torch.Generator().manual_seed(1))
    want = [run_select(r, scores, None, 16) for r in rows]
    b = rk.make_beams(n_groups=2, n_beams=4, n_vocab=5000, n_out=16, dtype="f32", end_token=2)
    streams, outs = [torch.cuda.Stream() for _ in rows], []
    for _ in rows:
        outs.append((torch.empty((2, 16), device="cuda"), *(torch.empty((2, 16), dtype=torch.int32, device="cuda") for _ in range(2)),
                     rk.alloc_beam_workspace(b)))
    sc = scores.cuda()
    torch.cuda.synchronize()
    for _ in range(20):
        for r, s, o in zip(rows, streams, outs):
            rk.restkv_beam_select(b, r, sc, *o, stream=s)
    torch.cuda.synchronize()
    for o, w in zip(outs, want):
        assert all(torch.equal(x.cpu(), y) for x, y in zip(o[:3], w))


def test_select_of_no_groups():
    b = rk.make_beams(n_groups=0, n_beams=4, n_vocab=50, dtype="f32")
    f, i = torch.empty((0, 4), device="cuda"), torch.empty((0, 4), dtype=torch.int32, device="cuda")
    rk.restkv_beam_select(b, torch.empty((0, 50), device="cuda"), f, f.clone(), i, i.clone(), rk.alloc_beam_workspace(b))
    torch.cuda.synchronize()


def test_select_in_place_and_on_another_stream():
    g = torch.Generator().manual_seed(5)
    x, scores = torch.randn((12, 3001), generator=g), -torch.rand((3, 4), generator=g)
    ended = torch.rand((3, 4), generator=g) < 0.4
    want = check_select(x, scores, ended, 4)
    got = run_select(x.cuda(), scores, ended, 4, in_place=True)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    xd, s = x.cuda(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        got = run_select(xd, scores, ended, 4, stream=s)
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_select_many_rows_and_large_rows():
    """More rows than one grid dimension takes is not tested here, but rows beyond 4 GiB and a vocabulary of millions are."""
    vocab, stride = 3_000_001, 2 ** 30 + 24                # the second row lies 4 GiB further
    flat = torch.zeros(stride + vocab, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(1)
    rows = torch.as_strided(flat, (2, vocab), (stride, 1))
    rows.copy_(torch.randn((2, vocab), generator=g, device="cuda"))
    check_select(rows, torch.tensor([[0.0, -0.1]]), None, 64)


def test_binding_refuses_wrong_select_tensors():
    b = rk.make_beams(n_groups=2, n_beams=3, n_vocab=50, dtype="f32")
    ws = rk.alloc_beam_workspace(b)
    x, f, i = torch.zeros((6, 50), device="cuda"), torch.zeros((2, 3), device="cuda"), torch.zeros((2, 3), dtype=torch.int32, device="cuda")
    good = dict(logits=x, scores=f, new_scores=f.clone(), parents=i, tokens=i.clone(), workspace=ws)
    rk.restkv_beam_select(b, **good)
    rk.restkv_beam_select(b, **{**good, "logits": x.view(2, 3, 50)})
    for name, bad in (("logits", x.bfloat16()), ("logits", x[:5]), ("logits", torch.zeros((6, 51), device="cuda")[:, :50]), ("logits", x.t()),
                      ("logits", x.cpu()), ("scores", f[:, :2]), ("scores", f.double()), ("parents", i.long()), ("tokens", i.cpu()),
                      ("new_scores", f.t()), ("workspace", None), ("workspace", ws[:300]), ("workspace", ws.cpu())):
        with pytest.raises(rk.RestkvError):
            rk.restkv_beam_select(b, **{**good, name: bad})
    for name in ("finished", "new_finished"):
        with pytest.raises(rk.RestkvError):
            rk.restkv_beam_select(b, **good, **{name: f})
    torch.cuda.synchronize()


# ---- reordering ---------------------------------------------------------------------------------


def check_reorder(p, n_beams, parents, layers=2, in_place=False, wide=0):
    """parents: per group a list.  Pools of several layers from one: each with other values."""
    pools = [{n: (x if not i else x.roll(i, 0)) for n, x in p.pool.items()} for i in range(layers)]
    def up(q):
        return rk.CachePages(pages_ref.pack(q["k"]).cuda(), pages_ref.pack(q["v"]).cuda(), q["k_scale"].cuda(), q["v_scale"].cuda()) \
            if p.q4 else rk.CachePages(q["k"].cuda(), q["v"].cuda())
    dev = [up(q) for q in pools]
    par = torch.tensor([x + [99] * wide for x in parents], dtype=torch.int32).cuda()[:, :n_beams]
    table = p.tensors["table"].clone()
    out = table if in_place else torch.full_like(table, -7)
    rk.restkv_beam_reorder(p.c, n_beams, par, table, p.tensors["lens"], rk.CacheLayers(dev) if layers != 1 else dev, None if in_place else out)
    want_table, moves = p.table.clone(), []
    heads = p.hkv if p.head_tables else 1
    most = p.c.max_len or p.width * p.ps
    for g, par_g in enumerate(parents):
        s0 = g * n_beams
        lens = [max(0, min(x, most)) for x in p.lens[s0]]
        for h in range(heads):
            mine = lens if heads == 1 else [lens[h]]
            lo, hi = min(mine) // p.ps, -(-max(mine) // p.ps)
            for b, (parent, giver) in enumerate(ref.deal(par_g, n_beams)):
                want_table[s0 + b, h, :lo] = p.table[s0 + parent, h, :lo]
                want_table[s0 + b, h, lo:hi] = p.table[s0 + giver, h, lo:hi]
                if giver != parent:
                    for col in range(lo, hi):
                        src, dst = int(p.table[s0 + parent, h, col]), int(p.table[s0 + giver, h, col])
                        if 0 <= src < p.c.n_pages and 0 <= dst < p.c.n_pages:
                            for x in range(p.hkv) if heads == 1 else [h]:
                                moves.append((src, dst, 0 if heads > 1 else x, max(0, min(lens[x] - col * p.ps, p.ps))))
    got_table = out.cpu().reshape(want_table.shape)
    assert torch.equal(got_table, want_table)
    for q, d in zip(pools, dev):
        want = {n: x.clone() for n, x in q.items()}
        for src, dst, h, n in moves:
            for x in want.values():
                if p.token_major:
                    x[dst, :n, h] = x[src, :n, h]
                else:
                    x[dst, h, :n] = x[src, h, :n]
        got = dict(k=d.k.cpu(), v=d.v.cpu())
        if p.q4:
            got = dict(k=pages_ref.unpack(got["k"]), v=pages_ref.unpack(got["v"]), k_scale=d.k_scale.cpu(), v_scale=d.v_scale.cpu())
        for n in want:
            bits = {1: torch.uint8, 2: torch.int16, 4: torch.int32}[want[n].element_size()]
            assert torch.equal(got[n].view(bits), want[n].view(bits)), n
    return got_table


REORDERS = [
    # positions of each group (per head: a list), n_beams, parents of each group, what
    ([17], 1, [[0]], dict()),
    ([17], 2, [[1, 1]], dict()),
    ([15, 16, 1, 0, 33], 4, [[0, 0, 1, 1], [3, 2, 1, 0], [2, 2, 2, 2], [1, 1, 0, 3], [0, 1, 2, 3]], dict(room=2)),
    ([40, 31], 3, [[2, 0, 0], [1, 2, 2]], dict(d=128, ps=32, token_major=True)),
    ([20, 64], 5, [[-1, 9, 1, 1, 2 ** 31 - 1], [4, 4, -5, 0, 0]], dict(hq=6, hkv=3)),          # entries that are none
    ([[5, 40], [33, 20], [16, 16]], 4, [[0, 0, 0, 0], [3, 3, 1, 1], [1, 0, 0, 2]], dict(head_lens=True, room=1)),
    ([[50, 0, 3], [17, 32, 90]], 3, [[1, 1, 1], [2, 2, 0]], dict(hq=6, hkv=3, d=128, head_lens=True)),
    ([[50, 0, 3], [17, 32, 90]], 3, [[1, 1, 1], [2, 2, 0]], dict(hq=3, hkv=3, head_lens=True, head_tables=True, room=1)),
    ([[50, 50, 50], [17, 17, 17]], 3, [[1, 1, 1], [2, 2, 0]], dict(hq=3, hkv=3, head_tables=True, room=1)),
    ([37], 64, [[(7 * b) % 11 for b in range(64)]], dict(hkv=1, hq=1)),
    ([200], 2, [[0, 0]], dict(max_len=150, ps=64)),                                            # longer than the room
    ([90, 3], 2, [[1, 1], [0, 0]], dict(hkv=8, hq=8, d=128, ps=64)),
]


@pytest.mark.parametrize("dtype,fmt", [("f32", None), ("bf16", None), ("bf16", "q4")])
@pytest.mark.parametrize("lens,n_beams,parents,more", REORDERS)
def test_reorder(lens, n_beams, parents, more, dtype, fmt):
    p = Plain(rk, lens=[x for x in lens for _ in range(n_beams)], new=[0] * (len(lens) * n_beams), dtype=dtype, fmt=fmt, seed=len(lens), **more)
    if p.width > 1 and "room" in more:      # pages for what is to come
        p.table[p.table == 2 ** 30] = 0
        p.tensors["table"] = (p.table if p.head_tables else p.table[:, 0]).contiguous().cuda()
    a = check_reorder(p, n_beams, parents)
    b = check_reorder(p, n_beams, parents, layers=1, in_place=True, wide=3)
    assert torch.equal(a, b)


def test_reorder_of_many_layers_groups_and_columns():
    """More layers than a launch takes addresses for, more groups and table entries than a wavefront has lanes."""
    p = Plain(rk, lens=[19] * 210, new=[0] * 210, hq=1, hkv=1, room=70)
    g = torch.Generator().manual_seed(2)
    check_reorder(p, 3, torch.randint(0, 3, (70, 3), generator=g).tolist(), layers=5)
    p = Plain(rk, lens=[19] * 2, new=[0] * 2, hq=1, hkv=1)
    check_reorder(p, 2, [[1, 1]], layers=70)
    check_reorder(p, 2, [[1, 1]], layers=0)


def test_reorder_leaves_pages_that_are_none():
    p = Plain(rk, lens=[20] * 6, new=[0] * 6, spare=0)
    p.table[0, 0, 1], p.table[4, 0, 1] = -1, 10 ** 6
    p.tensors["table"] = p.table[:, 0].contiguous().cuda()
    check_reorder(p, 3, [[0, 0, 1], [0, 0, 2]])


def test_reorder_large_pages():
    """Pages of thousands of positions, and shared by heads of very different lengths."""
    p = Plain(rk, lens=[[1500, 3], [1500, 3]], new=[0, 0], ps=1024, head_lens=True, hq=2, hkv=2)
    check_reorder(p, 2, [[1, 1]])


def test_binding_refuses_wrong_reorder_tensors():
    p = Plain(rk, lens=[20] * 4, new=[0] * 4)
    par = torch.zeros((2, 2), dtype=torch.int32, device="cuda")
    t = p.tensors
    rk.restkv_beam_reorder(p.c, 2, par, t["table"], t["lens"], [p.pages])
    other = rk.CachePages(p.pages.k.float(), p.pages.v.float())
    for args in ((2, par.long()), (2, par[:1]), (2, par.cpu()), (4, par), (3, par), (0, par), (2, par[:, :1].expand(2, 2))):
        with pytest.raises(rk.RestkvError):
            rk.restkv_beam_reorder(p.c, *args, t["table"], t["lens"], [p.pages])
    for tb, ln, la, to in ((t["table"].long(), t["lens"], [p.pages], None), (t["table"], t["lens"][:3], [p.pages], None),
                           (t["table"], t["lens"], [other], None), (t["table"], t["lens"], [p.pages], t["table"].cpu())):
        with pytest.raises(rk.RestkvError):
            rk.restkv_beam_reorder(p.c, 2, par, tb, ln, la, to)
    torch.cuda.synchronize()


# ---- attention ----------------------------------------------------------------------------------

FORMATS = [("f32", None, None), ("bf16", None, None), ("bf16", None, "f32"), ("bf16", "q4", None), ("f32", "q4", None)]


@pytest.fixture
def shared_once():
    """Shared pages read once, however short the caches are."""
    rk.restkv_debug_force_shared(True)
    yield
    rk.restkv_debug_force_shared(False)


def share(p, n_beams, shared):
    """The first shared[g] pages of each group (per head, with tables per head): those of its longest sequence, in all tables."""
    for g, n in enumerate(shared):
        of = range(g * n_beams, (g + 1) * n_beams)
        for h in range(p.table.shape[1]):
            long = max(of, key=lambda s: p.lens[s][h] if p.head_tables else max(p.lens[s]))
            for s in of:
                p.table[s, h, :max(n, 0)] = p.table[long, h, :max(n, 0)].clone()
    p.tensors["table"] = (p.table if p.head_tables else p.table[:, 0]).contiguous().cuda()
    return torch.tensor(shared, dtype=torch.int32).cuda()


def run_beams(p, n_beams, shared, q, out_type, lse=True, **more):
    out = torch.full((p.tokens, p.hq, p.d), 5.0, dtype=out_type, device="cuda")
    l = torch.full((p.tokens, p.hq), 5.0, dtype=torch.float32, device="cuda") if lse else None
    ws = rk.alloc_attend_beams_workspace(p.c, n_beams)
    if ws is not None:
        ws.fill_(255)
    rk.restkv_attend_beams(p.c, n_beams, shared, q.cuda(), p.pages, p.tensors["table"], p.tensors["lens"], out, l, ws,
                           new_start=p.tensors["new_start"], **more)
    return out.cpu(), None if l is None else l.cpu()


def check_beams(p, n_beams, shared, q, out_type, causal=True, scale=None):
    got, lse = run_beams(p, n_beams, shared, q, out_type)
    rows = [t for s, n in enumerate(p.new) for t in range(p.start[s], p.start[s] + min(n, p.c.max_new))]
    pages_ref.assert_attention(got, lse, pages_ref.attention(p, q, scale=scale, causal=causal), out_type, rows)
    rest = [t for t in range(p.tokens) if t not in set(rows)]
    assert (got[rest] == 5.0).all() and (lse[rest] == 5.0).all()
    return got, lse


ATTENDS = [
    # lens, new, n_beams, shared pages of each group, what
    ([1], [1], 1, [0], dict()),
    ([70, 70], [1, 1], 2, [4], dict()),
    ([65, 66, 80, 64], [1, 1, 1, 1], 4, [4], dict(d=128)),                              # a tail of one position, and of none in front
    ([130, 131, 140], [1] * 3, 3, [8], dict(hq=2, hkv=2)),
    ([300, 333, 290, 700], [1] * 4, 2, [16, 17], dict(d=128, hq=8, hkv=2)),
    ([300] * 4 + [40] * 4, [1] * 8, 4, [18, 0], dict(d=128, hq=8, hkv=2)),              # 16 rows; a group that shares nothing
    ([400] * 8, [1] * 8, 8, [25], dict(d=128, hq=8, hkv=2, ps=16)),                     # 32 rows; more pages than may be shared
    ([500, 513, 600, 512, 530, 700, 801, 520, 519], [1] * 9, 9, [31], dict(hq=8, hkv=1, d=128)),      # 72 rows
    ([260] * 20, [1] * 20, 20, [4], dict(hq=14, hkv=2, d=128, ps=64)),                  # 140 rows
    ([210] * 64, [1] * 64, 64, [12], dict(hq=2, hkv=1)),
    ([150, 170, 190], [3, 1, 7], 3, [9], dict(hq=6, hkv=2, token_major=True)),          # several new tokens
    ([150, 170, 190, 80], [30, 0, 7, 20], 2, [5, 3], dict(hq=6, hkv=2)),                # a beam without new tokens
    ([0, 170, 190, 0], [0, 1, 1, 0], 2, [8, 9], dict(hq=4, hkv=2, d=128)),
    ([0, 70, 190, 0], [1, 1, 2, 1], 2, [4, 4], dict(hq=4, hkv=2, d=128)),               # a beam that sees nothing
    ([150, 170], [40, 60], 2, [9], dict(hq=6, hkv=2, causal=False)),
    ([[90, 240], [95, 250], [333, 20], [340, 30]], [1] * 4, 2, [5, 20], dict(head_lens=True)),
    ([[90, 40, 300], [99, 45, 310]], [1, 2], 2, [17], dict(hq=6, hkv=3, d=128, head_lens=True, head_tables=True)),
    ([90, 140, 130], [1, 2, 1], 3, [5], dict(hq=6, hkv=3, head_tables=True)),
    ([200, 220], [1, 1], 2, [12], dict(scale=0.31, max_len=150)),                       # longer than the room
    ([200, 260], [90, 20], 2, [6], dict(max_new=33, room=3)),                           # the first 33 of 90
    ([170, 200], [2, 2], 2, [-3], dict(extra_tokens=3)),                                # a count below 0
    ([300] * 2, [1] * 2, 2, [2 ** 31 - 1], dict(d=128)),
    ([100] * 140, [1] * 140, 2, [6] * 70, dict(hq=2, hkv=1)),                           # more groups than lanes
    ([130] * 40, [1] * 40, 4, [8] * 10, dict(hq=4, hkv=4, d=128)),
    ([90 + 7 * i for i in range(96)], [i % 3 for i in range(96)], 3, [i % 9 for i in range(32)], dict(hq=6, hkv=2)),     # lengths that differ
    ([[90 + i, 300 - 3 * i] for i in range(40)], [1] * 40, 5, [5, 0, 9, 3, 1, 2, 4, 8], dict(head_lens=True, head_tables=True)),
    ([260 + i for i in range(66)], [1] * 66, 33, [16, 12], dict(hq=8, hkv=2, d=128)),                                    # 132 rows
    ([200, 290] * 20, [20, 31] * 20, 2, [8] * 20, dict(hq=4, hkv=2)),                                                    # blocks of rows of both kinds
    ([900] * 3 + [5] * 66, [1] * 69, 3, [50] + [0] * 22, dict(hq=4, hkv=2)),                                             # one long group among short ones
]


@pytest.mark.parametrize("dtype,fmt,out", FORMATS)
@pytest.mark.parametrize("lens,new,n_beams,shared,more", ATTENDS)
def test_attend_beams(lens, new, n_beams, shared, more, dtype, fmt, out, shared_once):
    p = Plain(rk, lens=lens, new=new, dtype=dtype, fmt=fmt, out_dtype=out, seed=sum(new), **more)
    out_type = torch.float32 if "f32" in (dtype, out) else torch.bfloat16
    sh = share(p, n_beams, [min(n, p.width) for n in shared])
    if max(shared) > p.width:
        sh.fill_(shared[0])
    q = (p.normal(p.tokens, p.hq, p.d) * 2).to(p.type)
    check_beams(p, n_beams, sh, q, out_type, causal=more.get("causal", True), scale=more.get("scale"))
    if sum(new) % 3 == 0:                                  # and as the sizes have it
        rk.restkv_debug_force_shared(False)
        check_beams(p, n_beams, sh, q, out_type, causal=more.get("causal", True), scale=more.get("scale"))


@pytest.mark.parametrize("dtype,fmt,out", FORMATS)
def test_attend_beams_long(dtype, fmt, out, shared_once):
    """Many chunks of the shared pages and of the beams' own, against restkv_attend, which reads every beam's."""
    for lens, n_beams, new, hq, hkv in (([5000, 5100, 6000, 4999], 4, 1, 8, 2), ([3000 + 37 * i for i in range(24)], 12, 2, 8, 2),
                                        ([9000] * 3 + [700] * 3, 3, 1, 4, 1)):
        p = Plain(rk, lens=[65] * len(lens), new=[new] * len(lens), dtype=dtype, fmt=fmt, out_dtype=out, d=128, hq=hq, hkv=hkv, ps=64)
        width = max(lens) // 64 + 1
        n_pages = width * len(lens)
        c = rk.make_cache(n_seqs=len(lens), n_q_heads=hq, n_kv_heads=hkv, head_dim=128, page_size=64, n_pages=n_pages, max_pages=width,
                          dtype=p.type, format=fmt, out_dtype=out, max_new=new)
        g = torch.Generator(device="cuda").manual_seed(4)
        rnd = lambda *s, t=p.type: torch.randn(s, generator=g, device="cuda").to(t)  # noqa: E731
        if fmt:
            step = torch.rand((2, n_pages, hkv, 64, 4, 1), generator=g, device="cuda") * 0.3 + 0.05
            sc = torch.cat((step, -8 * step), -1).bfloat16()
            codes = torch.randint(256, (2, n_pages, hkv, 64, 64), generator=g, device="cuda", dtype=torch.uint8)
            pages = rk.CachePages(codes[0], codes[1], sc[0], sc[1])
        else:
            pages = rk.CachePages(rnd(n_pages, hkv, 64, 128), rnd(n_pages, hkv, 64, 128))
        table = torch.randperm(n_pages, generator=g, device="cuda").int().view(len(lens), width)
        shared = [(min(lens[i:i + n_beams]) - new) // 64 for i in range(0, len(lens), n_beams)]
        for i, n in enumerate(shared):
            table[i * n_beams:(i + 1) * n_beams, :n] = table[i * n_beams, :n].clone()
        ln, sh = torch.tensor(lens, dtype=torch.int32).cuda(), torch.tensor(shared, dtype=torch.int32).cuda()
        q = rnd(len(lens) * new, hq, 128) * 2
        out_type = torch.float32 if "f32" in (dtype, out) else torch.bfloat16
        got, want = (torch.empty(q.shape, dtype=out_type, device="cuda") for _ in range(2))
        l1, l2 = (torch.empty(q.shape[:2], device="cuda") for _ in range(2))
        rk.restkv_attend_beams(c, n_beams, sh, q, pages, table, ln, got, l1, rk.alloc_attend_beams_workspace(c, n_beams))
        rk.restkv_attend(c, q, pages, table, ln, want, l2, rk.alloc_attend_workspace(c))
        # two answers, each within: weights to 2^-17 (float32: 2^-24) and rounding of the output by half a step, logits and sums over some
        # hundred chunks to 300 half steps of float32, of outputs that are sums of weights times values below 6
        half = torch.finfo(out_type).eps / 2
        tol = 2 * half * want.abs().float() + 2 * 6 * (300 * 2.0 ** -24 + (2.0 ** -17 if out_type == torch.bfloat16 else 2.0 ** -24))
        assert ((got.float() - want.float()).abs() <= tol).all(), ((got.float() - want.float()).abs() - tol).max().item()
        assert ((l1 - l2).abs() <= 2 * 300 * 2.0 ** -24 + 2.0 ** -23 * l2.abs()).all()


def long_case(fmt, n_beams, lens, width, ps, n_pages, hq, hkv, shared, d=64, seed=7):
    """restkv_attend_beams beside restkv_attend over pages of 65536 positions or so, made on the GPU."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    c = rk.make_cache(n_seqs=len(lens), n_q_heads=hq, n_kv_heads=hkv, head_dim=d, page_size=ps, n_pages=n_pages, max_pages=width, dtype="bf16",
                      format=fmt)
    pages = rk.alloc_cache_pages(c)
    for x in (pages.k, pages.v):
        x.random_(0, 256, generator=g) if fmt else x.normal_(generator=g)
    if fmt:
        for x in (pages.k_scale, pages.v_scale):
            x.copy_(torch.tensor([0.25, -2.0], dtype=torch.bfloat16))
    table = torch.full((len(lens), width), -1, dtype=torch.int32)
    free = list(range(n_pages - 1, -1, -1))
    for s, n in enumerate(lens):
        for i in range(-(-n // ps)):
            first = s // n_beams * n_beams
            table[s, i] = table[first, i] if s != first and i < shared[s // n_beams] else free.pop()
    table, ln = table.cuda(), torch.tensor(lens, dtype=torch.int32).cuda()
    q = torch.randn((len(lens), hq, d), generator=g, device="cuda").bfloat16()
    outs, lses = [torch.empty(q.shape, dtype=q.dtype, device="cuda") for _ in range(2)], [torch.empty(q.shape[:2], device="cuda") for _ in range(2)]
    sh = torch.tensor(shared, dtype=torch.int32).cuda()
    rk.restkv_attend_beams(c, n_beams, sh, q, pages, table, ln, outs[0], lses[0], rk.alloc_attend_beams_workspace(c, n_beams))
    rk.restkv_attend(c, q, pages, table, ln, outs[1], lses[1], rk.alloc_attend_workspace(c))
    a, b = (x.float() for x in outs)
    # outputs of below 2^2 in size: half a step each, weights to 2^-17, sums of some thousand tiles to 2^-13 of values below 8 at the most
    assert ((a - b).abs() <= 2.0 ** -7 * b.abs() + 2 * 8 * (2.0 ** -17 + 2.0 ** -13)).all(), (a - b).abs().max().item()
    assert ((lses[0] - lses[1]).abs() <= 2 * 2.0 ** -13 + 2.0 ** -22 * lses[1].abs()).all()


@pytest.mark.parametrize("fmt", [None, "q4"])
def test_attend_beams_with_room_for_a_billion_positions(fmt, shared_once):
    """Tables that could hold 2^30 positions: the work is cut by what is there."""
    long_case(fmt, 2, [200001, 333333, 70, 65], 16384, 65536, 12, 4, 1, [2, 0])
    long_case(fmt, 40, [140000 + 31 * i for i in range(40)], 16384, 65536, 44 + 41, 8, 1, [2])
    long_case(fmt, 20, [70000] * 20 + [66000 + i for i in range(20)] + [3] * 20, 16384, 65536, 62 + 42, 2, 1, [1, 1, 0])


@pytest.mark.parametrize("fmt", [None, "q4"])
def test_beams_pages_that_pass_four_gigabytes(fmt, shared_once):
    """The last pages of arrays of more than 2^32 bytes: attention over them, and rows copied between them."""
    ps, d = 65536, 64
    many = (1 << 32) // (ps * (d // 2 if fmt else 2 * d)) + 6
    long_case(fmt, 2, [140000, 150000], 4, ps, many, 4, 1, [2])
    c = rk.make_cache(n_seqs=2, n_q_heads=1, n_kv_heads=1, head_dim=d, page_size=ps, n_pages=many, max_pages=2, dtype="bf16", format=fmt)
    pages = rk.alloc_cache_pages(c)
    g = torch.Generator(device="cuda").manual_seed(1)
    every = [x for x in (pages.k, pages.v, pages.k_scale, pages.v_scale) if x is not None]
    for x in every:
        for at in (many - 1, many - 2, 0, 1):
            x[at].random_(0, 100, generator=g) if x.dtype is torch.uint8 else x[at].normal_(generator=g)
    before = [x[[many - 1, many - 2, 0, 1]].clone() for x in every]
    table = torch.tensor([[0, many - 2], [1, many - 1]], dtype=torch.int32).cuda()
    n = 65536 + 12345
    rk.restkv_beam_reorder(c, 2, torch.tensor([[0, 0]], dtype=torch.int32).cuda(), table, torch.tensor([n, n], dtype=torch.int32).cuda(), [pages])
    assert table.tolist() == [[0, many - 2], [0, many - 1]]
    for x, b in zip(every, before):
        b[0][:, :n - ps] = b[1][:, :n - ps]
        assert torch.equal(x[[many - 1, many - 2, 0, 1]].view(torch.uint8), b.view(torch.uint8))


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("dtype,fmt", [("f32", None), ("bf16", None), ("bf16", "q4")])
def test_what_beams_do_not_see_has_no_influence(dtype, fmt, bad, shared_once):
    """Junk behind the lengths, in the same pages as what is seen; a page that is not there, in front and behind."""
    p = Plain(rk, lens=[133, 140, 150, 129], new=[1, 3, 1, 1], dtype=dtype, fmt=fmt, junk=bad, hq=8, hkv=2)
    sh = share(p, 4, [8])
    p.table[:, 0, 3] = -1
    p.table[2, 0, 8] = 10 ** 6
    p.tensors["table"] = p.table[:, 0].contiguous().cuda()
    check_beams(p, 4, sh, p.normal(p.tokens, 8, 64).to(p.type), p.type)


def test_attend_beams_strided_and_without_lse(shared_once):
    p = Plain(rk, lens=[133, 140, 150, 129], new=[1, 3, 1, 1], hq=8, hkv=2, d=128)
    sh = share(p, 2, [8, 6])
    wide = p.normal(p.tokens, 1 + 8 * 128 + 7).bfloat16()
    q = wide[:, 1:1 + 1024].unflatten(1, (8, 128))
    want, _ = check_beams(p, 2, sh, q.contiguous(), torch.bfloat16)
    back = torch.full((8, p.tokens, 129), 5.0, dtype=torch.bfloat16, device="cuda")
    out = back[:, :, 1:].transpose(0, 1)
    ws = rk.alloc_attend_beams_workspace(p.c, 2)
    rk.restkv_attend_beams(p.c, 2, sh, wide.cuda()[:, 1:1 + 1024].unflatten(1, (8, 128)), p.pages, p.tensors["table"], p.tensors["lens"], out,
                           None, ws, new_start=p.tensors["new_start"])
    assert torch.equal(out.cpu(), want) and (back[:, :, 0] == 5.0).all()


def test_attend_beams_two_calls_at_once_and_on_another_stream(shared_once):
    p = Plain(rk, lens=[700, 720, 650, 900], new=[2, 1, 1, 1], d=128, hq=8, hkv=2)
    sh = share(p, 2, [40, 39])
    q = p.normal(p.tokens, 8, 128).bfloat16().cuda()
    streams, outs = [torch.cuda.Stream() for _ in range(2)], [torch.empty_like(q) for _ in range(3)]
    ws, t = [rk.alloc_attend_beams_workspace(p.c, 2) for _ in range(2)], p.tensors
    call = lambda i, w, **k: rk.restkv_attend_beams(p.c, 2, sh, q, p.pages, t["table"], t["lens"], outs[i], None, w, new_start=t["new_start"], **k)  # noqa: E731
    call(2, ws[0])
    torch.cuda.synchronize()
    for _ in range(20):
        for i, s in enumerate(streams):
            call(i, ws[i], stream=s)
    torch.cuda.synchronize()
    assert torch.equal(outs[0], outs[2]) and torch.equal(outs[1], outs[2])


MANY = dict(lens=[300 + 11 * i for i in range(72)], new=[1] * 72, hq=8, hkv=2, d=128)          # more parts than a wavefront has lanes


@pytest.mark.parametrize("fmt", [None, "q4"])
@pytest.mark.parametrize("n_beams", [3, 24])
def test_attend_of_many_beams_at_once_and_replayed(n_beams, fmt, shared_once):
    """Calls by a list: two at a time, and captured, with other lengths and counts of shared pages at each replay."""
    p = Plain(rk, fmt=fmt, **MANY)
    sh = share(p, n_beams, [18] * (72 // n_beams))
    q, t = p.normal(p.tokens, 8, 128).bfloat16().cuda(), p.tensors
    outs, ws = [torch.empty_like(q) for _ in range(4)], [rk.alloc_attend_beams_workspace(p.c, n_beams) for _ in range(3)]
    call = lambda i, w, **k: rk.restkv_attend_beams(p.c, n_beams, sh, q, p.pages, t["table"], t["lens"], outs[i], None, w, **k)  # noqa: E731
    call(2, ws[0])
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(10):
        for i, s in enumerate(streams):
            call(i, ws[i], stream=s)
    torch.cuda.synchronize()
    assert torch.equal(outs[0], outs[2]) and torch.equal(outs[1], outs[2])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(3, ws[2])
    lens = t["lens"].clone()
    for i in range(5):
        t["lens"].copy_((lens - 37 * i * (torch.arange(72, device="cuda") % 3)).clamp_min(0))
        sh.copy_(torch.arange(72 // n_beams, device="cuda") * i % 18)
        outs[3].zero_()
        graph.replay()
        torch.cuda.synchronize()
        call(2, ws[0])
        torch.cuda.synchronize()
        assert torch.equal(outs[3], outs[2]), i


def test_workspaces_are_not_exceeded(shared_once):
    """Bytes behind a workspace of just the size that is asked for stay as they are."""
    def guarded(n):
        x = torch.full((n + 4096 + 256,), 0xA5, dtype=torch.uint8, device="cuda")
        off = -x.data_ptr() % 256
        return x, x[off:off + n], x[off + n:]

    cases = [(MANY, 3, 18), (MANY, 24, 18), (dict(lens=[700, 720, 650, 900], new=[2, 1, 1, 3], hq=8, hkv=2, d=128), 2, 39),
             (dict(lens=[333] * 20, new=[1] * 20, hq=14, hkv=2, d=64), 20, 20),
             (dict(lens=[[90 + i, 300 - 3 * i] for i in range(40)], new=[5] * 40, hq=16, hkv=2, head_lens=True), 5, 5)]
    for fmt in (None, "q4"):
        for kw, n_beams, shared in cases:
            p = Plain(rk, fmt=fmt, **kw)
            sh = share(p, n_beams, [shared] * (len(p.new) // n_beams))
            need = rk.restkv_attend_beams_workspace_bytes(p.c, n_beams)
            _, ws, rest = guarded(need)
            q = p.normal(p.tokens, p.hq, p.d).bfloat16().cuda()
            want, got, t = torch.empty_like(q), torch.empty_like(q), p.tensors
            for out, w in ((got, ws), (want, rk.alloc_attend_beams_workspace(p.c, n_beams))):
                rk.restkv_attend_beams(p.c, n_beams, sh, q, p.pages, t["table"], t["lens"], out, None, w, new_start=t["new_start"])
            assert (rest == 0xA5).all() and torch.equal(got, want)
    for groups, beams, vocab, n_out in ((3, 4, 20000, 8), (2, 12, 5001, 64), (1, 1, 9, 1)):
        for dtype in (torch.float32, torch.bfloat16):
            b = rk.make_beams(n_groups=groups, n_beams=beams, n_vocab=vocab, n_out=n_out, dtype=dtype)
            _, ws, rest = guarded(rk.restkv_beam_workspace_bytes(b))
            flat = torch.randn(groups * beams * vocab + 1, device="cuda").to(dtype)
            for at in (0, 1):                              # rows at 16-byte addresses, and not
                i32 = lambda: torch.empty((groups, n_out), dtype=torch.int32, device="cuda")  # noqa: E731
                rk.restkv_beam_select(b, flat[at:at + groups * beams * vocab].view(-1, vocab), torch.zeros((groups, beams), device="cuda"),
                                      torch.empty((groups, n_out), device="cuda"), i32(), i32(), ws)
                assert (rest == 0xA5).all()


# ---- together -----------------------------------------------------------------------------------


class Search:
    """A toy model of two layers, decoded with beams over the paged cache: a token's keys, values and queries are rows of tables,
    logits a product with the attention's output."""

    def __init__(self, fmt=None, groups=2, beams=3, vocab=501, prompt=37, room=40, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        hq, hkv, d, ps, layers = 4, 2, 64, 16, 2
        self.groups, self.beams, self.vocab, self.prompt, self.layers = groups, beams, vocab, prompt, layers
        rnd = lambda *s, t=torch.bfloat16: torch.randn(s, generator=g, device="cuda").to(t)  # noqa: E731
        self.k, self.v, self.q, self.out_w = rnd(layers, vocab, hkv, d), rnd(layers, vocab, hkv, d), rnd(layers, vocab, hq, d), rnd(layers, hq * d, vocab)
        self.prompts = torch.randint(3, vocab, (groups, prompt), generator=g, device="cuda")
        n, width = groups * beams, (prompt + room + ps - 1) // ps
        desc = dict(n_q_heads=hq, n_kv_heads=hkv, head_dim=d, page_size=ps, n_pages=n * width, max_pages=width, dtype="bf16", format=fmt)
        self.step_cache = rk.make_cache(n_seqs=n, **desc)
        self.fill_cache = rk.make_cache(n_seqs=n, max_new=prompt, n_tokens=groups * prompt, **desc)
        self.table = torch.randperm(n * width, generator=g, device="cuda").int().view(n, width)
        self.pages = [rk.alloc_cache_pages(self.step_cache) for _ in range(layers)]
        self.both = rk.CacheLayers(self.pages)
        self.lens = torch.zeros(n, dtype=torch.int32, device="cuda")
        self.shared = torch.full((groups,), prompt // ps, dtype=torch.int32, device="cuda")
        self.desc = rk.make_beams(n_groups=groups, n_beams=beams, n_vocab=vocab, dtype="f32", end_token=0)
        self.ws, self.aws = rk.alloc_beam_workspace(self.desc), rk.alloc_attend_beams_workspace(self.step_cache, beams)
        i32 = lambda: torch.zeros((groups, beams), dtype=torch.int32, device="cuda")  # noqa: E731
        self.scores, self.ended, self.parents, self.tokens = torch.zeros((groups, beams), device="cuda"), i32(), i32(), i32()
        self.attended = torch.empty((layers, n, hq, d), dtype=torch.bfloat16, device="cuda")

    def start(self):
        """The prompts into the pages of each group's first beam, and the others behind them."""
        starts = [0]
        for s in range(self.groups * self.beams):
            starts.append(starts[-1] + (self.prompt - 1 if s % self.beams == 0 else 0))
        lens = torch.tensor([(self.prompt - 1) * (s % self.beams == 0) for s in range(self.groups * self.beams)], dtype=torch.int32).cuda()
        flat = torch.zeros(self.groups * self.prompt, dtype=torch.long, device="cuda")
        flat[:self.groups * (self.prompt - 1)] = self.prompts[:, :-1].reshape(-1)
        for i in range(self.layers):
            rk.restkv_append(self.fill_cache, self.k[i][flat], self.v[i][flat], self.pages[i], self.table, lens,
                             new_start=torch.tensor(starts, dtype=torch.int32).cuda())
        self.lens.fill_(self.prompt - 1)
        self.parents.zero_()
        rk.restkv_beam_reorder(self.step_cache, self.beams, self.parents, self.table, self.lens, self.both)
        self.scores.fill_(-math.inf)
        self.scores[:, 0] = 0
        self.ended.zero_()
        self.tokens.copy_(self.prompts[:, -1:].expand(-1, self.beams))

    def step(self):
        at = self.tokens.reshape(-1).clamp_min(0).long()
        self.lens.add_(1)
        logits = 0
        for i in range(self.layers):
            rk.restkv_append(self.step_cache, self.k[i][at], self.v[i][at], self.pages[i], self.table, self.lens)
            rk.restkv_attend_beams(self.step_cache, self.beams, self.shared, self.q[i][at], self.pages[i], self.table, self.lens,
                                   self.attended[i], None, self.aws)
            logits = logits + self.attended[i].flatten(1).float() @ self.out_w[i].float()
        self.logits = logits
        rk.restkv_beam_select(self.desc, logits, self.scores, self.scores, self.parents, self.tokens, self.ws, finished=self.ended,
                              new_finished=self.ended)
        rk.restkv_beam_reorder(self.step_cache, self.beams, self.parents, self.table, self.lens, self.both)


@pytest.mark.parametrize("fmt", [None, "q4"])
def test_a_search_follows_its_histories(fmt, shared_once):
    """Every step's attention is that of the tokens that a beam stands for, whatever pages they lie in; selections follow its logits."""
    m = Search(fmt)
    m.start()
    hist = [[m.prompts[g, :-1].tolist() for _ in range(m.beams)] for g in range(m.groups)]
    for step in range(22):                                 # over two ends of pages
        scores, ended, tokens = m.scores.cpu(), m.ended.cpu(), m.tokens.cpu()
        hist = [[hist[g][b] + [max(int(tokens[g, b]), 0)] for b in range(m.beams)] for g in range(m.groups)]
        m.step()
        for i in range(m.layers):
            for g in range(m.groups):
                for b in range(m.beams):
                    rows = torch.tensor(hist[g][b], device="cuda")
                    assert len(rows) == int(m.lens[g * m.beams + b])
                    k, v, q = m.k[i][rows].cpu(), m.v[i][rows].cpu(), m.q[i][rows[-1]].cpu().double()
                    if fmt:
                        k, v = (pages_ref.from_q4(*pages_ref.to_q4(x.float())) for x in (k, v))
                    for h in range(4):
                        w = torch.softmax(k[:, h // 2].double() @ q[h] / 8, 0)
                        want = w @ v[:, h // 2].double()
                        got = m.attended[i, g * m.beams + b, h].cpu().double()
                        # rounding of the output; logits below 40 to 100 half steps of float32; weights to 2^-17 and their bits in 4-bit rows
                        tol = 2.0 ** -8 * want.abs() + (2.0 ** -14 if not fmt else 2.0 ** -12) * (w @ v[:, h // 2].double().abs()) + 2.0 ** -16
                        assert ((got - want).abs() <= tol).all(), (step, i, g, b, h)
        got = (m.scores.cpu(), m.parents.cpu(), m.tokens.cpu(), m.ended.cpu())
        ref.assert_select(got, ref.select(m.logits.cpu(), scores, ended, m.beams, 0), m.vocab)
        hist = [[hist[g][p if p >= 0 else b] for b, p in enumerate(got[1][g].tolist())] for g in range(m.groups)]


@pytest.mark.parametrize("fmt", [None, "q4"])
def test_a_search_replayed_from_a_hip_graph(fmt, shared_once):
    """A step captured once, in two graphs that share the workspaces, against eager steps: the same tokens, scores, tables and pages."""
    a, b = Search(fmt, seed=3), Search(fmt, seed=3)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        a.start()
        a.step()
    torch.cuda.current_stream().wait_stream(s)
    graphs = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()]
    for gr in graphs:
        with torch.cuda.graph(gr):
            a.step()
    c = Search(fmt, seed=3)                                # the tables as they were
    a.table.copy_(c.table)
    for x in a.pages:
        for t in (x.k, x.v, x.k_scale, x.v_scale):
            if t is not None:
                t.zero_()
    a.start()
    b.start()
    for i in range(8):
        graphs[i & 1].replay()
        torch.cuda.synchronize()
        b.step()
        torch.cuda.synchronize()
        for x, y in ((a.scores, b.scores), (a.tokens, b.tokens), (a.parents, b.parents), (a.table, b.table), (a.ended, b.ended), (a.lens, b.lens),
                     (a.attended, b.attended)):
            assert torch.equal(x, y), i
        for x, y in zip(a.pages, b.pages):
            assert torch.equal(x.k.view(torch.uint8), y.k.view(torch.uint8)) and torch.equal(x.v.view(torch.uint8), y.v.view(torch.uint8))
