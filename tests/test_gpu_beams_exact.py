"""Selection of beams on the GPU held to what the header says of its arithmetic: places, pairs and flags one by one, sums and scores in 64 bits, and the
join of long lists (more continuations at the bound than it holds) for each number of its wavefronts."""
import math

import pytest
import torch

import paper_2605_08840_amd as rk
from test_gpu_beams import SELECTS, run_select

pytestmark = pytest.mark.gpu

U = 2.0 ** -24            # half a step of float32, relative
TYPES = [torch.float32, torch.bfloat16]


def tiles(rows, vocab, dtype):
    """Tiles of 1024 blocks of 16 bytes that a workgroup takes of a row, at most."""
    vec = 16 // dtype.itemsize
    blocks = -(-vocab // vec) + 1
    pieces = min(-(-blocks // 1024), max(1, 4 * torch.cuda.get_device_properties(0).multi_processor_count // rows))
    return -(-blocks // pieces // 1024) + 1


def bound(rows, vocab, dtype):
    """How far a score is off before its one rounding.  Relative errors of what is summed are errors of the logarithm.  Of an exponential e^-d: u of d
    for the difference to the maximum, u of its exponent (d in the same way), a step (2 u) of the exponential itself; d is ln(vocab) at most in the mean under the
    softmax.  31 u for the 32 terms that are summed in float32 (all positive).  2 u for each time that a sum is scaled to a
    larger maximum: a tile each, then wavefront, workgroup and row; the d of these add up to no more than the term's own, which is counted again."""
    return (4 * math.log(vocab) + 2 + 31 + 2 * (tiles(rows, vocab, dtype) + 3)) * U


def check(logits, scores, finished, n_out, end=2, tie_exact=False, **more):
    """Against 64 bits, place by place; logits on the GPU."""
    groups, beams = scores.shape
    vocab = logits.shape[1]
    got = run_select(logits, scores, finished, n_out, end, **more)
    tol = bound(groups * beams, vocab, logits.dtype)
    x = logits.double()
    top = x.max(1, keepdim=True)[0]
    s = scores.double().cuda().view(-1, 1) + ((x - top) - torch.log(torch.exp(x - top).sum(1, keepdim=True)))
    s[~torch.isfinite(s.float())] = -math.inf                      # NaN too
    # of each beam the best n_out + 1, in order: larger score, larger logit, lower token
    keep = min(n_out + 1, vocab)
    order = torch.sort(torch.where(torch.isfinite(s), x, -math.inf), dim=1, descending=True, stable=True)[1][:, :keep]
    best = s.gather(1, order).cpu().view(groups, beams, keep)
    order = order.cpu().view(groups, beams, keep)
    for g in range(groups):
        ended = [finished is not None and bool(finished[g, b]) for b in range(beams)]
        lists = []                                                 # of each beam: (score, token)
        for b in range(beams):
            c = float(scores[g, b])
            if ended[b]:
                lists.append([(c, end)] if math.isfinite(c) else [])
            else:
                lists.append([(v, t) for v, t in zip(best[g, b].tolist(), order[g, b].tolist()) if v > -math.inf])
        n = min(sum(len(x) for x in lists), n_out)
        value, parent, token, flag = (y[g].tolist() for y in got)
        assert value[n:] == [-math.inf] * (n_out - n) and parent[n:] == [-1] * (n_out - n) and token[n:] == [-1] * (n_out - n)
        assert flag[n:] == [1] * (n_out - n)
        taken, last = [0] * beams, None
        for k in range(n):
            b = parent[k]
            assert 0 <= b < beams and taken[b] < len(lists[b]), (g, k, b)
            want, t = lists[b][taken[b]]                           # within a beam the order is exact
            taken[b] += 1
            assert token[k] == t and flag[k] == int(ended[b] or t == end), (g, k, b, token[k], t)
            off = 0.0 if ended[b] else tol + 8 * 2.0 ** -53 * abs(want)
            assert abs(value[k] - want) <= off + U * abs(want), (g, k, value[k], want)
            if last is not None:                                   # between beams it is that of 64 bits, but for the errors of two sums
                assert value[k] <= value[k - 1]
                near = 0.0 if b == last[1] or tie_exact else 2 * tol + 16 * 2.0 ** -53 * abs(want)
                assert want <= last[0] + near, (g, k, want, last)
                assert not (tie_exact and want == last[0] and b < last[1]), (g, k)
            last = (want, b)
        for b in range(beams):                                     # nothing better was left
            if n == n_out and taken[b] < len(lists[b]):
                near = 0.0 if last[1] == b or tie_exact else 2 * tol + 16 * 2.0 ** -53 * abs(last[0])
                assert lists[b][taken[b]][0] <= last[0] + near, (g, b)
    return got


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("groups,beams,vocab,n_out", SELECTS)
def test_every_place(groups, beams, vocab, n_out, dtype):
    g = torch.Generator().manual_seed(groups * beams + vocab)
    logits = (3 * torch.randn((groups * beams, vocab), generator=g)).to(dtype).cuda()
    scores = -10 * torch.rand((groups, beams), generator=g)
    check(logits, scores, None, n_out)
    check(logits, scores, torch.rand((groups, beams), generator=g) < 0.4, n_out, end=vocab - 1)
    logits[torch.rand(logits.shape, generator=torch.Generator("cuda").manual_seed(1), device="cuda") < 0.9] = -math.inf
    check(logits, scores, torch.rand((groups, beams), generator=g) < 0.2, n_out, end=0)


@pytest.mark.parametrize("dtype", TYPES)
def test_every_place_of_few_values(dtype):
    """Hundreds of equal logits at the edge of every list."""
    g = torch.Generator().manual_seed(8)
    for beams, vocab, n_out in ((4, 9000, 64), (16, 20000, 33), (7, 40000, 12)):
        x = torch.randint(-3, 4, (2 * beams, vocab), generator=g).to(dtype).cuda()
        check(x, -torch.rand((2, beams), generator=g), None, n_out)


# beams, vocabulary in float32 and bfloat16, n_out, wavefronts of the join
JOINS = [(2, 9000, 17000, 64, 4), (8, 5000, 9000, 64, 8), (16, 30000, 30000, 64, 16), (64, 700, 700, 64, 16)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("beams,vocab32,vocab16,n_out,waves", JOINS)
def test_more_continuations_at_the_bound_than_the_join_lists(beams, vocab32, vocab16, n_out, waves, dtype):
    vocab = vocab32 if dtype is torch.float32 else vocab16
    pieces = -(-(vocab * dtype.itemsize // 16 + 1) // 1024)
    left = beams * pieces * n_out
    assert left > 64 * waves and waves == (16 if left > 1024 else 8 if left > 512 or beams >= 8 else 4)
    same, equal = torch.zeros((2 * beams, vocab), dtype=dtype, device="cuda"), torch.zeros((2, beams))
    want = list(range(n_out))
    for x in (same, same - 5.5):                                   # sums that are exact: the lowest beam's lowest tokens
        got = check(x, equal, None, n_out, end=vocab - 1, tie_exact=True)
        assert got[1].tolist() == [[0] * n_out] * 2 and got[2].tolist() == [want] * 2
    # half of the beams have ended: their continuations come first, in order, then the lowest of the others
    ended = torch.arange(beams).expand(2, -1) % 2 == 0
    got = check(same, equal, ended, n_out, end=3, tie_exact=True)
    first = list(range(0, beams, 2))
    assert got[1].tolist() == [(first + [1] * n_out)[:n_out]] * 2
    # ended ones far behind: none of them, but the lowest of the others; and those all ended
    low = torch.where(ended, torch.tensor(-100.0), torch.tensor(0.0))
    got = check(same, low, ended, n_out, tie_exact=True)
    assert got[1].tolist() == [[1] * n_out] * 2 and got[2].tolist() == [want] * 2
    check(same, equal, torch.ones((2, beams)), n_out, tie_exact=True)
    # one beam ahead of equal ones, which fill the list first or not: bounds are taken again
    scores = equal - 50
    scores[0, beams - 1], scores[1, beams // 2] = 0, 0
    x = same.clone()
    x[beams - 1].normal_(generator=torch.Generator("cuda").manual_seed(1))
    runs = [check(x, scores, None, n_out) for _ in range(5)]
    assert runs[0][1].tolist() == [[beams - 1] * n_out, [beams // 2] * n_out]
    assert all(torch.equal(a, b) for r in runs[1:] for a, b in zip(r, runs[0]))       # whatever arrives first


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab", [3, 1000, 12345, 300007])
def test_scores_are_64_bits_until_they_are_rounded(vocab, dtype):
    """Equal logits: exponentials and sums are exact, so a score is c - ln(vocab).  With c next to that logarithm the difference shows what float32 cannot hold."""
    c = torch.tensor([[math.log(vocab)]]).float()
    want = float(c.double()) - math.log(vocab)
    assert 0 < abs(want) < 2.0 ** -20
    got = run_select(torch.full((1, vocab), 0.75, dtype=dtype, device="cuda"), c, None, 2)
    # logarithm and difference in 64 bits to a few of their steps, one rounding
    assert abs(float(got[0][0, 0]) - want) <= 8 * 2.0 ** -53 * math.log(vocab) + U * abs(want), (got[0], want)


@pytest.mark.parametrize("dtype", TYPES)
def test_sums_of_tiles_are_64_bits(dtype):
    """A tile of ones, then four of 2.5e-8: float32 would lose the latter behind the former, in a thread, a wavefront or a workgroup."""
    rows, tile = 4 * torch.cuda.get_device_properties(0).multi_processor_count, 16384 // dtype.itemsize
    vocab = 5 * tile
    assert tiles(rows, vocab, dtype) > 5
    x = torch.full((rows, vocab), -17.5, dtype=dtype, device="cuda")
    x[:, :tile] = 0
    small = 4 * tile * math.exp(-17.5)
    c = torch.tensor(math.log(tile)).float()
    want = float(c.double()) - math.log(tile) - math.log1p(small / tile)
    got = run_select(x, c.expand(rows // 32, 32).contiguous(), None, 3)
    # small terms to 2 x 17.5 u for their exponents, 2 u, and 31 u for their sum; the ones are exact
    tol = (2 * 17.5 + 2 + 31) * U * small / tile + 8 * 2.0 ** -53 * math.log(tile) + U * abs(want)
    assert small / tile > 1000 * tol and ((got[0].double() - want).abs() <= tol).all(), (got[0][0], want, tol)
    assert (got[1] == 0).all() and (got[2] == torch.arange(3)).all()


@pytest.mark.parametrize("dtype", TYPES)
def test_the_order_is_that_of_64_bits(dtype):
    """Two scores that are one in float32: the larger one first, though it is the higher beam's."""
    x = torch.zeros((2, 1000), dtype=dtype, device="cuda")
    x[1, 7] = 2.0 ** -18                                           # 3.8e-6 ahead; a sum is off by 4 u at the most (1000 terms near one, 32 at a time: 35 u = 2e-6)
    got = run_select(x, torch.full((1, 2), -1000.0), None, 2)      # steps of 6e-5
    assert got[1][0, 0] == 1 and got[2][0, 0] == 7 and got[0][0, 0] == got[0][0, 1]


@pytest.mark.parametrize("dtype", TYPES)
def test_ended_beams_keep_their_scores(dtype):
    """To the bit, also where they are not among the rounded ones; flags of every place."""
    g = torch.Generator().manual_seed(4)
    x = torch.randn((12, 500), generator=g).to(dtype).cuda()
    scores = -3 * torch.rand((2, 6), generator=g)
    ended = torch.tensor([[1, 0, 1, 0, 0, 1], [0, 0, 0, 1, 0, 0]])
    got = check(x, scores, ended, 30, end=77)
    for g_ in range(2):
        for b in range(6):
            if ended[g_, b]:
                at = [k for k in range(30) if got[1][g_, k] == b]
                assert len(at) == 1 and got[0][g_, at[0]] == scores[g_, b] and got[2][g_, at[0]] == 77 and got[3][g_, at[0]] == 1
