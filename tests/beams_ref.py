"""Plain beams for the tests: 64 bits, loops, CPU."""
from __future__ import annotations

import math

import torch

F32 = 2.0 ** -24          # half a step, relative


def select(logits, scores, finished, n_out, end):
    """(scores, parents, tokens, ended) [G, n_out] by the definition in the header; the scores that come next too, for a look at ties."""
    groups, beams = scores.shape
    vocab = logits.shape[-1]
    logits = logits.reshape(groups, beams, vocab)
    out = (torch.full((groups, n_out), -math.inf, dtype=torch.float64), torch.full((groups, n_out), -1), torch.full((groups, n_out), -1),
           torch.ones((groups, n_out), dtype=torch.long), torch.full((groups,), -math.inf, dtype=torch.float64))
    for g in range(groups):
        every = []                                             # (-score, beam, -logit, token)
        for b in range(beams):
            c = float(scores[g, b])
            if finished is not None and int(finished[g, b]):
                if math.isfinite(c):
                    every.append((-c, b, 0.0, end))
                continue
            x = logits[g, b].double()
            m = x.max()
            s = c + ((x - m) - torch.log(torch.exp(x - m).sum()))
            v = torch.nonzero(torch.isfinite(s.float()))[:, 0]     # (finite as they are given out)
            if len(v) > n_out + 1:                             # (more cannot be taken: ties with the last one kept)
                v = v[s[v] >= s[v].topk(n_out + 1)[0][-1]]
            every += [(-float(s[i]), b, -float(x[i]), int(i)) for i in v]
        every.sort()
        for k, (s, b, _, v) in enumerate(every[:n_out]):
            out[0][g, k], out[1][g, k], out[2][g, k] = -s, b, v
            out[3][g, k] = int(v == end or bool(finished is not None and int(finished[g, b])))
        if len(every) > n_out:
            out[4][g] = -every[n_out][0]
    return out


def bound(vocab, score):
    """How far a score may be off.  With u = 2^-24: a difference to the maximum is off by u of its own size, at most ln(vocab) in the mean
    under the softmax; an exponential by 3 u, the sum of a thread's at most 128 of them by 128 u (all terms are positive); these are the relative error of the
    sum, so the error of its logarithm.  Then one rounding of the score."""
    return (math.log(vocab) + 3 + 128) * F32 + F32 * score.abs()


def assert_select(got, want, vocab):
    """got: (new_scores, parents, tokens, new_finished) of the library, on the CPU."""
    score, parent, token, ended, rest = want
    there = torch.isfinite(score)
    assert torch.equal(torch.isfinite(got[0]), there) and torch.equal(got[0][~there], torch.full_like(got[0][~there], -math.inf))
    tol = bound(vocab, score)
    off = (got[0].double() - score).abs()
    assert (off[there] <= tol[there]).all(), f"scores off by {off[there].max():.3g}"
    # the order is that of 64 bits, wherever scores of different beams lie further apart than the bounds
    for g in range(score.shape[0]):
        n = int(there[g].sum())
        same = torch.equal(got[1][g].long(), parent[g]) and torch.equal(got[2][g].long(), token[g])
        s = torch.cat((score[g, :n], rest[g:g + 1]))
        p = torch.cat((parent[g, :n], torch.tensor([-2])))
        near = ((s[:-1] - s[1:]) <= 2 * bound(vocab, s[:-1])) & (p[:-1] != p[1:]) & (s[:-1] != s[1:])
        assert same or near.any(), f"group {g}: {got[1][g].tolist()} {got[2][g].tolist()} for {parent[g].tolist()} {token[g].tolist()}"
        if same and got[3] is not None:
            assert torch.equal(got[3][g].long(), ended[g])


def deal(parents, n_beams):
    """Per beam of one group: (parent, whose pages of open columns it gets)."""
    p = [x if 0 <= x < n_beams else b for b, x in enumerate(parents)]
    heir = {x: (x if p[x] == x else p.index(x)) for x in p}
    spare = [x for x in range(n_beams) if x not in heir]
    return [(p[b], p[b] if heir[p[b]] == b else spare.pop(0)) for b in range(n_beams)]
