"""Performance cases of a beam search over the paged cache: what is timed, on which inputs, and the operators in plain form.

Decoding with several beams a request, or with several requests behind one prompt, on the pages of an evicted cache:

  select   restkv_beam_select: the best continuations of a request's beams from a step's logits
  reorder  restkv_beam_reorder: beams continue others: page tables dealt anew, rows of the last pages copied, in all layers
  attend   restkv_attend_beams: attention of the newest tokens over the pages, those that the beams share read once for all

The plain forms are elementary torch operations in 32 bits, rounded once at the end.  Log-probabilities are ordered in 64
bits: two candidates of different beams may lie closer than 32 bits tell.
"""
from __future__ import annotations

import math
import random

import torch

own = False
DEV = "cuda"

# (query heads, KV heads)
HEADS = [(4, 2), (8, 8), (16, 4), (28, 4), (32, 8), (64, 8)]


def _select(name, groups, beams, vocab, n_out, dtype, *, pad=0, finished=False, masked=0.0, first=False):
    c = dict(op="select", n_groups=groups, n_beams=beams, n_vocab=vocab, n_out=n_out, dtype=dtype, pad=pad, finished=finished,
             masked=masked, first=first)
    return {**c, "name": name} if name else c


def _cache(name, op, hq, hkv, d, groups, beams, shortest, longest, tail, *, dropped=0, layers=1, new=1, dtype="bf16", bits=16,
           page=64, head_lens=False, token_major=False, ragged=False):
    c = dict(op=op, n_q_heads=hq, n_kv_heads=hkv, head_dim=d, n_groups=groups, n_beams=beams, shortest=shortest, longest=longest,
             tail=tail, dropped=dropped, layers=layers, new_most=new, dtype=dtype, bits=bits, page_size=page,
             head_lens=head_lens, token_major=token_major, ragged=ragged)
    return {**c, "name": name} if name else c


def listed():
    return [
        # smallest: a step of one request with four beams: latency
        _select("select_tiny_f32", 1, 4, 32000, 8, "f32"),
        # a step of 16 requests over a vocabulary of odd size (rows that are not aligned), some beams have ended
        _select("select_step", 16, 4, 50257, 4, "bf16", finished=True),
        # few tokens allowed (a grammar), the rest masked
        _select("select_masked", 24, 6, 100003, 12, "bf16", masked=0.998, pad=5),
        # largest: many requests, a large vocabulary, logits in float32
        _select("select_large_f32", 64, 4, 131072, 8, "f32"),
        # many beams a request
        _select("select_wide", 16, 16, 131072, 32, "bf16"),
        # a step of 8 requests of four beams behind evicted prompts, all layers of a model: one beam of each is dropped
        _cache("reorder_step", "reorder", 32, 8, 128, 8, 4, 512, 512, 37, dropped=1, layers=32),
        # kept lengths that differ between the heads (several pages a beam are still open), float32, half of the beams dropped
        _cache("reorder_head_lens_f32", "reorder", 16, 4, 64, 6, 8, 200, 600, 90, dropped=4, layers=4, dtype="f32", bits=32, page=32,
               head_lens=True),
        # smallest: one request with four beams of a toy model in float32
        _cache("attend_tiny_f32", "attend", 4, 2, 64, 1, 4, 1024, 1024, 20, dtype="f32", bits=32, page=16),
        # a step of 8 requests of four beams behind prompts evicted to 2048
        _cache("attend_step", "attend", 32, 8, 128, 8, 4, 2048, 2048, 150),
        # long prompts kept whole, eight beams each
        _cache("attend_32k", "attend", 32, 8, 128, 2, 8, 32768, 32768, 300),
        # the same kind in 4 bits, prompts of unequal lengths
        _cache("attend_q4", "attend", 32, 8, 128, 4, 4, 8000, 32768, 200, bits=4),
        # 32 requests behind one system prompt, each with a conversation of its own length
        _cache("attend_common_prompt", "attend", 32, 8, 128, 1, 32, 16384, 16384, 1500, ragged=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    c = _drawn(rng)
    while work(c)["bytes"] > 2.8e8 or work(c)["flops"] > 8.5e9:          # no more than the largest listed one
        if c["op"] == "reorder":
            c["layers"] = max(1, c["layers"] // 2)
        else:
            c["longest"], c["shortest"] = c["longest"] // 2 + 1, c["shortest"] // 2 + 1
    return c


def _drawn(rng):
    op = rng.choice(["select", "select", "reorder", "attend", "attend"])
    if op == "select":
        beams = rng.choice([1, 2, 3, 4, 5, 8, 10, 16])
        vocab = _log_int(rng, 500, 200000)
        dtype = rng.choice(["f32", "bf16", "bf16"])
        groups = _log_int(rng, 1, max(1, min(64, 2 ** 25 // (beams * vocab))))
        return _select(None, groups, beams, vocab, min(64, beams * rng.choice([1, 1, 2, 4])), dtype, pad=rng.choice([0, 0, 8, 13]),
                       finished=rng.random() < 0.4, masked=rng.choice([0.0, 0.0, 0.02, 0.99]), first=rng.random() < 0.15)
    hq, hkv = rng.choice(HEADS)
    d = rng.choice([64, 128, 128])
    bits = rng.choice([16, 16, 32] if op == "reorder" else [4, 16, 16, 32])
    dtype = "f32" if bits == 32 or (bits == 4 and rng.random() < 0.2) else "bf16"
    page = rng.choice([16, 32, 64, 64, 128])
    beams = rng.choice([2, 3, 4, 5, 8, 12, 16])
    tail = _log_int(rng, 1, 400)
    head_lens, token_major = rng.random() < 0.25, rng.random() < 0.3
    if op == "reorder":
        layers = rng.choice([1, 4, 16, 32])
        longest = _log_int(rng, 32, 600)
        room = 2 ** 28 // (layers * hkv * d * (4 if bits == 32 else 2))                # positions of all sequences
        groups = _log_int(rng, 1, max(1, min(16, room // (longest + beams * (tail + 2 * page + (longest if head_lens else 0))))))
        return _cache(None, op, hq, hkv, d, groups, beams, max(1, longest // rng.choice([1, 2, 5])), longest, tail,
                      dropped=rng.randint(0, beams - 1), layers=layers, dtype=dtype, bits=bits, page=page, head_lens=head_lens,
                      token_major=token_major)
    groups = _log_int(rng, 1, 8)
    longest = _log_int(rng, 40, max(41, min(32768, 2 ** 19 * 8 // (groups * beams * hkv) - tail)))
    return _cache(None, op, hq, hkv, d, groups, beams, max(1, int(longest * rng.uniform(0.1, 1.0))), longest, tail,
                  new=rng.choice([1, 1, 1, 3]), dtype=dtype, bits=bits, page=page, head_lens=head_lens, token_major=token_major,
                  ragged=rng.random() < 0.3)


# ---- inputs -------------------------------------------------------------------------------------


def _value_type(c):
    return torch.float32 if c["dtype"] == "f32" else torch.bfloat16


def _lengths(c):
    """By the case alone.  Of every sequence the positions (new ones included) of each KV head, and its new tokens; of every
    group the pages in front that its beams share."""
    rng = random.Random(c["n_groups"] * 1000003 + c["n_beams"] * 10007 + c["longest"] * 101 + c["shortest"] * 7 + c["tail"])
    lens, new, shared = [], [], []
    for g in range(c["n_groups"]):
        prompt = c["longest"] if g == 0 else _log_int(rng, c["shortest"], c["longest"])
        kept = [max(1, prompt - (rng.randint(0, prompt // 2) if c["head_lens"] and h else 0)) for h in range(c["n_kv_heads"])]
        shared.append(min(kept) // c["page_size"])
        for b in range(c["n_beams"]):
            n = 0 if c["op"] == "reorder" else c["new_most"] if b == 0 or not c["ragged"] else rng.randint(1, c["new_most"])
            more = c["tail"] if b == 0 or not c["ragged"] else _log_int(rng, 1, c["tail"])
            lens.append([k + max(more, n) for k in kept])
            new.append(n)
    return lens, new, shared


def _select_inputs(c, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    groups, beams, vocab = c["n_groups"], c["n_beams"], c["n_vocab"]
    logits = torch.empty((groups * beams, vocab + c["pad"]), dtype=_value_type(c), device=DEV)
    for r in range(groups):                    # what a request's beams have in common, and each beam's own; a few likely tokens
        x = 2 * torch.randn((1, vocab), generator=g, device=DEV) + torch.randn((beams, vocab), generator=g, device=DEV)
        likely = torch.randint(vocab, (40,), generator=g, device=DEV)
        x[:, likely] += 6 * torch.rand((beams, 40), generator=g, device=DEV) + 2
        if c["masked"]:
            x[torch.rand((1, vocab), generator=g, device=DEV).expand(beams, vocab) < c["masked"]] = -math.inf
        logits[r * beams:(r + 1) * beams, :vocab] = x
    logits[:, vocab:] = 50.0                   # behind the rows: not looked at
    scores = -20 * torch.rand((groups, beams), generator=g, device=DEV) ** 2 - 5 * torch.rand((groups, 1), generator=g, device=DEV)
    finished = None
    if c["finished"]:
        finished = (torch.rand((groups, beams), generator=g, device=DEV) < 0.25).int()
    if c["first"]:                             # only a request's first beam stands for anything yet
        scores[:, 1:] = -math.inf
    return dict(case=c, logits=logits[:, :vocab], scores=scores, finished=finished)


def prepare(case, seed):
    c = case
    if c["op"] == "select":
        st = _select_inputs(c, seed)
        shape = (c["n_groups"], c["n_out"])
        st["new_scores"] = torch.empty(shape, dtype=torch.float32, device=DEV)
        for name in ("parents", "tokens", "new_finished"):
            st[name] = torch.empty(shape, dtype=torch.int32, device=DEV)
        if own:
            import paper_2605_08840_amd as rk
            st["rk"] = rk
            st["beams"] = rk.make_beams(n_groups=c["n_groups"], n_beams=c["n_beams"], n_vocab=c["n_vocab"], n_out=c["n_out"],
                                        dtype=_value_type(c), end_token=2, logit_stride=c["n_vocab"] + c["pad"])
            st["workspace"] = rk.alloc_beam_workspace(st["beams"])
        return st
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    rng = random.Random(seed)
    lens, new, shared = _lengths(c)
    ps, hkv, d, beams, layers = c["page_size"], c["n_kv_heads"], c["head_dim"], c["n_beams"], c["layers"]
    room = ps if c["op"] == "reorder" else 0                             # (pages for what is to come)
    width = max((max(x) + room + ps - 1) // ps for x in lens)
    # pages: a group's shared ones, then its sequences' own
    rows, used = [], 0
    for s, x in enumerate(lens):
        front = shared[s // beams]
        if s % beams == 0:
            common, used = list(range(used, used + front)), used + front
        mine = (max(x) + room + ps - 1) // ps - front
        rows.append(common + list(range(used, used + mine)) + [-1] * (width - front - mine))
        used += mine
    n_pages = used + 3
    order = list(range(n_pages))
    rng.shuffle(order)
    st = dict(case=c, n_pages=n_pages, width=width, longest=max(max(x) for x in lens), tokens=sum(new),
              table=torch.tensor([[order[p] if p >= 0 else -1 for p in r] for r in rows], dtype=torch.int32, device=DEV),
              lens=torch.tensor(lens if c["head_lens"] else [x[0] for x in lens], dtype=torch.int32, device=DEV))
    shape = (layers, n_pages, ps, hkv) if c["token_major"] else (layers, n_pages, hkv, ps)
    for name in ("k", "v"):
        if c["bits"] == 4:
            st[name + "_codes"] = torch.randint(256, shape + (d // 2,), generator=g, device=DEV, dtype=torch.uint8)
            step = 0.15 + 0.2 * torch.rand(shape + (d // 32, 1), generator=g, device=DEV)
            st[name + "_scale"] = torch.cat((step, -7.5 * step + 0.3 * torch.randn(step.shape, generator=g, device=DEV)), -1).bfloat16()
        else:
            st[name + "_pages"] = torch.randn(shape + (d,), generator=g, device=DEV, dtype=_value_type(c))
    if c["op"] == "reorder":
        parents = []
        for _ in range(c["n_groups"]):                                   # so many beams without a child, the others at random
            alive = sorted(rng.sample(range(beams), beams - c["dropped"]))
            p = alive + [rng.choice(alive) for _ in range(c["dropped"])]
            rng.shuffle(p)
            parents.append(p)
        st["parents"] = torch.tensor(parents, dtype=torch.int32, device=DEV)
        st["table_out"] = torch.empty_like(st["table"])
    else:
        if c["bits"] != 4:
            st["k_pages"][0, st["table"][:, 0].long(), 0] *= 3           # heavy keys at a sequence's first tokens
        starts = [0]
        for n in new:
            starts.append(starts[-1] + n)
        st["new_start"] = torch.tensor(starts, dtype=torch.int32, device=DEV)
        st["shared"] = torch.tensor(shared, dtype=torch.int32, device=DEV)
        st["q"] = torch.randn((st["tokens"], c["n_q_heads"], d), generator=g, device=DEV, dtype=_value_type(c))
        st["out"] = torch.empty_like(st["q"])
        st["lse"] = torch.empty((st["tokens"], c["n_q_heads"]), dtype=torch.float32, device=DEV)
    if own:
        import paper_2605_08840_amd as rk
        st["rk"] = rk
        st["cache"] = rk.make_cache(
            n_seqs=len(lens), n_q_heads=c["n_q_heads"], n_kv_heads=hkv, head_dim=d, dtype=_value_type(c),
            format="q4" if c["bits"] == 4 else None, page_size=ps, n_pages=n_pages, max_pages=width, max_new=c["new_most"],
            n_tokens=st["tokens"], token_major=c["token_major"], head_lens=c["head_lens"])
        st["pages"] = [rk.CachePages(*(st[n][i] for n in (("k_codes", "v_codes", "k_scale", "v_scale") if c["bits"] == 4 else
                                                          ("k_pages", "v_pages")))) for i in range(layers)]
        if c["op"] == "attend":
            st["workspace"] = rk.alloc_attend_beams_workspace(st["cache"], beams)
        else:
            st["layers"] = rk.CacheLayers(st["pages"])
    return st


def run(st):
    c = st["case"]
    if own:
        rk = st["rk"]
        if c["op"] == "select":
            rk.restkv_beam_select(st["beams"], st["logits"], st["scores"], st["new_scores"], st["parents"], st["tokens"], st["workspace"],
                                  finished=st["finished"], new_finished=st["new_finished"])
        elif c["op"] == "reorder":
            rk.restkv_beam_reorder(st["cache"], c["n_beams"], st["parents"], st["table"], st["lens"], st["layers"], st["table_out"])
        else:
            rk.restkv_attend_beams(st["cache"], c["n_beams"], st["shared"], st["q"], st["pages"][0], st["table"], st["lens"], st["out"],
                                   st["lse"], st["workspace"], new_start=st["new_start"])
    elif c["op"] == "select":
        _plain_select(st)
    elif c["op"] == "reorder":
        _plain_reorder(st)
    else:
        _plain_attend(st)
    if c["op"] == "select":
        return {n: st[n] for n in ("new_scores", "parents", "tokens", "new_finished")}
    if c["op"] == "reorder":
        return dict(table=st["table_out"], k=st["k_pages"], v=st["v_pages"])
    return dict(out=st["out"], lse=st["lse"])


# ---- plain forms --------------------------------------------------------------------------------


def _plain_select(st):
    c = st["case"]
    groups, beams, vocab, n_out = c["n_groups"], c["n_beams"], c["n_vocab"], c["n_out"]
    x = st["logits"].float() + 0.0                                       # (no -0)
    # a row's largest logits, of equal ones the lower token first: whole numbers of that order
    bits = x.view(torch.int32).long()
    key = (torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits) << 32) + (vocab - 1 - torch.arange(vocab, device=DEV))
    best = key.topk(min(n_out, vocab), -1)[0]
    token = vocab - 1 - (best & 0xFFFFFFFF)
    top = x.amax(-1, keepdim=True).double()
    total = (x.double() - top).exp().sum(-1, keepdim=True)
    score = st["scores"].reshape(-1, 1).double() + ((x.gather(-1, token).double() - top) - total.log())
    if st["finished"] is not None:                                       # one candidate, as it is
        ended = st["finished"].reshape(-1, 1) != 0
        first = torch.arange(token.shape[1], device=DEV) == 0
        score = torch.where(ended, torch.where(first, st["scores"].reshape(-1, 1).double(), -math.inf), score)
        token = torch.where(ended, 2, token)
    score = torch.where(torch.isfinite(score), score, -math.inf).reshape(groups, -1)
    order = score.sort(dim=-1, descending=True, stable=True)
    n = min(n_out, score.shape[1])
    at, value = order.indices[:, :n], order.values[:, :n]
    there = value > -math.inf
    parent = torch.where(there, at // best.shape[1], -1)
    token = torch.where(there, token.reshape(groups, -1).gather(1, at), -1)
    done = token == 2
    if st["finished"] is not None:
        done = done | (st["finished"].gather(1, parent.clamp_min(0)) != 0)
    st["new_scores"].fill_(-math.inf)
    st["parents"].fill_(-1)
    st["tokens"].fill_(-1)
    st["new_finished"].fill_(1)
    st["new_scores"][:, :n] = value.float()
    st["parents"][:, :n] = parent.int()
    st["tokens"][:, :n] = token.int()
    st["new_finished"][:, :n] = (done | ~there).int()


def _plain_reorder(st):
    c = st["case"]
    groups, beams, ps, hkv = c["n_groups"], c["n_beams"], c["page_size"], c["n_kv_heads"]
    old = st["table"].long().reshape(groups, beams, -1)
    mine = torch.arange(beams, device=DEV)
    p = st["parents"].long()
    child = p[:, :, None] == mine                                        # [group, beam, its parent]
    has_child = child.any(1)
    heir = torch.where(child.diagonal(dim1=1, dim2=2), mine, child.int().argmax(1))     # gets its parent's open pages
    takes = heir.gather(1, p) != mine                                    # gets the pages of a beam without a child
    spare = has_child.int().sort(dim=1, stable=True).indices                 # (those first)
    giver = torch.where(takes, spare.gather(1, (takes.cumsum(1) - 1).clamp_min(0)), p)
    of_parent = old.gather(1, p[..., None].expand_as(old))
    of_giver = old.gather(1, giver[..., None].expand_as(old))
    lens = st["lens"].long().reshape(groups, beams, -1)[:, 0].expand(-1, hkv)           # a group's beams are equally long
    col = torch.arange(st["width"], device=DEV)
    closed = col < (lens.amin(1) // ps)[:, None, None]
    open_ = ~closed & (col <= ((lens.amax(1) - 1) // ps)[:, None, None])
    st["table_out"].copy_(torch.where(closed, of_parent, torch.where(open_, of_giver, old)).reshape(groups * beams, -1))
    g, b, w = (open_ & takes[..., None]).nonzero(as_tuple=True)
    src, dst = of_parent[g, b, w], of_giver[g, b, w]
    i, head, at = (w[:, None, None] * ps + torch.arange(ps, device=DEV) < lens[g][:, :, None]).nonzero(as_tuple=True)
    here, there = ((src[i], at, head), (dst[i], at, head)) if c["token_major"] else ((src[i], head, at), (dst[i], head, at))
    st["k_pages"][(slice(None),) + there] = st["k_pages"][(slice(None),) + here]
    st["v_pages"][(slice(None),) + there] = st["v_pages"][(slice(None),) + here]


def _dense(st, name):
    """Rows of every sequence, float32 [S, Hkv, longest, d]; rows of pages that are not there are another page's."""
    c, ps, longest = st["case"], st["case"]["page_size"], st["longest"]
    table = st["table"].long().clamp_min(0)
    order = (0, 3, 1, 2, 4) if c["token_major"] else (0, 2, 1, 3, 4)
    if c["bits"] == 4:
        codes, scale = st[name + "_codes"][0][table], st[name + "_scale"][0][table].float()
        y = torch.stack((codes & 15, codes >> 4), -1).reshape(codes.shape[:-1] + (16, c["head_dim"] // 32, 2)).float()
        x = (scale[..., None, :, None, 1] + scale[..., None, :, None, 0] * y).flatten(-3)
    else:
        x = st[name + "_pages"][0][table].float()
    return x.permute(order).reshape(table.shape[0], c["n_kv_heads"], -1, c["head_dim"])[:, :, :longest]


def _plain_attend(st):
    c, starts, most, longest = st["case"], st["new_start"].long(), st["case"]["new_most"], st["longest"]
    n_seqs, hq, hkv, d = c["n_groups"] * c["n_beams"], c["n_q_heads"], c["n_kv_heads"], c["head_dim"]
    new = starts[1:] - starts[:-1]
    i = torch.arange(most, device=DEV)
    row = (starts[:-1, None] + i).clamp_max(st["tokens"] - 1)                    # [S, N]
    q = st["q"].float()[row].reshape(n_seqs, most, hkv, hq // hkv, d).permute(0, 2, 3, 1, 4).reshape(n_seqs, hkv, -1, d)
    s = torch.matmul(q, _dense(st, "k").transpose(-1, -2)).reshape(n_seqs, hkv, hq // hkv, most, longest) / math.sqrt(d)
    lens = st["lens"].long().reshape(n_seqs, -1).expand(-1, hkv)
    last = lens[:, :, None] - new[:, None, None] + i                             # [S, Hkv, N]: the last visible position
    s.masked_fill_(torch.arange(longest, device=DEV) > last[:, :, None, :, None], -math.inf)
    m = s.amax(-1, keepdim=True)
    p = s.sub_(m).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.reshape(n_seqs, hkv, -1, longest), _dense(st, "v")).reshape(total.shape[:-1] + (d,)) / total
    lse = (m + total.log())[..., 0]
    used = i < new[:, None]
    st["out"].copy_(o.permute(0, 3, 1, 2, 4).reshape(n_seqs, most, hq, d)[used])
    st["lse"].copy_(lse.permute(0, 3, 1, 2).reshape(n_seqs, most, hq)[used])


# ---- work and 64 bits ---------------------------------------------------------------------------


def work(case):
    c = case
    size = 4 if c["dtype"] == "f32" else 2
    if c["op"] == "select":
        rows = c["n_groups"] * c["n_beams"]
        return dict(bytes=rows * (c["n_vocab"] * size + 8) + c["n_groups"] * c["n_out"] * 16, flops=5 * rows * c["n_vocab"])
    lens, new, shared = _lengths(c)
    d, hkv, ps, beams = c["head_dim"], c["n_kv_heads"], c["page_size"], c["n_beams"]
    stored = d // 2 + d // 8 if c["bits"] == 4 else d * size
    if c["op"] == "reorder":
        first = lens[::beams]
        copied = c["dropped"] * sum(sum(max(0, n - min(x) // ps * ps) for n in x) for x in first)
        table = len(lens) * sum(max(x) // ps + 1 for x in first) // len(first)
        return dict(bytes=4 * c["layers"] * copied * stored + 8 * table, flops=0)
    rows = sum(sum(x) for x in lens) - (beams - 1) * sum(shared) * ps * hkv
    seen = sum(n * h - n * (n - 1) // 2 for x, n in zip(lens, new) for h in x)
    return dict(bytes=2 * rows * stored + sum(new) * c["n_q_heads"] * (2 * d * size + 4), flops=4 * d * (c["n_q_heads"] // hkv) * seen)


def _select64(st):
    """Scores in 64 bits, a request at a time, by a full order of its candidates."""
    c, every = st["case"], []
    for g in range(c["n_groups"]):
        score = []
        for b in range(c["n_beams"]):
            r, c0 = g * c["n_beams"] + b, st["scores"][g, b].double()
            if st["finished"] is not None and st["finished"][g, b]:
                score.append(c0.reshape(1))
                continue
            score.append(c0 + torch.log_softmax(st["logits"][r].double(), 0))
        x = torch.cat(score)
        x = x[torch.isfinite(x)].sort(descending=True)[0][:c["n_out"]]
        every.append(torch.cat((x, x.new_full((c["n_out"] - x.numel(),), -math.inf))))
    return dict(new_scores=torch.stack(every), parents=None, tokens=None, new_finished=None)


def _rows64(st, s, h, name, n):
    """The first n rows of one head of one sequence."""
    c, ps = st["case"], st["case"]["page_size"]
    t = torch.arange(n, device=DEV)
    page = st["table"][s, t // ps].long()
    where = (page, t % ps, torch.full_like(t, h)) if c["token_major"] else (page, torch.full_like(t, h), t % ps)
    if c["bits"] != 4:
        return st[name + "_pages"][0][where].double()
    codes, scale = st[name + "_codes"][0][where].long(), st[name + "_scale"][0][where].double()
    ch = torch.arange(c["head_dim"], device=DEV)
    code = (codes[:, ch // 2] >> (4 * (ch % 2))) & 15
    of = ch % (c["head_dim"] // 16) // 2
    return scale[:, of, 1] + scale[:, of, 0] * code


def exact(case, seed):
    c = case
    if c["op"] == "reorder":                         # (rows and page numbers as they are: nothing is computed)
        return None
    if c["op"] == "select":
        return _select64(_select_inputs(c, seed)) if c["n_groups"] * c["n_beams"] * c["n_vocab"] <= 2 ** 26 else None
    st = prepare(c, seed)
    lens, new, _ = _lengths(c)
    if sum(len(x) for x in lens) > 6000:
        return None
    d, per = c["head_dim"], c["n_q_heads"] // c["n_kv_heads"]
    out = torch.empty((st["tokens"], c["n_q_heads"], d), dtype=torch.float64, device=DEV)
    lse = torch.empty((st["tokens"], c["n_q_heads"]), dtype=torch.float64, device=DEV)
    first = 0
    for s, n in enumerate(new):
        for h in range(c["n_kv_heads"]):
            length = lens[s][h]
            k, v = _rows64(st, s, h, "k", length), _rows64(st, s, h, "v", length)
            heads = slice(h * per, (h + 1) * per)
            for i in range(n):
                seen = length - n + i + 1
                z = st["q"][first + i, heads].double() @ k[:seen].t() / math.sqrt(d)
                lse[first + i, heads] = torch.logsumexp(z, -1)
                out[first + i, heads] = torch.softmax(z, -1) @ v[:seen]
        first += n
    return dict(out=out, lse=lse)
