"""Performance cases of the paged cache: what is timed, on which inputs, and the operators in plain form.

After a layer's cache has been evicted the kept rows move into pages, decoding appends to them and attends to them, and
the rows come back as dense tensors when the cache is evicted again:

  append        restkv_append: new keys (rotated on the way) and values into the pages, new queries rotated beside them
  append_fetch  restkv_append into pages of 4 bits, then restkv_fetch of the cache: what the codes stand for
  attend        restkv_attend: attention of a sequence's newest tokens over its pages, with the log-sum-exp
  fetch         restkv_fetch: rows of the pages as the dense keys and values that an eviction takes

The plain forms are elementary torch operations in 32 bits, rounded once at the end.  Rotation and 4-bit codes are defined
with each product and each sum rounded to 32 bits, so that codes agree exactly; cosines and sines come from 64 bits.
"""
from __future__ import annotations

import math
import random

import torch

own = False
DEV = "cuda"

# (query heads, KV heads)
HEADS = [(4, 2), (8, 8), (16, 4), (28, 4), (32, 8), (64, 8)]


def _case(name, op, hq, hkv, d, n_seqs, shortest, longest, *, new=(1, 1), dtype="bf16", bits=16, page=64, rotary=0,
          interleaved=False, head_lens=False, token_major=False, wide_out=False):
    c = dict(op=op, n_q_heads=hq, n_kv_heads=hkv, head_dim=d, n_seqs=n_seqs, shortest=shortest, longest=longest,
             new_fewest=new[0], new_most=new[1], dtype=dtype, bits=bits, page_size=page, rotary=rotary,
             interleaved=interleaved, head_lens=head_lens, token_major=token_major, wide_out=wide_out)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # one decode step of 32 requests whose caches were evicted to 2048: latency
        _case("append_decode", "append", 32, 8, 128, 32, 2049, 2112, rotary=128),
        # a prompt of 32k tokens goes into the pages
        _case("append_prompt", "append", 32, 8, 128, 1, 32768, 32768, new=(32768, 32768), rotary=128),
        # a toy model in float32: ragged prompts, a quarter of the channels rotated in neighbouring pairs, small pages
        _case("append_f32_ragged", "append", 4, 2, 64, 5, 90, 1024, new=(33, 1001), dtype="f32", bits=32, page=16,
              rotary=16, interleaved=True, token_major=True),
        # a prompt of 8k tokens into 4 bits, and the values that the codes stand for
        _case("q4_prompt", "append_fetch", 32, 8, 128, 1, 8192, 8192, new=(8192, 8192), bits=4, rotary=128),
        # speculative steps of 1 to 4 tokens on caches of 4 bits, heads of 64, and the rows back for the next eviction
        _case("q4_speculative", "append_fetch", 28, 4, 64, 24, 1537, 2112, new=(1, 4), bits=4, rotary=64, page=32),
        # smallest: one token of a toy model in float32 over 1k tokens
        _case("attend_tiny_f32", "attend", 4, 2, 64, 1, 1024, 1024, dtype="f32", bits=32, page=16),
        # decode over evicted caches, a kept length for each head
        _case("attend_evicted", "attend", 32, 8, 128, 32, 1024, 2112, head_lens=True),
        # one request with its whole prompt of 128k tokens kept
        _case("attend_128k", "attend", 32, 8, 128, 1, 131072, 131072),
        # the same in 4 bits
        _case("attend_q4_128k", "attend", 32, 8, 128, 1, 131072, 131072, bits=4),
        # a batch of unequal lengths in 4 bits, groups of 8 query heads
        _case("attend_q4_batch", "attend", 64, 8, 128, 24, 65, 16000, bits=4, page=32),
        # the 64 queries of an observation window over 32k tokens, as restkv_score_from_attention takes them
        _case("attend_window_32k", "attend", 32, 8, 128, 1, 32768, 32768, new=(64, 64), wide_out=True),
        # decode-time re-eviction: the rows of 32 grown caches as dense tensors
        _case("fetch_reevict", "fetch", 32, 8, 128, 32, 2112, 2112),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["append", "append_fetch", "attend", "attend", "attend", "attend", "fetch"])
    hq, hkv = rng.choice(HEADS)
    d = rng.choice([64, 128, 128])
    bits = 4 if op == "append_fetch" else rng.choice([16, 16, 32] if op == "append" else [4, 16, 16, 32])
    dtype = "f32" if bits == 32 or (bits == 4 and rng.random() < 0.2) else "bf16"
    n_seqs = _log_int(rng, 1, 48)
    total = (32768 if dtype == "f32" or op != "attend" else 131072) * 8 // max(hkv, 4)
    longest = _log_int(rng, 16, max(16, total // n_seqs))
    shortest = max(1, int(longest * rng.uniform(0.05, 1.0)))
    kind = rng.random()
    if op in ("append", "append_fetch") and kind < 0.5:
        most = max(1, _log_int(rng, 1, longest))
    elif op == "attend" and kind < 0.35:
        most = min(longest, _log_int(rng, 2, 64))
        longest = min(longest, max(most, 2 ** 20 // (n_seqs * most)))
        shortest = min(shortest, longest)
    else:
        most = 1
    return _case(None, op, hq, hkv, d, n_seqs, shortest, longest, new=(max(1, most // 2), most), dtype=dtype, bits=bits,
                 page=rng.choice([16, 32, 64, 64, 128, 256]),
                 rotary=rng.choice([0, 16, d // 2, d, d]) if op.startswith("append") else 0, interleaved=rng.random() < 0.3,
                 head_lens=rng.random() < 0.3, token_major=rng.random() < 0.3,
                 wide_out=op == "attend" and dtype == "bf16" and n_seqs == 1)


# ---- inputs -------------------------------------------------------------------------------------


def _lengths(c):
    """Per sequence the cached tokens (new ones included) of each KV head, and the new tokens: by the case alone."""
    rng = random.Random(c["n_seqs"] * 1000003 + c["longest"] * 101 + c["shortest"] * 7 + c["new_most"])
    lens, new = [], []
    for s in range(c["n_seqs"]):
        n = c["new_most"] if s == 0 else rng.randint(c["new_fewest"], c["new_most"])
        length = c["longest"] if s == 0 else _log_int(rng, c["shortest"], c["longest"])
        kept = [max(n, length - (rng.randint(0, length // 2) if c["head_lens"] and h else 0)) for h in range(c["n_kv_heads"])]
        lens.append(kept)
        new.append(n)
    return lens, new


def _value_type(c):
    return torch.float32 if c["dtype"] == "f32" else torch.bfloat16


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    vt, ps, hq, hkv, d = _value_type(case), case["page_size"], case["n_q_heads"], case["n_kv_heads"], case["head_dim"]
    lens, new = _lengths(case)
    n_seqs, tokens = case["n_seqs"], sum(new)
    per_seq = [(max(x) + ps - 1) // ps for x in lens]
    width, n_pages = max(per_seq), sum(per_seq) + 3
    order = torch.randperm(n_pages, generator=torch.Generator().manual_seed(seed)).tolist()
    rows, at = [], 0
    for n in per_seq:
        rows.append(order[at:at + n] + [-1] * (width - n))
        at += n
    starts = [0]
    for n in new:
        starts.append(starts[-1] + n)
    st = dict(case=case, table=torch.tensor(rows, dtype=torch.int32, device=DEV),
              lens=torch.tensor(lens if case["head_lens"] else [x[0] for x in lens], dtype=torch.int32, device=DEV),
              new_start=torch.tensor(starts, dtype=torch.int32, device=DEV), tokens=tokens, width=width, n_pages=n_pages,
              longest=max(max(x) for x in lens))

    def normal(*shape, dtype=vt):
        return torch.randn(shape, generator=g, device=DEV, dtype=dtype)

    shape = (n_pages, ps, hkv) if case["token_major"] else (n_pages, hkv, ps)
    if case["bits"] == 4:
        st["k_codes"] = torch.empty(shape + (d // 2,), dtype=torch.uint8, device=DEV)
        st["k_scale"] = torch.empty(shape + (d // 32, 2), dtype=torch.bfloat16, device=DEV)
        st["v_codes"], st["v_scale"] = torch.empty_like(st["k_codes"]), torch.empty_like(st["k_scale"])
        for name in ("k", "v"):
            for lo in range(0, n_pages, max(1, 2 ** 16 // ps)):        # (in parts, to bound the temporaries)
                part = slice(lo, lo + max(1, 2 ** 16 // ps))
                codes, scale = _to_four_bits(normal(*st[name + "_codes"][part].shape[:-1], d, dtype=torch.float32))
                st[name + "_codes"][part], st[name + "_scale"][part] = codes, scale
    else:
        st["k_pages"], st["v_pages"] = normal(*shape, d), normal(*shape, d)
        st["k_pages"][st["table"][:, 0].long(), 0] *= 4                # heavy keys at a sequence's first tokens
    if case["op"].startswith("append"):
        st["k"], st["v"] = normal(tokens, hkv, d), normal(tokens, hkv, d)
        st["q"] = normal(tokens, hq, d)
        st["q_out"] = torch.empty_like(st["q"])
        # true positions: the evicted tokens in front still count
        gone = torch.arange(n_seqs, device=DEV) * 17
        seq = torch.bucketize(torch.arange(tokens, device=DEV), st["new_start"][1:].long(), right=True)
        first = torch.tensor([max(x) - n for x, n in zip(lens, new)], device=DEV)
        st["positions"] = (gone + first - st["new_start"][:-1]).index_select(0, seq).add_(torch.arange(tokens, device=DEV)).int()
        n_positions = st["longest"] + 17 * n_seqs
        half = max(case["rotary"] // 2, 1)
        angle = torch.arange(n_positions, device=DEV, dtype=torch.float64)[:, None] * \
            (10000.0 ** (-torch.arange(half, device=DEV, dtype=torch.float64) / half))
        st["cos"], st["sin"] = angle.cos().float(), angle.sin().float()
        if not case["rotary"]:
            st["cos"] = st["sin"] = None
    if case["op"] == "attend":
        st["q"] = normal(tokens, hq, d)
        if case["wide_out"]:       # [Hq, T, d] and [Hq, T] in float32
            st["out"] = torch.empty((hq, tokens, d), dtype=torch.float32, device=DEV).transpose(0, 1)
            st["lse"] = torch.empty((hq, tokens), dtype=torch.float32, device=DEV).transpose(0, 1)
        else:
            st["out"] = torch.empty((tokens, hq, d), dtype=vt, device=DEV)
            st["lse"] = torch.empty((tokens, hq), dtype=torch.float32, device=DEV)
    if case["op"] in ("fetch", "append_fetch"):
        st["k_out"] = torch.empty((n_seqs, hkv, st["longest"], d), dtype=vt, device=DEV)
        st["v_out"] = torch.empty_like(st["k_out"])
    if own:        # what a program keeps beside its pages
        _handle(st)
    return st


def _handle(st):
    import paper_2605_08840_amd as rk
    c = st["case"]
    st["rk"] = rk
    st["cache"] = rk.make_cache(
        n_seqs=c["n_seqs"], n_q_heads=c["n_q_heads"], n_kv_heads=c["n_kv_heads"], head_dim=c["head_dim"], dtype=_value_type(c),
        format="q4" if c["bits"] == 4 else None, page_size=c["page_size"], n_pages=st["n_pages"], max_pages=st["width"],
        max_new=c["new_most"], n_tokens=st["tokens"], token_major=c["token_major"], head_lens=c["head_lens"],
        rotary_dim=c["rotary"], interleaved=c["interleaved"],
        n_positions=0 if st.get("cos") is None else st["cos"].shape[0], out_head_major=c["wide_out"],
        out_dtype=torch.float32 if c["wide_out"] else None)
    if c["bits"] == 4:
        st["pages"] = rk.CachePages(st["k_codes"], st["v_codes"], st["k_scale"], st["v_scale"])
    else:
        st["pages"] = rk.CachePages(st["k_pages"], st["v_pages"])
    if c["op"] == "attend":
        st["workspace"] = rk.alloc_attend_workspace(st["cache"])


def run(st):
    c = st["case"]
    if own:
        rk = st["rk"]
        if c["op"].startswith("append"):
            rk.restkv_append(st["cache"], st["k"], st["v"], st["pages"], st["table"], st["lens"], new_start=st["new_start"],
                             positions=st["positions"], cos=st["cos"], sin=st["sin"], q=st["q"], q_out=st["q_out"])
        if c["op"] == "append":
            return dict(k=st["k_pages"], v=st["v_pages"], q=st["q_out"])
        if c["op"] == "attend":
            rk.restkv_attend(st["cache"], st["q"], st["pages"], st["table"], st["lens"], st["out"], st["lse"], st["workspace"],
                             new_start=st["new_start"])
            return dict(out=st["out"], lse=st["lse"])
        rk.restkv_fetch(st["cache"], st["pages"], st["table"], st["lens"], st["k_out"], st["v_out"])
        return dict(k=st["k_out"], v=st["v_out"])
    if c["op"] == "append":
        _append(st)
        return dict(k=st["k_pages"], v=st["v_pages"], q=st["q_out"])
    if c["op"] == "append_fetch":
        _append(st)
        return _fetch(st)
    return _attend(st) if c["op"] == "attend" else _fetch(st)


# ---- plain forms --------------------------------------------------------------------------------


def _bf16_below(x):
    """Largest bfloat16 that is not above x (float32)."""
    u = x.contiguous().view(torch.int32)
    cut = u & -65536
    return torch.where((u < 0) & (u != cut), cut + 65536, cut).view(torch.float32)


def _to_four_bits(x):
    """Rows of float32 as codes (two a byte, the lower channel in the low half) and {step, zero} of each group.  A unit is
    d/16 channels; group f holds the channels at places 2f and 2f+1 of every unit."""
    d = x.shape[-1]
    y = x.reshape(x.shape[:-1] + (16, d // 32, 2))
    low, high = y.amin((-3, -1)), y.amax((-3, -1))
    zero = _bf16_below(low)
    spread = high - zero
    step = -_bf16_below(-(spread / torch.full_like(spread, 15)))      # (a true division: by a number it is a product)
    step = torch.where(spread > 0, step.clamp_min(2.0 ** -100), 0.0)
    fine = torch.isfinite(y).all(-1).all(-2) & torch.isfinite(step) & torch.isfinite(zero)
    step, zero = torch.where(fine, step, 0.0), torch.where(fine, zero, math.nan)
    inverse = torch.where(step > 0, torch.ones_like(step) / step, 0.0)
    codes = ((y - zero[..., None, :, None]) * inverse[..., None, :, None]).round().clamp(0, 15)
    codes = torch.where(step[..., None, :, None] > 0, codes, 0.0).to(torch.uint8).reshape(x.shape)
    packed = codes[..., 0::2] | (codes[..., 1::2] << 4)
    return packed, torch.stack((step, zero), -1).to(torch.bfloat16)


def _from_four_bits(codes, scale):
    d = codes.shape[-1] * 2
    c = torch.stack((codes & 15, codes >> 4), -1).reshape(codes.shape[:-1] + (16, d // 32, 2)).float()
    s = scale.float()
    return (s[..., None, :, None, 1] + s[..., None, :, None, 0] * c).reshape(codes.shape[:-1] + (d,))


def _rotate(st, x):
    """Rows [T, H, d] rotated by their positions, in float32."""
    c, x = st["case"], x.float()
    if not c["rotary"]:
        return x
    cos, sin = (st[n].index_select(0, st["positions"].long())[:, None] for n in ("cos", "sin"))
    turned, rest = x[..., :c["rotary"]], x[..., c["rotary"]:]
    if c["interleaved"]:
        a, b = turned[..., 0::2], turned[..., 1::2]
        y = torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2)
    else:
        a, b = turned.chunk(2, -1)
        y = torch.cat((a * cos - b * sin, b * cos + a * sin), -1)
    return torch.cat((y, rest), -1)


def _slots(st):
    """Page and place of every new token, for each KV head: [T, Hkv]."""
    c, starts = st["case"], st["new_start"].long()
    t = torch.arange(st["tokens"], device=DEV)
    seq = torch.bucketize(t, starts[1:], right=True)
    lens = st["lens"].long().reshape(c["n_seqs"], -1).expand(-1, c["n_kv_heads"])
    at = lens[seq] - (starts[1:] - starts[:-1])[seq, None] + (t - starts[seq])[:, None]
    return st["table"].long()[seq[:, None], at // c["page_size"]], at % c["page_size"]


def _append(st):
    c = st["case"]
    page, place = _slots(st)
    head = torch.arange(c["n_kv_heads"], device=DEV)[None].expand_as(page)
    where = (page, place, head) if c["token_major"] else (page, head, place)
    k, v = _rotate(st, st["k"]), st["v"].float()
    if c["bits"] == 4:
        for name, x in (("k", k), ("v", v)):
            st[name + "_codes"][where], st[name + "_scale"][where] = _to_four_bits(x)
    else:
        st["k_pages"][where], st["v_pages"][where] = k.to(st["k_pages"].dtype), v.to(st["v_pages"].dtype)
    st["q_out"].copy_(_rotate(st, st["q"]))


def _dense(st, name, longest):
    """Rows 0 .. longest of every sequence, float32 [S, Hkv, longest, d]; rows of pages that are not there are another page's."""
    c, ps = st["case"], st["case"]["page_size"]
    table = st["table"][:, :(longest + ps - 1) // ps].long().clamp_min(0)
    order = (0, 3, 1, 2, 4) if c["token_major"] else (0, 2, 1, 3, 4)
    if c["bits"] == 4:
        x = _from_four_bits(st[name + "_codes"][table], st[name + "_scale"][table])
    else:
        x = st[name + "_pages"][table].float()
    return x.permute(order).reshape(c["n_seqs"], c["n_kv_heads"], -1, c["head_dim"])[:, :, :longest]


def _visible(st, longest):
    """[S, Hkv, longest]: the rows that are there."""
    c = st["case"]
    lens = st["lens"].reshape(c["n_seqs"], -1, 1).expand(-1, c["n_kv_heads"], 1)
    return torch.arange(longest, device=DEV) < lens


def _fetch(st):
    there = _visible(st, st["longest"])[..., None]
    for n in ("k", "v"):
        st[n + "_out"].copy_(torch.where(there, _dense(st, n, st["longest"]), 0.0))
    return dict(k=st["k_out"], v=st["v_out"])


def _attend(st):
    c, starts, most, longest = st["case"], st["new_start"].long(), st["case"]["new_most"], st["longest"]
    n_seqs, hq, hkv, d = c["n_seqs"], c["n_q_heads"], c["n_kv_heads"], c["head_dim"]
    new = starts[1:] - starts[:-1]
    i = torch.arange(most, device=DEV)
    row = (starts[:-1, None] + i).clamp_max(st["tokens"] - 1)                    # [S, N]
    q = st["q"].float()[row].reshape(n_seqs, most, hkv, hq // hkv, d).permute(0, 2, 3, 1, 4).reshape(n_seqs, hkv, -1, d)
    k, v = _dense(st, "k", longest), _dense(st, "v", longest)
    s = torch.matmul(q, k.transpose(-1, -2)).reshape(n_seqs, hkv, hq // hkv, most, longest) / math.sqrt(d)
    lens = st["lens"].long().reshape(n_seqs, -1).expand(-1, hkv)
    last = lens[:, :, None] - new[:, None, None] + i                             # [S, Hkv, N]: the last visible key
    s.masked_fill_(torch.arange(longest, device=DEV) > last[:, :, None, :, None], -math.inf)
    m = s.amax(-1, keepdim=True)
    p = s.sub_(m).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.reshape(n_seqs, hkv, -1, longest), v).reshape(total.shape[:-1] + (d,)) / total
    lse = (m + total.log())[..., 0]
    o = o.permute(0, 3, 1, 2, 4).reshape(n_seqs, most, hq, d)
    lse = lse.permute(0, 3, 1, 2).reshape(n_seqs, most, hq)
    used = i < new[:, None]
    st["out"].copy_(o[used])
    st["lse"].copy_(lse[used])
    return dict(out=st["out"], lse=st["lse"])


# ---- work and 64 bits ---------------------------------------------------------------------------


def work(case):
    lens, new = _lengths(case)
    d, hq, hkv, size = case["head_dim"], case["n_q_heads"], case["n_kv_heads"], 4 if case["dtype"] == "f32" else 2
    stored = d // 2 + d // 8 if case["bits"] == 4 else d * size
    tokens, rows = sum(new), sum(sum(x) for x in lens)
    if case["op"] == "attend":
        seen = sum(n * h - n * (n - 1) // 2 for x, n in zip(lens, new) for h in x)
        out = 4 if case["wide_out"] else size
        return dict(bytes=2 * rows * stored + tokens * hq * (d * (size + out) + 4), flops=4 * d * (hq // hkv) * seen)
    moved, turned = 0, 0
    if case["op"].startswith("append"):
        moved += tokens * (2 * hkv * (d * size + stored) + 2 * hq * d * size + 4 * case["rotary"] + 4)
        turned += 3 * tokens * (hq + hkv) * case["rotary"]
    if case["op"] in ("fetch", "append_fetch"):
        moved += 2 * rows * stored + 2 * case["n_seqs"] * hkv * max(max(x) for x in lens) * d * size
        turned += 4 * rows * d if case["bits"] == 4 else 0
    return dict(bytes=moved, flops=turned)


def _f32(x):
    return x.float().double()


def _turn64(st, x, rounded):
    """Definition of the rotation, channel by channel; `rounded`: products and sums rounded to 32 bits."""
    c, y, fl = st["case"], x.double().clone(), _f32 if rounded else lambda z: z
    half = c["rotary"] // 2
    pos = st["positions"].long()
    for j in range(half):
        a, b = (2 * j, 2 * j + 1) if c["interleaved"] else (j, j + half)
        cos, sin = st["cos"][pos, j].double()[:, None], st["sin"][pos, j].double()[:, None]
        xa, xb = x[..., a].double(), x[..., b].double()
        y[..., a] = fl(fl(xa * cos) - fl(xb * sin))
        y[..., b] = fl(fl(xb * cos) + fl(xa * sin))
    return y


def _bf16_toward(x, up):
    """Nearest bfloat16 of x (64 bits) on the given side, by its exponent."""
    e = torch.clamp_min(torch.frexp(x)[1].long() - 8, -133)
    unit = torch.tensor([2.0 ** i for i in range(-133, 130)], dtype=torch.float64, device=x.device)[e + 133]
    n = x / unit
    return (torch.ceil(n) if up else torch.floor(n)) * unit


def _four64(x):
    """What the 4-bit codes of rows x (64 bits, exact in 32) stand for, group by group."""
    d, y = x.shape[-1], x.clone()
    place = torch.arange(d, device=x.device) % (d // 16) // 2
    for f in range(d // 32):
        part = x[..., place == f]
        zero = _bf16_toward(part.min(-1, keepdim=True)[0], False)
        spread = _f32(part.max(-1, keepdim=True)[0] - zero)
        step = _bf16_toward(_f32(spread / 15), True)
        code = torch.round(_f32(_f32(part - zero) * _f32(1 / step))).clamp(0, 15)
        y[..., place == f] = torch.where(step > 0, zero + step * torch.nan_to_num(code), zero)
    return y


def _rows64(st, s, h, name):
    """Rows of one head of one sequence, 64 bits."""
    c, ps = st["case"], st["case"]["page_size"]
    n = int(st["lens"][s, h] if c["head_lens"] else st["lens"][s])
    at = torch.arange(n, device=DEV)
    page, place = st["table"][s].long()[at // ps], at % ps
    where = (page, place, h) if c["token_major"] else (page, h, place)
    if c["bits"] != 4:
        return st[name + "_pages"][where].double()
    d = c["head_dim"]
    codes, scale = st[name + "_codes"][where].long(), st[name + "_scale"][where].double()
    ch = torch.arange(d, device=DEV)
    code = (codes[:, ch // 2] >> (4 * (ch % 2))) & 15
    f = ch % (d // 16) // 2
    return scale[:, f, 1] + scale[:, f, 0] * code


def exact(case, seed):
    st = prepare(case, seed)
    c, lens, starts = case, st["lens"], st["new_start"].tolist()
    hq, hkv, d, ps = c["n_q_heads"], c["n_kv_heads"], c["head_dim"], c["page_size"]
    if c["op"] == "attend":
        out = torch.zeros((st["tokens"], hq, d), dtype=torch.float64, device=DEV)
        lse = torch.zeros((st["tokens"], hq), dtype=torch.float64, device=DEV)
        for s in range(c["n_seqs"]):
            a, b = starts[s], starts[s + 1]
            for h in range(hkv):
                k, v, g = _rows64(st, s, h, "k"), _rows64(st, s, h, "v"), slice(h * (hq // hkv), (h + 1) * (hq // hkv))
                logits = torch.matmul(st["q"][a:b, g].double().reshape(-1, d), k.t().contiguous()) * d ** -0.5
                last = k.shape[0] - (b - a) + torch.arange(b - a, device=DEV).repeat_interleave(hq // hkv)
                logits[torch.arange(k.shape[0], device=DEV)[None] > last[:, None]] = -math.inf
                out[a:b, g] = torch.matmul(torch.softmax(logits, -1), v).reshape(b - a, -1, d)
                lse[a:b, g] = torch.logsumexp(logits, -1).reshape(b - a, -1)
        return dict(out=out, lse=lse)
    if c["op"].startswith("append"):
        q, k, v = _turn64(st, st["q"], False), _turn64(st, st["k"], c["bits"] == 4), st["v"].double()
        if c["bits"] == 4:
            k, v = _four64(k), _four64(v)
    if c["op"] == "append":
        pools = {n: st[n + "_pages"].double() for n in ("k", "v")}
    else:
        pools = {n: torch.zeros(st["k_out"].shape, dtype=torch.float64, device=DEV) for n in ("k", "v")}
    for s in range(c["n_seqs"]):
        for h in range(hkv):
            n = int(lens[s, h] if c["head_lens"] else lens[s])
            if c["op"] != "append":
                for name in ("k", "v"):
                    pools[name][s, h, :n] = _rows64(st, s, h, name)
            if c["op"].startswith("append"):
                a, b = starts[s], starts[s + 1]
                at = torch.arange(n - (b - a), n, device=DEV)
                page, place = st["table"][s].long()[at // ps], at % ps
                where = (s, h, at) if c["op"] != "append" else (page, place, h) if c["token_major"] else (page, h, place)
                pools["k"][where], pools["v"][where] = k[a:b, h], v[a:b, h]
    return dict(pools, q=q) if c["op"] == "append" else pools
