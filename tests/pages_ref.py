"""Plain paged cache for the tests: 64 bits (or 32 where a definition rounds), loops, CPU."""
from __future__ import annotations

import math

import torch

F32 = 2.0 ** -24          # half a step, relative


def bf16_down(x):
    """Largest bfloat16 that is not above x (float32, CPU), by trying the neighbours of the nearest."""
    y = x.to(torch.bfloat16)
    low = torch.nextafter(y, torch.full_like(y, -math.inf))
    return torch.where(y.float() > x, low, y).float()


def to_q4(x):
    """Rows of float32 (CPU) as codes, {step, zero} and values, by the definition in the header."""
    d = x.shape[-1]
    codes, scale = torch.zeros(x.shape, dtype=torch.uint8), torch.zeros(x.shape[:-1] + (d // 32, 2))
    group = torch.arange(d) % (d // 16) // 2
    for f in range(d // 32):
        part = x[..., group == f]
        zero = bf16_down(part.amin(-1))
        spread = part.amax(-1) - zero
        step = -bf16_down(-(spread / torch.tensor(15.0)))
        step = torch.where(spread > 0, step.clamp_min(2.0 ** -100), torch.zeros(()))
        bad = ~torch.isfinite(part).all(-1) | ~torch.isfinite(step) | ~torch.isfinite(zero)
        step, zero = step.masked_fill(bad, 0.0), zero.masked_fill(bad, math.nan)
        code = ((part - zero[..., None]) * (torch.ones(()) / step)[..., None]).round().clamp(0, 15)
        codes[..., group == f] = torch.where(step[..., None] > 0, code, torch.zeros(())).to(torch.uint8)
        scale[..., f, 0], scale[..., f, 1] = step, zero
    return codes, scale.to(torch.bfloat16)


def from_q4(codes, scale):
    """Values of unpacked codes, 64 bits (exact)."""
    d = codes.shape[-1]
    f = torch.arange(d) % (d // 16) // 2
    return scale[..., f, 1].double() + scale[..., f, 0].double() * codes.double()


def pack(codes):
    return codes[..., 0::2] | (codes[..., 1::2] << 4)


def unpack(packed):
    return torch.stack((packed & 15, packed >> 4), -1).flatten(-2)


def rotate(x, cos, sin, rot, pairs):
    """Rows x [..., d] float32 with cos, sin [..., rot/2]: each product and each sum rounded to float32."""
    y = x.clone()
    for j in range(rot // 2):
        a, b = (2 * j, 2 * j + 1) if pairs else (j, j + rot // 2)
        y[..., a] = x[..., a] * cos[..., j] - x[..., b] * sin[..., j]
        y[..., b] = x[..., b] * cos[..., j] + x[..., a] * sin[..., j]
    return y


class Plain:
    """A paged cache on the CPU beside the one on the GPU: pools full of junk, pages in shuffled order."""

    def __init__(self, rk, *, lens, new, seed=0, hq=4, hkv=2, d=64, ps=16, dtype="bf16", fmt=None, token_major=False,
                 head_lens=False, head_tables=False, spare=2, junk=math.nan, room=0, spread=1.0, **more):
        """lens: per sequence, or per sequence a list by KV head; new: new tokens of each sequence."""
        g = torch.Generator().manual_seed(seed)
        self.g, self.rk, self.hq, self.hkv, self.d, self.ps = g, rk, hq, hkv, d, ps
        self.type = torch.float32 if dtype == "f32" else torch.bfloat16
        self.q4 = fmt == "q4"
        self.lens = [[x] * hkv if isinstance(x, int) else list(x) for x in lens]
        self.new, n_seqs = list(new), len(lens)
        need = [[(x + ps - 1) // ps for x in row] for row in self.lens]
        self.width = max([1] + [max(x) for x in need]) + room
        heads = hkv if head_tables else 1
        used = sum(sum(x) if head_tables else max(x) for x in need)
        n_pages = used + spare
        order = torch.randperm(n_pages, generator=g).tolist()
        table = torch.full((n_seqs, heads, self.width), 2 ** 30, dtype=torch.int32)      # entries behind the last: no pages
        for s in range(n_seqs):
            for h in range(heads):
                for i in range(need[s][h] if head_tables else max(need[s])):
                    table[s, h, i] = order.pop()
        self.table, self.head_tables, self.token_major = table, head_tables, token_major
        self.start = [0]
        for n in new:
            self.start.append(self.start[-1] + n)
        self.tokens = self.start[-1] + more.pop("extra_tokens", 0)
        self.c = rk.make_cache(n_seqs=n_seqs, n_q_heads=hq, n_kv_heads=hkv, head_dim=d, page_size=ps, n_pages=n_pages,
                               max_pages=self.width, dtype=self.type, format=fmt, max_new=more.pop("max_new", max(1, max(new))),
                               n_tokens=self.tokens, token_major=token_major, head_lens=head_lens, head_tables=head_tables, **more)
        pool_heads = 1 if head_tables else hkv
        shape = (n_pages, ps, pool_heads) if token_major else (n_pages, pool_heads, ps)
        rnd = lambda *s: torch.randn(s, generator=g) * spread  # noqa: E731
        self.pool = {}
        for name in ("k", "v"):
            if self.q4:
                codes, scale = to_q4(rnd(*shape, d))
                self.pool[name], self.pool[name + "_scale"] = codes, scale
            else:
                self.pool[name] = rnd(*shape, d).to(self.type)
        # what no sequence holds is junk
        held = torch.zeros(shape, dtype=torch.bool)
        for s in range(n_seqs):
            for h in range(hkv):
                for t in range(self.lens[s][h]):
                    held[self.where(s, h, t)] = True
        for name in ("k", "v"):
            x = self.pool[name + "_scale"] if self.q4 else self.pool[name]
            x[~held] = junk
        self.tensors = dict(
            table=(table if head_tables else table[:, 0]).contiguous().cuda(),
            lens=torch.tensor(self.lens if head_lens else [x[0] for x in self.lens], dtype=torch.int32).cuda(),
            new_start=torch.tensor(self.start, dtype=torch.int32).cuda())
        self.up()

    def up(self):
        """The pools on the GPU."""
        p = self.pool
        self.pages = self.rk.CachePages(pack(p["k"]).cuda(), pack(p["v"]).cuda(), p["k_scale"].cuda(), p["v_scale"].cuda()) \
            if self.q4 else self.rk.CachePages(p["k"].cuda(), p["v"].cuda())

    def down(self):
        """What the GPU's pools hold, unpacked."""
        q = self.pages
        if not self.q4:
            return dict(k=q.k.cpu(), v=q.v.cpu())
        return dict(k=unpack(q.k.cpu()), v=unpack(q.v.cpu()), k_scale=q.k_scale.cpu(), v_scale=q.v_scale.cpu())

    def where(self, s, h, t):
        page = int(self.table[s, h if self.head_tables else 0, t // self.ps])
        head = 0 if self.head_tables else h
        return (page, t % self.ps, head) if self.token_major else (page, head, t % self.ps)

    def rows(self, s, h, name, n=None):
        """Rows 0 .. n of a head, 64 bits; absent pages: None in `there`."""
        n = self.lens[s][h] if n is None else n
        d, there = torch.zeros(n, self.d, dtype=torch.float64), torch.ones(n, dtype=torch.bool)
        for t in range(n):
            page = int(self.table[s, h if self.head_tables else 0, t // self.ps])
            if not 0 <= page < self.c.n_pages:
                there[t] = False
                continue
            w = self.where(s, h, t)
            d[t] = from_q4(self.pool[name][w], self.pool[name + "_scale"][w]) if self.q4 else self.pool[name][w].double()
        return d, there

    def normal(self, *shape):
        return torch.randn(shape, generator=self.g)


def attention(p: Plain, q, scale=None, causal=True):
    """(out, lse, bound of out, bound of lse) [T, Hq, ...] in 64 bits for queries q [T, Hq, d] (CPU).

    Bounds of the float32 arithmetic, with u = 2^-24.  A logit is a sum of d products (4 bits: groups of sums of q (16 + code),
    scaled, and zeros added): at most (d + 8) u times the sum of the terms' magnitudes, plus 2 u of its own size for the
    scaling and 2 u for the difference with the reference.  A weight is 2^x of that: relative error of the same size and 2 u.
    Output: twice the weights' error, what the weights lose as bf16 parts (2^-17; 2^-24 in three), and a sum of
    as many terms as products follow each other (keys of a wavefront by 16, then 64 chunks and 8 more), all times the
    sum of P |v| (4 bits: of P (31 step + |zero| + 16 step))."""
    G, d = p.hq // p.hkv, p.d
    scale = d ** -0.5 if scale is None else scale
    out = torch.zeros(q.shape[0], p.hq, d, dtype=torch.float64)
    lse = torch.full((q.shape[0], p.hq), -math.inf, dtype=torch.float64)
    e_out, e_lse = torch.zeros_like(out), torch.zeros_like(lse)
    parts = F32 if p.c.out_dtype == p.rk.RESTKV_F32 else 2.0 ** -17
    for s, n in enumerate(p.new):
        n = min(n, p.c.max_new)
        for h in range(p.hkv):
            told = p.lens[s][h]
            have = min(told, p.c.max_len or told)
            k, there = p.rows(s, h, "k", have)
            v, _ = p.rows(s, h, "v", have)
            kk, vv = k.abs(), v.abs()
            if p.q4:
                kk, vv = bulk(p, s, h, "k", have), bulk(p, s, h, "v", have)
            for i in range(n):
                sees = max(0, min(have, told - n + i + 1)) if causal else have
                m = there[:sees].nonzero()[:, 0]
                if not len(m):
                    continue
                for g in range(G):
                    t, hd = p.start[s] + i, h * G + g
                    x = q[t, hd].double()
                    logit = (k[m] @ x) * scale
                    e_logit = float(F32 * ((d + 8) * ((kk[m] @ x.abs()) * scale).max() + 4 * logit.abs().max() + 4))
                    w = torch.softmax(logit, 0)
                    out[t, hd] = w @ v[m]
                    lse[t, hd] = torch.logsumexp(logit, 0)
                    terms = have / 64 + 80
                    e_out[t, hd] = (2 * e_logit + 4 * F32 + parts + terms * F32) * (w @ vv[m])
                    e_lse[t, hd] = e_logit + (terms + 4 + 2 * abs(float(lse[t, hd]))) * F32
    return out, lse, e_out, e_lse


def bulk(p, s, h, name, n):
    """Sum of the magnitudes of what a 4-bit value is put together from, [n, d]."""
    x = torch.zeros(n, p.d, dtype=torch.float64)
    f = torch.arange(p.d) % (p.d // 16) // 2
    for t in range(n):
        page = int(p.table[s, h if p.head_tables else 0, t // p.ps])
        if 0 <= page < p.c.n_pages:
            sc = p.pool[name + "_scale"][p.where(s, h, t)].double()
            x[t] = 47 * sc[f, 0] + sc[f, 1].abs()
    return x


def assert_attention(got, lse, want, out_type, rows):
    """got, lse (CPU) of the given token rows against attention()'s answer; rounding to the output's type on top."""
    out, l64, e_out, e_lse = want
    half = torch.finfo(out_type).eps / 2
    g, w, e = got[rows].double(), out[rows], e_out[rows]
    assert torch.equal(torch.isnan(g), torch.isnan(w)), "NaN in other places"
    off = (g - w).abs() - (half * (w.abs() + e) + e)
    off = torch.where(torch.isnan(w), torch.zeros_like(off), off)
    assert (off <= 0).all(), f"out: {off.max().item():.3g} over its bound, at {(off == off.max()).nonzero()[0].tolist()}"
    if lse is not None:
        a, b = lse[rows].double(), l64[rows]
        assert torch.equal(torch.isneginf(a), torch.isneginf(b)), "-inf in other places"
        fine = torch.isfinite(b)
        off = ((a - b).abs() - e_lse[rows])[fine]
        assert off.numel() == 0 or (off <= 0).all(), f"lse: {off.max().item():.3g} over its bound"
