"""Plain forms of the operators on a held pool (K and V at 8 or 4 bits) and the inputs their tests share (CPU, no code of the library).

Every element's place in the pool is worked out on its own from the format's description; the rule of quantisation is written in
numpy's binary32."""
import math

import numpy as np
import torch

from paged_reference import Batch

TILE = 16


def quantise(x, bits, span):
    """x: float tensor [..., dim] in its own type -> codes (uint8), scale, zero (fp16) [..., groups]."""
    x32 = x.float().numpy()
    with np.errstate(all="ignore"):
        if x.dtype == torch.bfloat16:
            x16 = np.where(np.isfinite(x32), np.clip(x32, -65504, 65504), np.nan).astype(np.float16)
        else:
            x16 = x32.astype(np.float16)
        g = x16.astype(np.float32).reshape(*x.shape[:-1], -1, span)
        bad = ~np.isfinite(g).all(-1)
        low, high = g.min(-1) + np.float32(0), g.max(-1)
        top = np.float32(2 ** bits - 1)
        scale = (np.abs(high - low) * (np.float32(1) / top)).astype(np.float16)      # (a range of 0 is +0 whatever the zeros' signs)
        s32 = scale.astype(np.float32)
        inverse = np.float32(1) / s32
        codes = np.minimum(np.rint((g - low[..., None]) * inverse[..., None]), top)
        codes = np.where((s32 == 0)[..., None] | bad[..., None], 0, codes).astype(np.uint8)
    scale, zero = np.where(bad, np.float16(0), scale), np.where(bad, np.float16(np.nan), low.astype(np.float16))
    return codes.reshape(x.shape), scale.astype(np.float16), zero.astype(np.float16)


def values(codes, scale, zero, dtype=None):
    """What codes stand for: float64, or rounded once to a row's type (from the exact sum, which binary32 holds to half a step)."""
    span = codes.shape[-1] // scale.shape[-1]
    v = codes.reshape(*scale.shape, span).astype(np.float64) * scale.astype(np.float64)[..., None] + zero.astype(np.float64)[..., None]
    v = torch.from_numpy(v.reshape(codes.shape))
    if dtype is None:
        return v
    v = v.float()                                             # one binary32 rounding, then the type's
    return v.clamp(-65504, 65504).half() if dtype == torch.float16 else v.to(dtype)


class Format:
    """Where the codes and parameters of a token lie in a tile."""

    def __init__(self, dim, bits, span):
        self.dim, self.bits, self.groups = dim, bits, dim // span
        W = dim * bits // 128
        VW = next(x for x in (4, 2, 1) if W % x == 0)
        self.codes, self.params = 2 * dim * bits, 64 * self.groups
        self.tile = 2 * (self.codes + self.params)
        c = np.arange(dim)
        self.byte = np.zeros((2, TILE, dim), dtype=np.int64)
        self.shift = np.zeros((2, dim), dtype=np.int64)
        for t in range(TILE):
            i = t // 8
            # K: words of 32 bits
            word, w = c // (32 // bits), c // (32 // bits) // 4
            at = ((((i * (W // VW) + w // VW) * 8 + t % 8) * 4 + word % 4) * VW + w % VW) * 4
            bit = c % (32 // bits) * bits
            self.byte[0, t] = at + bit // 8
            self.shift[0] = bit % 8
            # V: units of 16 bits, two tokens side by side
            unit, w = c // (16 // bits), c // (16 // bits) // 8
            j, e = t % 8 // 2, t % 2
            at = ((((i * (W // VW) + w // VW) * 8 + unit % 8) * 4 + j) * VW + w % VW) * 4 + e * 2
            bit = c % (16 // bits) * bits
            self.byte[1, t] = self.codes + at + bit // 8
            self.shift[1] = bit % 8
        self.param = 2 * self.codes + np.arange(2)[:, None, None, None] * self.params + (np.arange(TILE)[None, :, None, None] * self.groups
                                                                                         + np.arange(self.groups)[None, None, :, None]) * 4 + np.arange(4)

    def put(self, tile, half, t, codes, scale, zero):
        """A token's codes [dim] and parameters [groups] into a tile (uint8 [tile bytes])."""
        tile[self.byte[half, t]] = 0                           # a byte has codes of one token only
        np.bitwise_or.at(tile, self.byte[half, t], (codes.astype(np.int64) << self.shift[half]).astype(np.uint8))
        tile[self.param[half, t]] = np.stack([scale, zero], -1).view(np.uint8).reshape(self.groups, 4)

    def get(self, tiles, half, t):
        """codes [..., dim], scale, zero [..., groups] of token t of tiles [..., tile bytes]."""
        codes = (tiles[..., self.byte[half, t]] >> self.shift[half]) & (2 ** self.bits - 1)
        p = np.ascontiguousarray(tiles[..., self.param[half, t]]).view(np.float16)
        return codes.astype(np.uint8), p[..., 0], p[..., 1]


class HeldBatch(Batch):
    """A Batch whose tokens lie in a held pool.  Rows that no token lies in hold junk codes and NaN parameters."""

    def __init__(self, lens, bits=4, span=None, store=True, seed=0, **kw):
        super().__init__(lens, seed=seed, **kw)
        self.bits, self.span = bits, span or self.dim
        self.format = Format(self.dim, bits, self.span)
        g = np.random.default_rng(seed)
        self.pool = g.integers(0, 256, (self.layers, self.heads, self.n_slots * self.chunk // TILE, self.format.tile), dtype=np.uint8)
        self.pool[..., 2 * self.format.codes:] = np.frombuffer(np.float16(np.nan).tobytes() * (self.format.params), dtype=np.uint8)
        if store:
            for b in range(len(self.lens)):
                for t, row in enumerate(self.rows(b).tolist()):
                    for l in range(self.layers):
                        for h in range(self.heads):
                            for half in range(2):
                                self.store(self.pool, l, h, half, row, self.kv[l, half, h, row])

    def store(self, pool, layer, head, half, row, x):
        codes, scale, zero = quantise(x[None], self.bits, self.span)
        self.format.put(pool[layer, head, row // TILE], half, row % TILE, codes[0], scale[0], zero[0])

    def row_values(self, pool, layer, half, row, dtype=None):
        """Values of all heads [heads, dim] of a pool row."""
        return values(*self.format.get(pool[layer, :, row // TILE], half, row % TILE), dtype)


def write(batch, layer, k, v, first_row, dtype):
    """(pool, k_seen, v_seen) of a write of rows k, v [rows, heads, dim]; seen rows that are nobody's are 7."""
    b_ = batch
    pool = b_.pool.copy()
    seen = [torch.full(k.shape, 7.0, dtype=dtype) for _ in range(2)]
    for b, length in enumerate(b_.lens):
        f0, f1 = (b, b + min(1, length)) if first_row is None else (first_row[b], first_row[b + 1])
        rows = b_.rows(b).tolist()
        for r in range(f0, f1):
            row = rows[length - (f1 - r)]
            for half, x in enumerate((k, v)):
                for h in range(b_.heads):
                    b_.store(pool, layer, h, half, row, x[r, h])
                seen[half][r] = b_.row_values(pool, layer, half, row, dtype)
    return pool, seen[0], seen[1]


def attend(batch, pool=None, layer=0, window=0, append=False, scale=None):
    """(out, lse, pool, (out_tol, lse_tol)) in float64.  Tolerances: a logit is made of dim products q * code and group sums of q,
    which scale and zero-point multiply, each step off by at most 2^-23 of the terms' absolute sum (truncating adders included);
    bfloat16 queries enter exactly.  A weight then is off by twice that and a few 2^-22; the pair of 16-bit parts adds 2^-20 of
    the weighted code and 2^-29 of the largest weight times the largest scale for every code."""
    b_ = batch
    scale = b_.scale if scale is None else scale
    pool = (b_.pool if pool is None else pool).copy()
    n, G, dim = len(b_.lens), b_.group, b_.dim
    out = torch.zeros(n, b_.heads * G, dim, dtype=torch.float64)
    lse = torch.full((n, b_.heads * G), -math.inf, dtype=torch.float64)
    out_tol, lse_tol = torch.zeros_like(out), torch.zeros_like(lse)
    half_step = torch.finfo(b_.dtype).eps / 2
    groups = dim // b_.span
    for b, length in enumerate(b_.lens):
        if length == 0:
            continue
        rows = b_.rows(b).numpy()
        if append:
            for h in range(b_.heads):
                b_.store(pool, layer, h, 0, int(rows[-1]), b_.k_new[b, h])
                b_.store(pool, layer, h, 1, int(rows[-1]), b_.v_new[b, h])
        rows = rows[max(0, length - window) if window else 0:]
        parts = []                                            # (codes * scale, zero) of K, V: [tokens, heads, dim]
        top_scale = np.zeros(b_.heads)
        for half in range(2):
            c, z = np.zeros((len(rows), b_.heads, dim)), np.zeros((len(rows), b_.heads, dim))
            for t in range(TILE):
                mine = rows % TILE == t
                codes, s, zero = b_.format.get(pool[layer][:, rows[mine] // TILE], half, t)
                s, zero = (np.repeat(x.astype(np.float64), b_.span, -1) for x in (s, zero))
                c[mine], z[mine] = (codes * s).swapaxes(0, 1), zero.swapaxes(0, 1)
                if half and mine.any():
                    top_scale = np.maximum(top_scale, s.max((1, 2)))
            parts.append((torch.from_numpy(c), torch.from_numpy(z)))
        for h in range(b_.heads):
            (kc, kz), (vc, vz) = ((c[:, h], z[:, h]) for c, z in parts)
            sl = slice(h * G, (h + 1) * G)
            q = b_.q[b, sl].double()
            s = q @ (kc + kz).T * scale
            es = (q.abs() @ (kc.abs() + kz.abs()).T).amax(1, keepdim=True) * abs(scale) * (dim + groups + 4) * 2.0 ** -23
            es = es + s.abs().amax(1, keepdim=True) * 2.0 ** -21 + 2.0 ** -20 + len(rows) * 2.0 ** -24
            p = torch.softmax(s, 1)
            v = vc + vz
            lse[b, sl] = torch.logsumexp(s, 1)
            lse_tol[b, sl] = es[:, 0] + lse[b, sl].abs() * 2.0 ** -23
            out[b, sl] = p @ v
            tol = out[b, sl].abs() * half_step + (2 * es + 2.0 ** -19) * (p @ (vc.abs() + vz.abs())) + 2.0 ** -25
            lost = p.amax(1, keepdim=True) * top_scale[h] * len(rows) * (2 ** b_.bits - 1) * 2.0 ** -29
            out_tol[b, sl] = tol + lost
    return out, lse, pool, (out_tol, lse_tol)
