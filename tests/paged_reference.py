"""Plain 64-bit forms of the paged-cache operators and the inputs their tests share (CPU, no code of the library)."""
import math

import torch

SPARE = 3     # slots of a test pool that no sequence lists


class Batch:
    """A pool, a batch of sequences in it and the operands of a decode call, in host memory.
    Every pool row that holds no token is filled with `junk` (NaN unless the pool is to be compressed)."""

    def __init__(self, lens, heads=2, group=1, dim=64, chunk=16, dtype=torch.float16, layers=1, seed=0, max_len=None, junk=math.nan,
                 gain=1.0):
        g = torch.Generator().manual_seed(seed)
        self.lens, self.heads, self.group, self.dim, self.chunk, self.dtype, self.layers = list(lens), heads, group, dim, chunk, dtype, layers
        self.max_len = max_len or max(max(lens), 1)
        n = len(lens)
        width = -(-self.max_len // chunk)
        need = [-(-x // chunk) for x in lens]
        self.n_slots = sum(need) + SPARE
        order = torch.randperm(self.n_slots, generator=g).tolist()
        self.table = torch.full((n, width), -7, dtype=torch.int32)
        for b in range(n):
            for i in range(need[b]):
                self.table[b, i] = order.pop()
        self.kv = torch.full((layers, 2, heads, self.n_slots * chunk, dim), junk, dtype=dtype)
        for b in range(n):
            rows = self.rows(b)
            x = torch.randn(layers, 2, heads, len(rows), dim, generator=g, dtype=torch.float64)
            x[:, 0] *= gain
            self.kv[:, :, :, rows] = x.to(dtype)
        qkv = torch.randn(n, heads * (group + 2), dim, generator=g, dtype=torch.float64).to(dtype)
        self.q, self.k_new, self.v_new = qkv[:, :heads * group], qkv[:, heads * group:heads * (group + 1)], qkv[:, heads * (group + 1):]
        self.qkv = qkv
        self.mass = torch.rand(layers, n, heads, self.max_len, generator=g).pow(6) * 20
        self.mass[self.mass < 1e-3] = 0.0

    def rows(self, b, table=None, upto=None):
        """Pool rows of the tokens of sequence b."""
        table = self.table if table is None else table
        t = torch.arange(self.lens[b] if upto is None else upto)
        return table[b].long()[t // self.chunk] * self.chunk + t % self.chunk

    @property
    def scale(self):
        return self.dim ** -0.5


def attend(batch, layer=0, window=0, append=False, mass_in=None, mass_before=None, scale=None):
    """(out, lse, mass, kv, bounds) in float64.  bounds: how far out, lse and mass may be off by the arithmetic alone:
    a logit is a sum of dim products in binary32 (each addition off by at most 2^-23 of the terms' absolute sum, truncating
    adders included) -> es; a weight exp(s - lse) then by 2 es and a few 2^-22 (exponential, sum, the pair of 16-bit parts:
    2^-16); everything a weight is multiplied with adds up with the weights."""
    b_ = batch
    scale = b_.scale if scale is None else scale
    kv = b_.kv.clone()
    n, G, dim = len(b_.lens), b_.group, b_.dim
    out = torch.zeros(n, b_.heads * G, dim, dtype=torch.float64)
    lse = torch.full((n, b_.heads * G), -math.inf, dtype=torch.float64)
    mass = None if mass_before is None else mass_before.double().clone()
    out_tol, lse_tol = torch.zeros_like(out), torch.zeros_like(lse)
    mass_tol = None if mass is None else torch.zeros_like(mass)
    half = torch.finfo(b_.dtype).eps / 2
    for b, length in enumerate(b_.lens):
        if length == 0:
            continue
        rows = b_.rows(b)
        if append:
            kv[layer, 0, :, rows[-1]] = b_.k_new[b]
            kv[layer, 1, :, rows[-1]] = b_.v_new[b]
        if mass is not None:
            old = torch.zeros(b_.heads, length, dtype=torch.float64) if mass_in is None else mass_in[b, :, :length].double()
            mass[b, :, :length] = old
            mass_tol[b, :, :length] = old * 2.0 ** -23
        first = max(0, length - window) if window else 0
        for h in range(b_.heads):
            k, v = kv[layer, 0, h, rows[first:]].double(), kv[layer, 1, h, rows[first:]].double()
            q = b_.q[b, h * G:(h + 1) * G].double()
            s = q @ k.T * scale
            es = (q.abs() @ k.abs().T).amax(1, keepdim=True) * abs(scale) * dim * 2.0 ** -23 + s.abs().amax(1, keepdim=True) * 2.0 ** -21
            es = es + 2.0 ** -20 + len(rows) * 2.0 ** -24
            p = torch.softmax(s, 1)
            sl = slice(h * G, (h + 1) * G)
            lse[b, sl] = torch.logsumexp(s, 1)
            lse_tol[b, sl] = es[:, 0] + lse[b, sl].abs() * 2.0 ** -23
            out[b, sl] = p @ v
            out_tol[b, sl] = out[b, sl].abs() * half + (2 * es + 2.0 ** -16) * (p @ v.abs()) + 2.0 ** -25
            if mass is not None:
                mass[b, h, first:length] += p.sum(0)
                mass_tol[b, h, first:length] += (2 * es * p).sum(0) + p.sum(0) * 2.0 ** -22
    return out, lse, mass, kv, (out_tol, lse_tol, mass_tol)


def evict(batch, mass, budget, recent, dst_table=None, mass_before=None):
    """(kept, new_lens, mass_out, kv): sorted by (mass descending, position ascending), NaN and -inf last."""
    b_ = batch
    L, n, H, _ = mass.shape
    kept = torch.full((L, n, H, budget), -1, dtype=torch.int32)
    out = mass.clone() if mass_before is None else mass_before.clone()
    kv = b_.kv.clone()
    new_lens = torch.tensor([min(budget, x) for x in b_.lens], dtype=torch.int32)
    for b, length in enumerate(b_.lens):
        m = min(budget, length)
        if m == 0:
            continue
        r = min(recent, m)
        src = b_.rows(b)
        dst = b_.rows(b, dst_table, m)
        for l in range(L):
            for h in range(H):
                w = mass[l, b, h, :length].tolist()
                order = sorted(range(length - r), key=lambda t: (-(w[t] if w[t] == w[t] else -math.inf), t))
                ids = sorted(order[:m - r]) + list(range(length - r, length))
                kept[l, b, h, :m] = torch.tensor(ids, dtype=torch.int32)
                out[l, b, h, :length] = 0
                out[l, b, h, :m] = mass[l, b, h, ids]
                kv[l, :, h, dst] = b_.kv[l, :, h, src[ids]]
    return kept, new_lens, out, kv


def bits(t):
    return t.contiguous().view(torch.int16)
