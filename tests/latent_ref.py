"""The latent cache's operators by their definition, in 64 bits (not collected: no test_ prefix).

Rounding errors that the tests allow, as shares of a row's 2-norm.  A rounding to
bf16 is off by at most 2^-8 of the value, and by 0.0017 of it in the root mean square
(uniform errors within half steps, mantissas spread over a power of two); to fp32
by 2^-16 times that.

* bf16 attention rounds the queries in the latents' space (or the keys made from
  the latents), whose errors reach a score as 0.0017 times the root of its products'
  squares summed, at most about 0.0017 where scores' deviation is 1; the
  probabilities; the sums of latents (or the values); and the output: 0.0017 sqrt(4),
  and 2.5 times that for the scatter from row to row.
* fp32 sums of n products in one chain are off by about sqrt(n) 2^-24 of the
  products' root square sum: 24 for a score's up to 576, less for the products on both
  sides, exponents of up to 2^4 by 2^4 2^-24, sums over keys in chains of a few
  hundred 20: 128 2^-24 bounds their square sum 2.5 times over.
"""

import math

import numpy as np
import torch

RMS_BF16 = 0.0017
TOL = {torch.bfloat16: 2.5 * 2 * RMS_BF16, torch.float32: 128 * 2.0 ** -24}


def rotate(x, pos, theta):
    """fp64 x [R, heads, rope], pairs (i, i + rope / 2) turned by pos theta^(-2i / rope)."""
    half = x.shape[-1] // 2
    angle = pos.double()[:, None] * float(np.float32(theta)) ** (-torch.arange(half, dtype=torch.float64, device=x.device) / half)
    c, s = angle.cos()[:, None], angle.sin()[:, None]
    a, b = x[..., :half], x[..., half:]
    return torch.cat([a * c - b * s, b * c + a * s], -1)


def append(q, kv, norm_w, pos, H, nope, rope, rank, theta, eps):
    """(q rotated [R, H, nope + rope], entries [R, rank + rope]) in fp64."""
    q = q.double().view(-1, H, nope + rope)
    kv = kv.double()
    c = kv[:, :rank]
    c = c / (c.square().mean(1, keepdim=True) + float(np.float32(eps))).sqrt() * norm_w.double()
    return (torch.cat([q[..., :nope], rotate(q[..., nope:], pos, theta)], -1),
            torch.cat([c, rotate(kv[:, None, rank:], pos, theta)[:, 0]], 1))


def attend(q, held, pos0, w_k, w_v, scale, rank):
    """One sequence: q [r, H, nope + rope] at pos0.., held [pos0 + r, rank + rope] -> fp64 [r, H, v].  A key that a row does
    not see takes no part in it, whatever it holds."""
    r, H, _ = q.shape
    nope = w_k.shape[1]
    out = torch.empty(r, H, w_v.shape[1], dtype=torch.float64, device=q.device)
    held = held.double()
    c, key = held[:, :rank].contiguous(), held[:, rank:].contiguous()
    hidden = torch.arange(len(held), device=q.device) > pos0 + torch.arange(r, device=q.device)[:, None]
    for h in range(H):
        k = torch.cat([c @ w_k[h].double().t().contiguous(), key], 1)
        v = c @ w_v[h].double().t().contiguous()
        w = (q[:, h].double() @ k.t().contiguous() * scale).masked_fill(hidden, -math.inf)
        p = torch.softmax(w, 1)
        o = p @ torch.where(torch.isfinite(v), v, 0.0)
        for t in torch.nonzero(~torch.isfinite(v).all(1))[:, 0].tolist():  # what such a value does to the rows that see it
            o = torch.where(hidden[:, t:t + 1], o, o + p[:, t:t + 1] * v[t])
        out[:, h] = o
    return out


class Case:
    """A batch over a shuffled cache: pages that no sequence has, and slots past a sequence's end, hold NaN."""

    def __init__(self, dtype, rows, pos0, H, nope=128, rope=64, rank=512, v=128, seed=0, spare=3, sharp=1.0):
        g = torch.Generator(device="cuda")
        g.manual_seed(1000 + seed)
        rng = np.random.default_rng(seed)
        self.dtype, self.H, self.nope, self.rope, self.rank, self.v = dtype, H, nope, rope, rank, v
        self.rows, self.pos0 = np.array(rows, np.int32), np.array(pos0, np.int32)
        need = [(r + p + 15) // 16 if r else 0 for r, p in zip(rows, pos0)]
        self.P = sum(need) + spare
        perm = rng.permutation(self.P).astype(np.int32)
        self.table = np.full((len(rows), max(need) + 1), -1, np.int32)  # entries that no row needs are never read
        o = 0
        for i, n in enumerate(need):
            self.table[i, :n] = perm[o:o + n]
            o += n
        self.pages = torch.full((self.P, 16, rank + rope), math.nan, dtype=dtype, device="cuda")
        for i, (r, p) in enumerate(zip(rows, pos0)):
            if r:
                t = torch.arange(r + p, device="cuda")
                page = torch.from_numpy(self.table[i].astype(np.int64)).to("cuda")[t // 16]
                self.pages[page, t % 16] = torch.randn(r + p, rank + rope, generator=g, device="cuda").to(dtype)
        self.q = (sharp * torch.randn(int(self.rows.sum()), H, nope + rope, generator=g, device="cuda")).to(dtype)
        w = (torch.randn(H, nope + v, rank, generator=g, device="cuda") / math.sqrt(rank)).to(dtype)
        self.w_k, self.w_v = w[:, :nope], w[:, nope:]
        self.scale = 1 / math.sqrt(nope + rope)
        self.out = torch.full((int(self.rows.sum()) + 2, H * v), 7.0, dtype=dtype, device="cuda")

    def args(self, B):
        return (B.SPEC_F32 if self.dtype is torch.float32 else B.SPEC_BF16, self.rows, self.pos0)

    def workspace(self, B):
        n = B.spec_op_attention_latent_workspace_bytes(*self.args(B), self.table.shape[1], self.H, self.nope, self.rope,
                                                       self.rank, self.v)
        return torch.full((n + 256,), 0xFF, dtype=torch.uint8, device="cuda")  # NaN wherever nothing was written

    def run(self, B, ws=None, stream=None):
        ws = self.workspace(B) if ws is None else ws
        B.spec_op_attention_latent(*self.args(B), self.table, self.P, self.H, self.nope, self.rope, self.rank, self.v,
                                   self.scale, self.q, self.pages, self.w_k, self.w_v, self.out, ws, stream)
        return self.out[:len(self.q)].view(-1, self.H, self.v)

    def slots(self, i):
        t = np.arange(self.rows[i] + self.pos0[i])
        return torch.from_numpy(self.table[i][t // 16].astype(np.int64) * 16 + t % 16).to("cuda")

    def ref(self):
        flat, got, r0 = self.pages.view(-1, self.rank + self.rope), [], 0
        for i, r in enumerate(self.rows.tolist()):
            if r:
                got.append(attend(self.q[r0:r0 + r], flat[self.slots(i)], int(self.pos0[i]), self.w_k, self.w_v, self.scale,
                                  self.rank))
            r0 += r
        return torch.cat(got)


def row_error(got, ref):
    """Largest relative 2-norm of the difference over the last dim."""
    return float(((got.double() - ref).norm(dim=-1) / ref.norm(dim=-1)).max())
