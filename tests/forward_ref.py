"""Plain 64-bit implementations of the calls around the forward (append,
attention, logits) on the host, with the bound on a result's error that its
arithmetic allows, and the caches that their tests run on."""
from __future__ import annotations

import math

import numpy as np
import torch

HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}   # half a step, relative
TINY = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -24}  # and below the normals


class Cache:
    """A cache whose every value outside the sequences' entries is NaN: a
    left-padded batch (page 0) or shuffled pages; `n` entries a sequence, `T`
    more for the window.  `room` further columns, or unused pages."""

    def __init__(self, n, T, H, D, page=0, layers=2, layer=1, room=3, seed=0, slots=False, width=None, device="cuda"):
        self.n, self.T, self.H, self.D, self.page, self.layer = [int(x) for x in n], T, H, D, page, layer
        B = len(self.n)
        r = np.random.default_rng(seed)
        if page:
            per = [-(-(x + T) // page) for x in self.n]
            N = sum(per) + room
            ids = r.permutation(N)
            self.table_np = np.full((B, max(per) + (0 if slots else 2)), -1, np.int32)
            at = 0
            for i, m in enumerate(per):
                self.table_np[i, :m] = ids[at:at + m]
                at += m
            self.max_len = max(self.n) + T
            shape = (layers, 2, N, H, page, D)
            self.table = torch.as_tensor(self.table_np, device=device)
            self.lens = torch.as_tensor(np.asarray(self.n, np.int32), device=device)
        else:
            self.W_in = width or max(self.n) + T
            shape = (layers, 2, B, H, self.W_in + room, D)
            self.pad_np = np.asarray([self.W_in - T - x for x in self.n], np.int32)
            self.pad = torch.as_tensor(self.pad_np, device=device)
        self.kv = torch.full(shape, float("nan"), dtype=torch.bfloat16)
        self.shape = shape

    def where(self, i, j):
        if self.page:
            return int(self.table_np[i, j // self.page]), j % self.page
        return i, int(self.pad_np[i]) + j

    def fill(self, count, g, scale=1.0):
        """Random entries 0 .. n + count - 1 of every sequence, on the host."""
        for i, x in enumerate(self.n):
            m = x + count
            if not m:
                continue
            rows, cols = zip(*(self.where(i, j) for j in range(m)))
            e = (scale * torch.randn((2, m, self.H, self.D), generator=g)).to(torch.bfloat16)
            for part in range(2):
                self.kv[self.layer, part][torch.tensor(rows), :, torch.tensor(cols)] = e[part]
        return self

    def entries(self, i, m):
        """Entries 0 .. m - 1 of sequence i: (keys, values), each [m][H][D] fp64."""
        rows, cols = zip(*(self.where(i, j) for j in range(m)))
        kv = self.kv[self.layer]
        return tuple(kv[p][torch.tensor(rows), :, torch.tensor(cols)].double() for p in (0, 1))


def append(x, q_heads, H, n, T, q_norm, k_norm, eps, inv_freq, adjacent):
    """One sequence's projections x [T][Hq+2H][D] -> (queries and keys [T][Hq+H][D], values, bound on the fp32 error of
    the former): bound = (|a| + |b|) * 2^-18.

    The fp32 path: a norm's sum has 8 + 5 rounding steps, its root, quotient and products 5 more: a relative error below
    2^-19; the angle's fraction of a turn is rounded once (2^-25 of a turn, 2^-22 in sine and cosine with their own
    error), two products and a sum add 3 * 2^-24."""
    D = x.shape[-1]
    x = x.double()
    y = x[:, : q_heads + H].clone()
    for sl, w in ((slice(0, q_heads), q_norm), (slice(q_heads, q_heads + H), k_norm)):
        if w is not None:
            y[:, sl] = y[:, sl] / torch.sqrt((y[:, sl] ** 2).sum(-1, keepdim=True) / D + eps) * w.double()
    out, size = y.clone(), y.abs()
    for j in range(0 if inv_freq is None else inv_freq.numel()):
        a, b = (2 * j, 2 * j + 1) if adjacent else (j, j + inv_freq.numel())
        for r in range(T):
            t = (n + r) * float(inv_freq[j])
            c, s = math.cos(t), math.sin(t)
            out[r, :, a] = y[r, :, a] * c - y[r, :, b] * s
            out[r, :, b] = y[r, :, b] * c + y[r, :, a] * s
        both = y[:, :, a].abs() + y[:, :, b].abs()
        size[:, :, a] = both
        size[:, :, b] = both
    return out, x[:, q_heads + H:], size * 2.0 ** -18


def attend(q, k, v, n, scale):
    """One sequence: q [T][Hq][D], k and v [n + T][H][D] -> (out [T][Hq][D] fp64, bound on the error of a bf16 result).

    A weight's relative error e: its rounding to bf16 (2^-8), and twice the score's absolute error (D fp32 sums of
    products, each off by 2^-24 of the sum of their magnitudes; 2^-22 of the score in the exponential's argument) and the
    exponential's own.  Weights off by e move the normed sum by at most 2 e (sum p |v| + |out|); its fp32 sums add at most
    one rounding an entry of a lane (n / 32 and the joins), the output's rounding half a step."""
    T, Hq, D = q.shape
    H = k.shape[1]
    q = q.double()
    out = torch.zeros((T, Hq, D), dtype=torch.float64)
    bound = torch.zeros_like(out)
    for h in range(Hq):
        kh, vh = k[:, h // (Hq // H)], v[:, h // (Hq // H)]
        for r in range(T):
            m = n + r + 1
            z = scale * (kh[:m] @ q[r, h])
            p = torch.softmax(z, 0)
            out[r, h] = p @ vh[:m]
            dz = float((abs(scale) * (kh[:m].abs() @ q[r, h].abs())).max()) * (D * 2.0 ** -24) + float(z.abs().max()) * 2.0 ** -21
            e = 2.0 ** -8 + 2 * dz + 2.0 ** -20
            sums = (m / 32 + 64) * 2.0 ** -24
            mag = p @ vh[:m].abs()
            bound[r, h] = (2 * e + sums) * (mag + out[r, h].abs()) + 2.0 ** -8 * out[r, h].abs() + 2.0 ** -133
    return out, bound


def logits(x, hist, drafts, prompt, rep, pres, freq, bias, mask, dtype):
    """One sequence: x [k+1][V] -> (out fp64, bound on the error of a result in `dtype`).  hist: list of tokens; bias:
    list of (id, value); mask: bool [k+1][V] or None."""
    y = x.double().clone()
    R, V = y.shape
    size = torch.zeros_like(y)
    for r in range(R):
        told, held = {}, set()
        for j, t in enumerate(list(hist) + list(drafts[:r])):
            if not 0 <= t < V:
                continue
            held.add(t)
            if j >= prompt:
                told[t] = told.get(t, 0) + 1
        for t in held:
            if rep is not None:
                y[r, t] = y[r, t] / rep if y[r, t] > 0 else y[r, t] * rep
            size[r, t] = y[r, t].abs()
        for t, m in told.items():
            less = (freq or 0.0) * m + (pres or 0.0)
            y[r, t] -= less
            size[r, t] += abs(less)
        for t, b in bias:
            if 0 <= t < V:
                size[r, t] += y[r, t].abs() + abs(b)
                y[r, t] += b
        if mask is not None:
            y[r][~mask[r]] = -math.inf
    size = torch.nan_to_num(size, posinf=0.0)
    # at most 4 fp32 roundings and one a bias, each relative to the magnitudes met
    b = size * (4 + len(bias)) * 2.0 ** -24 + HALF[dtype] * torch.nan_to_num(y, posinf=0.0, neginf=0.0).abs() * (1 + 2.0 ** -10)
    return y, b + TINY[dtype]


def check(got, want, bound, what):
    """Elementwise |got - want| <= bound; infinities and NaN in the same places."""
    got = got.detach().double().cpu()
    assert got.shape == want.shape, what
    fine = torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want)), f"{what}: NaN in other places"
    assert torch.equal(got[~fine & ~torch.isnan(want)], want[~fine & ~torch.isnan(want)]), f"{what}: infinities differ"
    off = (got - want).abs()[fine]
    over = off > bound[fine]
    assert not bool(over.any()), (f"{what}: {int(over.sum())} of {over.numel()} beyond the bound, worst "
                                  f"{float((off / bound[fine]).max()):.3g} times it")
