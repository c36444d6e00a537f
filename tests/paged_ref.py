"""Plain 64-bit forms of the paged-cache operators, and inputs for their tests.

Error bounds of the attention outputs, per row and head, from the arithmetic: with weights w_j
of the visible keys and A = sum_j w_j |v_j|,
  * the output's own rounding: H |out|, H half a step of the type (2^-8 or 2^-24);
  * a relative error d of every unnormalised weight moves the ratio by at most 2 d A; d holds the
    weight's rounding to the storage type before the product with V (H for bf16), the score's
    error, at most scale * (hd + 4) * 2^-24 * sum_d |q_d k_jd| + 4 * 2^-24 * |s_j - max|, and the
    exponential's, 2^-22;
  * sums over n keys in fp32: (n + 64) 2^-24 A on either side of the ratio.
"""
from __future__ import annotations

import math

import numpy as np
import torch

PAGE = 16


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


class Case:
    """A cache with pages in random order, filled with `fill` where no sequence's keys lie."""

    def __init__(self, rows, keys, heads, dtype, seed=0, ragged=True, extra_rows=0, shared=0, extra_pages=3,
                 q_pad=0, max_pages=None, fill=None):
        hq, hkv, hd = heads
        g = torch.Generator().manual_seed(seed)
        self.rows, self.keys, self.hq, self.hkv, self.hd, self.dtype = rows, keys, hq, hkv, hd, dtype
        self.n = sum(rows) + extra_rows
        sh = shared // PAGE
        need = [max(0, (k + PAGE - 1) // PAGE - sh) for k in keys]
        self.width = max_pages or max(1, sh + max(need))
        self.n_pages = sh + sum(need) + extra_pages
        order = torch.randperm(self.n_pages, generator=g).tolist()
        self.table = torch.full((len(rows), self.width), -1, dtype=torch.int32)
        at = sh
        for s, c in enumerate(need):
            ids = (order[:sh] + order[at:at + c])[:self.width]
            self.table[s, :len(ids)] = torch.tensor(ids, dtype=torch.int32)
            at += c
        kp = torch.randn(self.n_pages, hkv, PAGE, hd, generator=g)
        vp = torch.randn(self.n_pages, hkv, hd, PAGE, generator=g)
        if fill is not None:
            used_k, used_v = torch.zeros_like(kp, dtype=torch.bool), torch.zeros_like(vp, dtype=torch.bool)
            for s, k in enumerate(keys):
                for j in range(k):
                    used_k[self.table[s, j // PAGE], :, j % PAGE] = True
                    used_v[self.table[s, j // PAGE], :, :, j % PAGE] = True
            kp[~used_k] = fill
            vp[~used_v] = fill
        self.kp, self.vp = kp.to(dtype), vp.to(dtype)
        full = torch.randn(self.n, hq * hd + q_pad, generator=g) * 1.5
        self.q_full = full.to(dtype)
        self.start = torch.tensor([0] + list(np.cumsum(rows)), dtype=torch.int32) if ragged else None
        self.kv_len = torch.tensor(keys, dtype=torch.int32)

    @property
    def q(self):
        return self.q_full[:, :self.hq * self.hd].unflatten(1, (self.hq, self.hd))

    def first(self, s):
        return int(sum(self.rows[:s]))

    def place(self, s, j):
        """Page and slot of position j of sequence s."""
        return int(self.table[s, j // PAGE]), j % PAGE

    def keys_of(self, s):
        k = max(0, min(self.keys[s], self.width * PAGE))
        pages = self.table[s, :(k + PAGE - 1) // PAGE].long()
        ok = ((pages >= 0) & (pages < self.n_pages)).repeat_interleave(PAGE)[:k]
        pages = pages.clamp(0, self.n_pages - 1)
        K = self.kp[pages].transpose(1, 2).reshape(-1, self.hkv, self.hd)[:k].double()
        V = self.vp[pages].permute(0, 3, 1, 2).reshape(-1, self.hkv, self.hd)[:k].double()
        return K, V, ok

    def to(self, device):
        q = self.q_full.to(device)[:, :self.hq * self.hd].unflatten(1, (self.hq, self.hd))
        return dict(k=self.kp.to(device), v=self.vp.to(device), table=self.table.to(device), q=q,
                    kv_len=self.kv_len.to(device), start=None if self.start is None else self.start.to(device))


def ref_attention(c: Case, window=0, sinks=0, scale=None):
    """(out, bound) [rows][heads][hd] in float64; rows of no sequence: zeros and infinity."""
    scale = scale or 1 / math.sqrt(c.hd)
    G, H = c.hq // c.hkv, half_step(c.dtype)
    out = torch.zeros(c.n, c.hq, c.hd, dtype=torch.float64)
    tol = torch.full((c.n, c.hq, c.hd), math.inf, dtype=torch.float64)
    u = 2.0 ** -24
    for s, n in enumerate(c.rows):
        if n == 0:
            continue
        K, V, ok = c.keys_of(s)
        a = c.first(s)
        pos = (c.keys[s] - n + torch.arange(n))[:, None]
        j = torch.arange(K.shape[0])[None]
        vis = ok[None] & (j <= pos)
        if window:
            vis = vis & ((j > pos - window) | (j < sinks))
        for h in range(c.hkv):
            q = c.q[a:a + n, h * G:(h + 1) * G].double().transpose(0, 1)               # [G][n][hd]
            k, v = K[:, h], V[:, h]
            kz = torch.where(torch.isfinite(k), k, 0.0)
            sc = scale * (q @ k.T)          # column j has key j alone
            sc = torch.where(vis, sc, -math.inf)
            m = sc.amax(-1, keepdim=True) if K.shape[0] else torch.full(sc.shape[:2] + (1,), -math.inf).double()
            m0 = torch.where(m == -math.inf, 0.0, m)
            w = torch.exp(sc - m0)
            den = w.sum(-1, keepdim=True)
            w = torch.where(den > 0, w / den, torch.where(den == 0, 0.0, torch.nan))
            vf = torch.where(torch.isfinite(v), v, 0.0)
            o = w @ vf
            # visible keys with non-finite values, one by one (a weight of zero meets none of them)
            for jj in torch.nonzero(~torch.isfinite(v).all(-1)).flatten().tolist():
                add = torch.where((w[..., jj] > 0)[..., None], w[..., jj][..., None] * (v[jj] - vf[jj]), 0.0)
                o = o + torch.nan_to_num(add, nan=math.nan, posinf=math.inf, neginf=-math.inf)
            A = w @ vf.abs()
            sabs = scale * (q.abs() @ kz.abs().T)
            gap = torch.where(vis, (sc - m0).abs(), 0.0)
            d = torch.where(vis & (w > 0), (c.hd + 4) * u * sabs + 4 * u * gap, 0.0).amax(-1, keepdim=True) \
                if K.shape[0] else torch.zeros(sc.shape[:2] + (1,)).double()
            d = d + 2.0 ** -22 + (H if c.dtype == torch.bfloat16 else 0.0)
            nk = K.shape[0]
            t = H * o.abs() + (2 * d + 2 * (nk + 64) * u) * A * (1 + 2 ** -6) + 1e-30
            out[a:a + n, h * G:(h + 1) * G] = o.transpose(0, 1)
            tol[a:a + n, h * G:(h + 1) * G] = t.transpose(0, 1)
    return out, tol


def ref_append(c: Case, q, k, v, rope=None, rot=0, q_norm=None, k_norm=None, eps=1e-6):
    """(q_out, K pages, V pages) in float64 and their bounds: half a step of the stored value, and
    fp32 arithmetic of a norm (relative (hd / 2 + 8) 2^-24) and of two products and a sum."""
    H, u = half_step(c.dtype), 2.0 ** -24
    cap = c.width * PAGE
    qo = torch.full((c.n, c.hq, c.hd), math.nan, dtype=torch.float64)
    qt = torch.full_like(qo, math.inf)
    kp, vp = c.kp.double(), c.vp.double()
    kt, vt = torch.zeros_like(kp), torch.zeros_like(vp)

    def turn(x, w, p):
        x = x.double()
        rel = 2 * u
        if w is not None:
            x = x / torch.sqrt(x.square().mean(-1, keepdim=True) + eps) * w.double()
            rel = (c.hd / 2 + 8) * u
        mag = x.abs()
        if rope is not None:
            h = rot // 2
            cs, sn = rope[0, p].double(), rope[1, p].double()
            a, b = x[..., :h], x[..., h:rot]
            mag = torch.cat([(a * cs).abs() + (b * sn).abs(), (b * cs).abs() + (a * sn).abs(), mag[..., rot:]], -1)
            x = torch.cat([a * cs - b * sn, b * cs + a * sn, x[..., rot:]], -1)
        return x, H * x.abs() + (rel + 4 * u) * mag * (1 + 2 ** -6) + 1e-30

    for s, n in enumerate(c.rows):
        for i in range(n):
            r, p = c.first(s) + i, c.keys[s] - n + i
            if p < 0 or p >= cap:
                continue
            if q is not None:
                qo[r], qt[r] = turn(q[r], q_norm, p)
            page, slot = c.place(s, p)
            if not 0 <= page < c.n_pages:
                continue
            kp[page, :, slot], kt[page, :, slot] = turn(k[r], k_norm, p)
            vp[page, :, :, slot] = v[r].double()
            vt[page, :, :, slot] = H * v[r].double().abs() if v.dtype != c.dtype else 0.0
    return (qo, qt), (kp, kt), (vp, vt)
