"""Plain 64-bit implementations of drafted trees and selected blocks for the GPU tests, and the error bounds of their comparisons."""
from __future__ import annotations

import math

import numpy as np
import torch

import serving_ref as ref

U_BF16, U_F16, U_F32 = ref.U_BF16, ref.U_F16, ref.U_F32


def tree(rng, n, chain=0.0):
    """Parents of a random tree of n nodes; with probability `chain` a node hangs on the one before it."""
    return [-1] + [i - 1 if rng.random() < chain else rng.randrange(i) for i in range(1, n)]


def plan(parents, words):
    """(depths, mask words as int64) of one request, or None where a parent does not come before its node."""
    sees, depths = [], []
    for i, p in enumerate(parents):
        if not -1 <= p < i:
            return None
        sees.append((sees[p] if p >= 0 else 0) | 1 << i)
        depths.append(depths[p] + 1 if p >= 0 else 0)
    mask = np.array([[s >> 32 * w & 0xFFFFFFFF for w in range(words)] for s in sees], np.uint32).reshape(len(parents), words)
    return depths, mask.view(np.int32)


def bits_of(mask, n):
    """[rows, n] truth values of mask words (int32, [rows, words])."""
    m = np.asarray(mask, np.int32)
    b = np.unpackbits(m.view(np.uint8).reshape(m.shape[0], -1), axis=1, bitorder="little")
    return np.pad(b, ((0, 0), (0, max(0, n - b.shape[1]))))[:, :n].astype(bool)


def walk(parents, tokens, choices):
    """Accepted nodes of one request."""
    way = [0]
    while True:
        at = way[-1]
        to = [c for c in range(at + 1, len(parents)) if parents[c] == at and tokens[c] == choices[at]]
        if not to:
            return way
        way.append(to[0])


def attend_seen(q, cache, layer, q_start, lens, tables, n_kv, scale, fill, see_of):
    """(out, lse, tol, lse_tol) in 64 bits; see_of(r, head, n): [new tokens, n] truth values, which keys a row sees (keys that the table does not name
    are left out here).  Rows outside every request, and requests for which see_of gives None, keep `fill`."""
    T, hq, d = q.shape
    g, dev = hq // n_kv, q.device
    out = torch.full((T, hq, d), float(fill), dtype=torch.float64, device=dev)
    lse = torch.full((T, hq), float(fill), dtype=torch.float64, device=dev)
    tol, ltol = torch.zeros_like(out), torch.zeros_like(lse)
    u_p = U_F16 if cache.fp8 else U_BF16
    for r in range(len(lens)):
        a, b, n = q_start[r], q_start[r + 1], lens[r]
        if not (0 <= a <= b <= T) or n < 0 or a == b:
            continue
        k, v, ok = ref.cache_rows(cache, layer, tables[r], n, cache.num_blocks)
        for h in range(hq):
            see = see_of(r, h // g, n)
            if see is None:
                continue
            see = torch.as_tensor(np.asarray(see), device=dev) & ok[None]
            kh, vh, x = k[:, h // g], v[:, h // g], q[a:b, h].double()
            if n == 0:
                out[a:b, h], lse[a:b, h] = 0.0, -math.inf
                continue
            s = torch.where(see, (x @ torch.nan_to_num(kh).T) * scale, -math.inf)
            m = s.amax(1, keepdim=True)
            w = torch.where(see, torch.exp(s - torch.where(torch.isinf(m), 0.0, m)), 0.0)
            total = w.sum(1, keepdim=True)
            l1 = torch.where(total == 0, 1.0, total)
            vz = torch.where(torch.isfinite(vh), vh, 0.0)
            o = (w @ vz) / l1
            for j in (~torch.isfinite(vh)).any(1).nonzero().flatten().tolist():  # values that are not finite count where they are seen
                bad = torch.where(torch.isfinite(vh[j]), 0.0, vh[j])
                o += torch.where(see[:, j, None] & ~torch.isfinite(vh[j])[None], w[:, j, None] * bad[None], 0.0)
            out[a:b, h] = o
            lse[a:b, h] = (m + torch.log(l1))[:, 0]
            # fp32 accumulation of d products, scaling and exp2 in fp32: absolute error of a score in natural units
            ds = scale * ((x.abs() @ torch.nan_to_num(kh).abs().T) * see).amax(1, keepdim=True) * (d + 8) * U_F32 + 2.0**-20
            av = (w @ vz.abs()) / l1
            t = U_BF16 * o.abs() + (u_p + 3 * ds) * av + 1e-30
            if cache.fp8:  # fp16 weights below 2^-14 of the largest have an absolute step of 2^-25
                t = t + 2.0**-25 * (see.double() @ vz.abs()) / l1
            tol[a:b, h] = t
            ltol[a:b, h] = (2 * ds + U_F32 * 4 * torch.nan_to_num(m, neginf=0.0).abs() + 2.0**-20)[:, 0]
    return out, lse, tol, ltol


def scores(q, box):
    """Scores of blocks in 64 bits: q [group, d], box [blocks, 2, d]; NaN stays."""
    x = q.double()[:, None]
    # (the form of the definition with sums of positive and negative parts: a coordinate where q is zero and a bound infinite is NaN in both)
    p, n = x.clamp(min=0).sum(0), x.clamp(max=0).sum(0)
    return (p * box[:, 1].double() + n * box[:, 0].double()).sum(1)


def magnitudes(q, box):
    """Sums of the magnitudes of what `scores` sums."""
    x = q.double()[:, None]
    p, n = x.clamp(min=0).sum(0), x.clamp(max=0).sum(0)
    return (p * box[:, 1].double().abs() - n * box[:, 0].double().abs()).sum(1)


def choose(score, named, n_select, n_first, n_last, all_blocks):
    """Chosen blocks in rising order: score fp32 [blocks], named: which the table names."""
    s = np.where(np.isnan(score), np.inf, score)
    must = [b for b in range(len(s)) if named[b] and (b < n_first or b >= all_blocks - n_last)]
    rest = [b for b in np.argsort(-s, kind="stable") if named[b] and b not in set(must)]
    return sorted(must + [int(b) for b in rest[: max(0, n_select - len(must))]])
