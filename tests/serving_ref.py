"""Plain 64-bit implementations of the serving calls (block tables, append, attention) for the GPU tests, and the error bounds
that their comparisons use."""
from __future__ import annotations

import math

import numpy as np
import torch

F8 = torch.float8_e4m3fn
U_BF16, U_F16, U_F32, U_E4M3 = 2.0**-8, 2.0**-11, 2.0**-24, 2.0**-4


def grow(start, new, tables, free, taken, bs, num_blocks, capacity, max_position, max_blocks):
    """The allocation rule of memstore_grow_blocks, request after request."""
    tables, free = np.array(tables, np.int64), list(free)
    n_free, taken0 = len(free), taken
    list_ok = 0 <= taken <= n_free
    asked, upto, q_start, lens, status = 0, 0, [0], [], []
    pos_out, slot_out = np.full(capacity, -1, np.int64), np.full(capacity, -1, np.int64)
    for r, (s, n_in) in enumerate(zip(start, new)):
        n = max(n_in, 0)
        st = (64 if s < 0 else 0) | (256 if n_in < 0 else 0)
        upto += n
        if n > 0 and upto > capacity:
            st |= 256
        if s + n > max_position:
            st |= 16
        held, want = -(-max(s, 0) // bs), -(-max(s + n, 0) // bs)
        if want > max_blocks:
            st |= 4
        if st == 0:
            asked += want - held
            if want > held and not (list_ok and taken0 + asked <= n_free):
                st |= 128
        a, b = min(upto - n, capacity), min(upto, capacity)
        if st == 0:
            for j in range(held, want):
                blk = free[taken]
                taken += 1
                if not 0 <= blk < num_blocks:
                    blk, st = -1, st | 8
                tables[r, j] = blk
            for i in range(n):
                p = s + i
                blk = tables[r, p // bs]
                pos_out[a + i] = p
                if 0 <= blk < num_blocks:
                    slot_out[a + i] = blk * bs + p % bs
                else:
                    st |= 8
        q_start.append(b)
        lens.append(s + n if (st & ~8) == 0 else s)
        status.append(st)
    return tables, q_start, lens, pos_out, slot_out, taken, status


def rotate(x, positions, inv_freq, rotary_dim, interleaved):
    """Rows [T, H, D] in 64 bits at their positions; inv_freq: the fp32 frequencies."""
    R = rotary_dim
    x = x.double()
    a = positions.double()[:, None, None] * torch.as_tensor(np.asarray(inv_freq, np.float64), device=x.device)
    c, s = a.cos(), a.sin()
    out = x.clone()
    if interleaved:
        u, w = x[..., 0:R:2], x[..., 1:R:2]
        out[..., 0:R:2], out[..., 1:R:2] = u * c - w * s, w * c + u * s
    else:
        u, w = x[..., : R // 2], x[..., R // 2 : R]
        out[..., : R // 2], out[..., R // 2 : R] = u * c - w * s, w * c + u * s
    return out


def cache_rows(cache, layer, table, n, num_blocks):
    """(K, V, valid) of a request's first n tokens in 64 bits: [n, h, d]; keys whose block the table does not name are invalid."""
    bs = cache.block_size
    j = torch.arange(n, device=cache.k.device)
    col = j // bs
    ok = col < table.numel()
    blk = torch.where(ok, table.long()[col.clamp(max=max(table.numel() - 1, 0))] if table.numel() else torch.zeros_like(j), -1)
    ok = ok & (blk >= 0) & (blk < num_blocks)
    blk = blk.clamp(0, num_blocks - 1)
    out = []
    for t, scale in ((cache.k, cache.k_scale), (cache.v, cache.v_scale)):
        x = t[layer] if not getattr(cache, "_views", None) else t
        x = x.transpose(1, 2) if cache.layout == "HND" else x
        x = x[blk, j % bs]
        out.append(x.view(F8).double() * float(np.float32(scale)) if cache.fp8 else x.double())
    return out[0], out[1], ok


def attend(q, cache, layer, q_start, seq_lens, tables, n_kv, scale, out_fill):
    """(out, lse, tol, lse_tol) in 64 bits; rows outside every request keep out_fill (tol 0)."""
    T, hq, d = q.shape
    g = hq // n_kv
    dev = q.device
    out = torch.full((T, hq, d), float(out_fill), dtype=torch.float64, device=dev)
    lse = torch.full((T, hq), float(out_fill), dtype=torch.float64, device=dev)
    tol, ltol = torch.zeros_like(out), torch.zeros_like(lse)
    u_p = U_F16 if cache.fp8 else U_BF16
    for r in range(len(seq_lens)):
        a, b, n = q_start[r], q_start[r + 1], seq_lens[r]
        if not (0 <= a <= b <= T) or n < 0 or a == b:
            continue
        k, v, ok = cache_rows(cache, layer, tables[r], n, cache.num_blocks)
        pos = torch.arange(n - (b - a), n, device=dev)
        see = (torch.arange(n, device=dev)[None] <= pos[:, None]) & ok[None]
        for h in range(hq):
            kh, vh = k[:, h // g], v[:, h // g]
            x = q[a:b, h].double()
            s = (x @ kh.T) * scale
            s = torch.where(see, s, -math.inf)
            m = s.amax(1, keepdim=True) if n else torch.full((b - a, 1), -math.inf, device=dev, dtype=torch.float64)
            m0 = torch.where(torch.isinf(m) & (m < 0), 0.0, m)
            w = torch.where(see, torch.exp(s - m0), 0.0)
            l = w.sum(1, keepdim=True)
            l1 = torch.where(l == 0, 1.0, l)
            vz = torch.where(torch.isfinite(vh), vh, 0.0)  # (values that are not finite count only where they are seen)
            o = (w @ vz) / l1
            if not torch.isfinite(vh).all():
                for j in (~torch.isfinite(vh)).any(1).nonzero().flatten().tolist():
                    bad = torch.where(torch.isfinite(vh[j]), 0.0, vh[j])
                    o += torch.where(see[:, j, None] & ~torch.isfinite(vh[j])[None], w[:, j, None] * bad[None], 0.0)
            out[a:b, h] = o
            lse[a:b, h] = (m + torch.log(l1))[:, 0]
            # fp32 accumulation of d products, scaling and exp2 in fp32: absolute error of a score in natural units
            ds = scale * ((x.abs() @ torch.nan_to_num(kh).abs().T) * see).amax(1, keepdim=True) * (d + 8) * U_F32 + 2.0**-20 if n else 2.0**-20
            av = (w @ vz.abs()) / l1
            t = U_BF16 * o.abs() + (u_p + 3 * ds) * av + 1e-30
            if cache.fp8:  # fp16 weights below 2^-14 have an absolute step of 2^-25
                t = t + 2.0**-25 * (see.double() @ vz.abs()) / l1
            tol[a:b, h] = t
            ltol[a:b, h] = (2 * ds + U_F32 * 4 * torch.nan_to_num(m, neginf=0.0).abs() + 2.0**-20)[:, 0]
    return out, lse, tol, ltol
