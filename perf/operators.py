"""The serving operators around the paged KV cache, with their plain forms in elementary torch operations.

  grow    block tables and slot maps built on the device from request lengths and a list of free blocks
  append  queries and keys of new tokens rotated at their positions, keys and values written into the paged cache
  attend  attention of every request's new tokens over its tokens in the paged cache

With ``own`` false ``run`` computes the plain forms, with ``own`` true it calls the library.
"""
import math
import random

import numpy as np
import torch

own = False

_FP8 = torch.float8_e4m3fn


# ------------------------------------------------------------------------------------------------ cases
def _grow(name, nreq, block_size, start, new, shape_seed, pad=0, short=0):
    return {"name": name, "op": "grow", "nreq": nreq, "block_size": block_size, "start_lo": start[0], "start_hi": start[1], "new_lo": new[0],
            "new_hi": new[1], "pad": pad, "short": short, "shape_seed": shape_seed}  # fmt: skip


def _append(name, tokens, heads, kv_heads, dim, block_size, fp8, start, theta, shape_seed, interleaved=False, rotary=0, head_major=False, pad=0):
    return {"name": name, "op": "append", "tokens": tokens, "heads": heads, "kv_heads": kv_heads, "dim": dim, "block_size": block_size, "fp8": fp8,
            "start": start, "theta": theta, "shape_seed": shape_seed, "interleaved": interleaved, "rotary": rotary, "head_major": head_major,
            "pad": pad}  # fmt: skip


def _attend(name, nreq, heads, kv_heads, dim, block_size, fp8, ctx, shape_seed, chunks=0, chunk=(1, 1), lse=False, head_major=False):
    return {"name": name, "op": "attend", "nreq": nreq, "heads": heads, "kv_heads": kv_heads, "dim": dim, "block_size": block_size, "fp8": fp8,
            "ctx_lo": ctx[0], "ctx_hi": ctx[1], "chunks": chunks, "chunk_lo": chunk[0], "chunk_hi": chunk[1], "lse": lse, "head_major": head_major,
            "shape_seed": shape_seed}  # fmt: skip


def listed():
    return [
        # one decode step of 100 concurrent users: one token each, most of them inside their last block
        _grow("grow decode 100 users", 100, 16, (500, 1300), (1, 1), 1),
        # a step that admits prompts beside running requests, packed arrays padded to a bucket, pool almost exhausted
        _grow("grow mixed 256", 256, 32, (0, 4100), (1, 611), 2, pad=777, short=40),
        # long prompts admitted at once: a million slots
        _grow("grow prompts 1M tokens", 48, 16, (0, 5000), (9000, 33000), 3),
        # the new token of each of 100 users, Llama-3.1-8B heads
        _append("append decode 100 users", 100, 32, 8, 128, 16, False, 1300, 5.0e5, 4),
        # a prompt of 4,097 tokens, 14B-class heads, padded to a bucket
        _append("append prompt 4097", 4097, 40, 8, 128, 32, False, 4096, 1.0e6, 5, pad=255),
        # the same kind of step into an 8-bit cache, far positions
        _append("append prompt 8191 8-bit", 8191, 32, 8, 128, 16, True, 90000, 5.0e5, 6),
        # one user's next token after 50 injected facts
        _attend("decode one request", 1, 32, 8, 128, 16, False, (2033, 2033), 7),
        # 100 users' next tokens over 20 injected facts each
        _attend("decode 100 users", 100, 32, 8, 128, 16, False, (500, 1300), 8),
        # long contexts in an 8-bit cache
        _attend("decode long 8-bit", 16, 32, 8, 128, 16, True, (7000, 32700), 9, lse=True),
        # a question of 61 tokens right after the injected facts
        _attend("question after facts", 1, 32, 8, 128, 16, False, (2073, 2073), 10, chunks=1, chunk=(61, 61), lse=True),
        # a 2,047-token chunk of a prompt behind 100 injected facts of the 14B-class shape
        _attend("chunk 2047 of a prompt", 1, 40, 8, 128, 32, False, (13700, 13700), 11, chunks=1, chunk=(2047, 2047)),
        # continuous batching: chunks of several prompts beside decoding requests, 64-element heads, head-major blocks
        _attend("mixed batch", 24, 16, 4, 64, 16, False, (300, 4100), 12, chunks=5, chunk=(100, 515), head_major=True),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["grow", "append", "attend", "attend"])
    shape_seed = rng.randrange(1 << 30)
    block_size = rng.choice([16, 16, 32, 64])
    if op == "grow":
        nreq = _log(rng, 1, 512)
        hi = _log(rng, 1, min(33000, max(1, 900000 // nreq)))
        start = _log(rng, 1, 30000)
        c = _grow("", nreq, block_size, (rng.randrange(start), start), (rng.randint(0, hi), hi), shape_seed, pad=rng.choice([0, 5, 600]),
                  short=rng.choice([0, 0, 30]))  # fmt: skip
    elif op == "append":
        heads, kv_heads = rng.choice([(32, 8), (40, 8), (16, 4), (8, 8), (28, 4)])
        dim = rng.choice([64, 128, 128, 256])
        tokens = _log(rng, 1, 8191 * 32 * 128 // (max(heads, 32) * max(dim, 128)))
        c = _append("", tokens, heads, kv_heads, dim, block_size, rng.choice([False, True]), rng.randrange(100000), rng.choice([1.0e4, 5.0e5, 1.0e6]),
                    shape_seed, rng.choice([False, True]), rng.choice([0, 0, dim // 2]), rng.choice([False, True]), rng.choice([0, 7, 100]))  # fmt: skip
    else:
        top = max(_cost(x) for x in listed())
        while True:
            heads, kv_heads = rng.choice([(32, 8), (40, 8), (16, 4), (8, 8), (28, 4), (16, 1)])
            dim = rng.choice([64, 128, 128, 128])
            nreq = _log(rng, 1, 128)
            hi = _log(rng, 16, 32000)
            lo = rng.randint(1, hi)
            chunks = rng.choice([0, 0, 1, nreq, rng.randint(0, nreq)])
            chunk_hi = _log(rng, 1, 2048)
            c = _attend("", nreq, heads, kv_heads, dim, block_size, rng.choice([False, True]), (lo, hi), shape_seed, chunks,
                        (rng.randint(1, chunk_hi), chunk_hi), rng.choice([False, True]), rng.choice([False, True]))  # fmt: skip
            q, ctx = _attend_lengths(c)
            padded = nreq * max(q) * max(ctx) * heads
            if _cost(c) <= top and padded <= 1.2e9 and nreq * max(ctx) * kv_heads * dim <= 6.0e8:
                break
    del c["name"]
    return c


def _cost(case):
    w = work(case)
    return max(w["bytes"], w["flops"] / 100)


# ------------------------------------------------------------------------------------------------ lengths (by the case alone)
def _grow_lengths(case):
    r = random.Random(case["shape_seed"])
    start = [r.randint(case["start_lo"], case["start_hi"]) for _ in range(case["nreq"])]
    new = [r.randint(case["new_lo"], case["new_hi"]) for _ in range(case["nreq"])]
    return start, new


def _attend_lengths(case):
    """New tokens and tokens in the cache (the new ones among them) of every request."""
    r = random.Random(case["shape_seed"])
    q = [r.randint(case["chunk_lo"], case["chunk_hi"]) if i < case["chunks"] else 1 for i in range(case["nreq"])]
    ctx = [max(r.randint(case["ctx_lo"], case["ctx_hi"]), n) for n in q]
    order = list(range(case["nreq"]))
    r.shuffle(order)
    return [q[i] for i in order], [ctx[i] for i in order]


def _blocks(n, bs):
    return -(-n // bs)


# ------------------------------------------------------------------------------------------------ inputs
def _generator(seed, case):
    return torch.Generator(device="cuda").manual_seed(int(seed) * 1000003 + case["shape_seed"])


def _cache(case, num_blocks, gen):
    """K and V of one layer of a paged cache, filled as after earlier writes: [blocks, bs, h, d] or [blocks, h, bs, d]."""
    bs, h, d = case["block_size"], case["kv_heads"], case["dim"]
    shape = (1, num_blocks, h, bs, d) if case["head_major"] else (1, num_blocks, bs, h, d)
    out = []
    for scale in (0.02, 0.015):
        x = torch.randn(shape, generator=gen, device="cuda", dtype=torch.bfloat16)
        out.append((x.float() / scale).clamp_(-448, 448).to(_FP8).view(torch.uint8) if case["fp8"] else x)
    return out


def _with_library(case, state):
    """The handles that a user's program keeps: the store (it knows the rotation) and the description of the cache."""
    if own:
        from paper_2607_27090_b200.memstore import ROPE_HALF_SPLIT, ROPE_INTERLEAVED, MemStore, PagedCache

        h, d, bs = case.get("kv_heads", 1), case.get("dim", 64), case["block_size"]
        state["store"] = MemStore(n_layers=1, n_kv_heads=h, head_dim=d, emb_dim=64, max_facts_per_user=1, max_kv_tokens=0, rope_theta=case.get("theta", 1.0e4),
                                  rope_style=ROPE_INTERLEAVED if case.get("interleaved") else ROPE_HALF_SPLIT, rotary_dim=case.get("rotary", 0))  # fmt: skip
        k, v = state.get("k_cache"), state.get("v_cache")
        if k is None:  # building tables takes no more of the cache than its geometry
            k = v = torch.empty((1, 1, bs, h, d), dtype=torch.bfloat16, device="cuda")
        token, head = (d, bs * d) if case.get("head_major") else (h * d, d)
        state["cache"] = PagedCache(k, v, state["num_blocks"] * bs * h * d, bs * h * d, token, head, state["num_blocks"], bs, k_scale=0.02, v_scale=0.015)
    return state


def prepare(case, seed):
    gen = _generator(seed, case)
    dev = {"device": "cuda"}
    bs = case["block_size"]
    if case["op"] == "grow":
        start, new = _grow_lengths(case)
        held = [_blocks(s, bs) for s in start]
        need = [_blocks(s + n, bs) - h for s, n, h in zip(start, new, held)]
        n_free = max(0, sum(need) + 3 - case["short"])
        num_blocks = sum(held) + n_free + 5
        ids = torch.randperm(num_blocks, generator=gen, **dev).to(torch.int32)
        taken = 5
        width = max(h + n for h, n in zip(held, need)) + 1
        rows = torch.tensor([r for r, h in enumerate(held) for _ in range(h)], dtype=torch.int64, **dev)
        cols = torch.tensor([j for h in held for j in range(h)], dtype=torch.int64, **dev)
        tables = torch.full((case["nreq"], width), -1, dtype=torch.int32, **dev)
        tables[rows, cols] = ids[n_free + 5 :]
        state = {"case": case, "start_lens": torch.tensor(start, dtype=torch.int32, **dev), "new_lens": torch.tensor(new, dtype=torch.int32, **dev),
                 "block_tables": tables, "free_blocks": ids[: n_free + 5].contiguous(), "n_taken": torch.tensor([taken], dtype=torch.int32, **dev),
                 "token_capacity": sum(new) + case["pad"], "num_blocks": num_blocks}  # fmt: skip
    elif case["op"] == "append":
        T, P, hq, hk, d = case["tokens"], case["pad"], case["heads"], case["kv_heads"], case["dim"]
        num_blocks = _blocks(T, bs) + 9
        k, v = _cache(case, num_blocks, gen)
        qkv = torch.randn((T + P, (hq + 2 * hk) * d), generator=gen, dtype=torch.bfloat16, **dev)  # one projection's output
        slots = torch.randperm(num_blocks, generator=gen, **dev)[: _blocks(T, bs)].repeat_interleave(bs) * bs + torch.arange(_blocks(T, bs) * bs, **dev) % bs
        none = torch.full((P,), -1, dtype=torch.int64, **dev)
        positions = torch.arange(case["start"], case["start"] + T, dtype=torch.int32, **dev)
        state = {"case": case, "q": qkv[:, : hq * d].unflatten(1, (hq, d)), "k": qkv[:, hq * d : (hq + hk) * d].unflatten(1, (hk, d)),
                 "v": qkv[:, (hq + hk) * d :].unflatten(1, (hk, d)), "positions": torch.cat([positions, none.int()]), "slots": torch.cat([slots[:T], none]),
                 "q_out": torch.zeros((T + P, hq, d), dtype=torch.bfloat16, **dev), "k_cache": k, "v_cache": v, "num_blocks": num_blocks}  # fmt: skip
    else:
        q_lens, ctx = _attend_lengths(case)
        used = [_blocks(c, bs) for c in ctx]
        num_blocks = sum(used) + 3
        k, v = _cache(case, num_blocks, gen)
        ids = torch.randperm(num_blocks, generator=gen, **dev).to(torch.int32)
        tables = torch.zeros((case["nreq"], max(used) + 2), dtype=torch.int32, **dev)
        rows = torch.tensor([r for r, n in enumerate(used) for _ in range(n)], dtype=torch.int64, **dev)
        cols = torch.tensor([j for n in used for j in range(n)], dtype=torch.int64, **dev)
        tables[rows, cols] = ids[: sum(used)]
        q = 1.5 * torch.randn((sum(q_lens), case["heads"], case["dim"]), generator=gen, **dev)
        q_start = torch.tensor([0] + list(np.cumsum(q_lens)), dtype=torch.int32, **dev)
        state = {"case": case, "q": q.to(torch.bfloat16), "q_start": q_start, "seq_lens": torch.tensor(ctx, dtype=torch.int32, **dev), "block_tables": tables,
                 "max_q_len": max(q_lens), "max_seq_len": max(ctx), "k_cache": k, "v_cache": v, "num_blocks": num_blocks}  # fmt: skip
    return _with_library(case, state)


# ------------------------------------------------------------------------------------------------ the passes
def run(state):
    case = state["case"]
    if own:
        return _run_own(case, state)
    return {"grow": _plain_grow, "append": _plain_append, "attend": _plain_attend}[case["op"]](case, state)


def _run_own(case, s):
    if case["op"] == "grow":
        g = s["store"].grow_blocks(s["start_lens"], s["new_lens"], s["block_tables"], s["cache"], s["free_blocks"], s["n_taken"], s["token_capacity"])
        return {"tables": s["block_tables"], "q_start": g.q_start, "seq_lens": g.seq_lens, "positions": g.positions, "slots": g.slots, "n_taken": g.n_taken,
                "status": g.status}  # fmt: skip
    if case["op"] == "append":
        s["store"].append(0, s["q"], s["k"], s["v"], s["positions"], s["slots"], s["cache"], q_out=s["q_out"])
        return _append_outputs(case, s)
    out, lse, _ = s["store"].attend(0, s["q"], s["cache"], s["q_start"], s["seq_lens"], s["block_tables"], max_q_len=s["max_q_len"], want_lse=case["lse"])
    return [out, lse] if case["lse"] else out


def _append_outputs(case, s):
    stored = [x.view(_FP8) if case["fp8"] else x for x in (s["k_cache"], s["v_cache"])]
    return [s["q_out"], *stored]


def _plain_grow(case, s):
    bs, tables = case["block_size"], s["block_tables"]
    nreq, width = tables.shape
    start, new = s["start_lens"].long(), s["new_lens"].long()
    held = (start + bs - 1) // bs
    need = (start + new + bs - 1) // bs - held
    upto = need.cumsum(0)
    taken = s["n_taken"].long()
    served = (need == 0) | (taken + upto <= s["free_blocks"].numel())
    first = taken + upto - need
    col = torch.arange(width, device=tables.device)[None]
    fresh = served[:, None] & (col >= held[:, None]) & (col < (held + need)[:, None])
    at = (first[:, None] + col - held[:, None]).clamp(0, s["free_blocks"].numel() - 1)
    tables.copy_(torch.where(fresh, s["free_blocks"][at], tables))
    ends = new.cumsum(0)
    q_start = torch.cat([ends.new_zeros(1), ends])
    token = torch.arange(s["token_capacity"], device=tables.device)
    r = torch.searchsorted(ends, token, right=True)
    inside = r < nreq
    r = r.clamp(max=nreq - 1)
    pos = start[r] + token - q_start[r]
    good = inside & served[r]
    slot = tables[r, (pos // bs).clamp(max=width - 1)].long() * bs + pos % bs
    status = torch.where(served, 0, 128)
    n_taken = taken + torch.where(served & (need > 0), upto, 0).amax()
    return {"tables": tables, "q_start": q_start.int(), "seq_lens": torch.where(served, start + new, start).int(),
            "positions": torch.where(good, pos, -1).int(), "slots": torch.where(good, slot, -1), "n_taken": n_taken.int(), "status": status.int()}  # fmt: skip


def _plain_rotate(case, x, positions):
    """Rows of [tokens, heads, dim] rotated at their positions; angles in 64 bits of a frequency rounded to 32."""
    R = case["rotary"] or case["dim"]
    f = (case["theta"] ** (-2.0 * torch.arange(R // 2, device=x.device, dtype=torch.float64) / R)).float().double()
    angle = positions.double()[:, None] * f
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    x = x.float()
    y, rest = x[..., :R], x[..., R:]
    if case["interleaved"]:
        a, b = y[..., 0::2], y[..., 1::2]
        y = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    else:
        a, b = y[..., : R // 2], y[..., R // 2 :]
        y = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    return torch.cat([y, rest], -1).to(torch.bfloat16)


def _plain_append(case, s):
    T, bs = case["tokens"], case["block_size"]  # the padding is behind the last token
    positions, slots = s["positions"][:T], s["slots"][:T]
    s["q_out"][:T] = _plain_rotate(case, s["q"][:T], positions)
    rows = {"k_cache": _plain_rotate(case, s["k"][:T], positions), "v_cache": s["v"][:T]}
    blk, off = slots // bs, slots % bs
    stored = {n: (x.float() / sc).clamp(-448, 448).to(_FP8).view(torch.uint8) if case["fp8"] else x for (n, x), sc in zip(rows.items(), (0.02, 0.015))}
    k, v = (s[n][0].transpose(1, 2) if case["head_major"] else s[n][0] for n in ("k_cache", "v_cache"))
    k[blk, off] = stored["k_cache"]
    v[blk, off] = stored["v_cache"]
    return _append_outputs(case, s)


def _plain_rows(case, s, cache, scale, index, live):
    """[nreq, h, keys, d] in 32 bits: the rows of the cache that the tables name."""
    x = cache[0].transpose(1, 2) if case["head_major"] else cache[0]
    x = x[index // case["block_size"], index % case["block_size"]]
    x = x.view(_FP8).float() * scale if case["fp8"] else x.float()
    return torch.where(live[:, :, None, None], x, 0.0).transpose(1, 2).contiguous()


def _plain_attend(case, s):
    n, hq, hk, d, bs = case["nreq"], case["heads"], case["kv_heads"], case["dim"], case["block_size"]
    g, qmax, kmax = hq // hk, s["max_q_len"], s["max_seq_len"]
    dev = s["q"].device
    q_start, lens = s["q_start"].long(), s["seq_lens"].long()
    q_lens = q_start[1:] - q_start[:-1]
    key = torch.arange(kmax, device=dev)
    live = key[None] < lens[:, None]
    index = s["block_tables"].long()[:, key // bs] * bs + key % bs
    k = _plain_rows(case, s, s["k_cache"], 0.02, index, live)
    v = _plain_rows(case, s, s["v_cache"], 0.015, index, live)
    i = torch.arange(qmax, device=dev)
    row = (q_start[:-1, None] + i).clamp(max=s["q"].shape[0] - 1)  # padded to the longest chunk
    q = s["q"][row].float().unflatten(2, (hk, g)).permute(0, 2, 3, 1, 4).reshape(n, hk, g * qmax, d)
    scores = torch.matmul(q, k.transpose(2, 3)).view(n, hk, g, qmax, kmax).mul_(1.0 / math.sqrt(d))
    pos = (lens - q_lens)[:, None] + i
    scores.masked_fill_((key > pos[..., None])[:, None, None], -math.inf)
    m = scores.amax(-1, keepdim=True)
    p = scores.sub_(m).exp_()
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p.view(n, hk, g * qmax, kmax), v).view(n, hk, g, qmax, d) / total
    has = i[None] < q_lens[:, None]
    out = out.permute(0, 3, 1, 2, 4).reshape(n, qmax, hq, d)[has].to(torch.bfloat16)
    if not case["lse"]:
        return out
    return [out, (m + total.log())[..., 0].permute(0, 3, 1, 2).reshape(n, qmax, hq)[has]]


# ------------------------------------------------------------------------------------------------ what a pass cannot do without
def work(case):
    if case["op"] == "grow":
        start, new = _grow_lengths(case)
        bs, T = case["block_size"], sum(new) + case["pad"]
        fresh = sum(_blocks(s + n, bs) - _blocks(s, bs) for s, n in zip(start, new))
        return {"bytes": 12 * T + 8 * fresh + 20 * case["nreq"] + 12, "flops": T}
    if case["op"] == "append":
        T, hq, hk, d = case["tokens"], case["heads"], case["kv_heads"], case["dim"]
        cached = 2 * hk * d * (1 if case["fp8"] else 2)
        return {"bytes": T * ((2 * hq + 2 * hk) * d * 2 + cached + 12), "flops": T * (hq + hk) * 3 * (case["rotary"] or d)}
    q, ctx = _attend_lengths(case)
    hq, hk, d = case["heads"], case["kv_heads"], case["dim"]
    pairs = sum(n * (c - n) + n * (n + 1) // 2 for n, c in zip(q, ctx))
    kv = sum(ctx) * 2 * hk * d * (1 if case["fp8"] else 2)
    return {"bytes": kv + sum(q) * hq * (4 * d + (4 if case["lse"] else 0)) + 4 * sum(_blocks(c, case["block_size"]) for c in ctx), "flops": 4 * pairs * hq * d}


# ------------------------------------------------------------------------------------------------ the definitions in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    return {"grow": _exact_grow, "append": _exact_append, "attend": _exact_attend}[case["op"]](case, s)


def _exact_grow(case, s):
    """An allocator that serves request after request."""
    bs, start, new = case["block_size"], s["start_lens"].tolist(), s["new_lens"].tolist()
    tables, free = s["block_tables"].cpu().numpy().copy(), s["free_blocks"].cpu().numpy()
    taken, asked, q_start, lens, status = s["n_taken"].item(), s["n_taken"].item(), [0], [], []
    positions, slots = np.full(s["token_capacity"], -1, np.int32), np.full(s["token_capacity"], -1, np.int64)
    for r, (a, n) in enumerate(zip(start, new)):
        first, last = _blocks(a, bs), _blocks(a + n, bs)
        asked += last - first
        fits = last == first or asked <= len(free)
        if fits and last > first:
            tables[r, first:last] = free[taken : taken + last - first]
            taken += last - first
        if fits:
            pos = np.arange(a, a + n)
            positions[q_start[-1] : q_start[-1] + n] = pos
            slots[q_start[-1] : q_start[-1] + n] = tables[r, pos // bs].astype(np.int64) * bs + pos % bs
        q_start.append(q_start[-1] + n)
        lens.append(a + n if fits else a)
        status.append(0 if fits else 128)
    i32 = lambda x: torch.tensor(np.asarray(x, np.int32))  # noqa: E731
    return {"tables": i32(tables), "q_start": i32(q_start), "seq_lens": i32(lens), "positions": i32(positions), "slots": torch.tensor(slots),
            "n_taken": i32([taken]), "status": i32(status)}  # fmt: skip


def _exact_append(case, s):
    T, bs, d = case["tokens"], case["block_size"], case["dim"]
    R = case["rotary"] or d
    freq = torch.tensor([float(np.float32(case["theta"] ** (-2.0 * i / R))) for i in range(R // 2)], dtype=torch.float64, device="cuda")
    turn = torch.polar(torch.ones(T, R // 2, dtype=torch.float64, device="cuda"), s["positions"][:T].double()[:, None] * freq)[:, None]

    def rotated(x):
        x = x[:T].double()
        pair = x[..., :R].unflatten(-1, (R // 2, 2)) if case["interleaved"] else x[..., :R].unflatten(-1, (2, R // 2)).transpose(-1, -2)
        z = torch.view_as_real(torch.view_as_complex(pair.contiguous()) * turn)
        return torch.cat([z.flatten(-2) if case["interleaved"] else z.transpose(-1, -2).flatten(-2), x[..., R:]], -1)

    q_out = s["q_out"].double()
    q_out[:T] = rotated(s["q"])
    out = [q_out]
    for name, rows, scale in (("k_cache", rotated(s["k"]), 0.02), ("v_cache", s["v"][:T].double(), 0.015)):
        cache = s[name].view(_FP8).float().double() if case["fp8"] else s[name].double()
        if case["fp8"]:
            rows = (rows / float(np.float32(scale))).clamp(-448, 448)
        for h in range(case["kv_heads"]):
            plane = cache[0, :, h] if case["head_major"] else cache[0, :, :, h]
            plane[s["slots"][:T] // bs, s["slots"][:T] % bs] = rows[:, h]
        out.append(cache)
    return out


def _exact_attend(case, s):
    """Request by request and head by head."""
    hq, hk, d, bs = case["heads"], case["kv_heads"], case["dim"], case["block_size"]
    g = hq // hk
    q_lens, ctx = _attend_lengths(case)
    if sum(n * c for n, c in zip(q_lens, ctx)) * hq * d > 5e11 or case["nreq"] * hk > 2000:
        return None
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(s["q"].shape[:2], dtype=torch.float64, device="cuda")
    scales = [float(np.float32(0.02)), float(np.float32(0.015))] if case["fp8"] else [1.0, 1.0]
    at = 0
    for r, (n, c) in enumerate(zip(q_lens, ctx)):
        table = s["block_tables"][r, : _blocks(c, bs)].long()
        k, v = ((x[0].transpose(1, 2) if case["head_major"] else x[0])[table].flatten(0, 1)[:c] for x in (s["k_cache"], s["v_cache"]))
        if case["fp8"]:
            k, v = k.view(_FP8).float(), v.view(_FP8).float()
        later = torch.arange(c, device="cuda")[None] > torch.arange(c - n, c, device="cuda")[:, None]
        for h in range(hk):
            kh, vh = k[:, h].double() * scales[0], v[:, h].double() * scales[1]
            for j in range(h * g, (h + 1) * g):
                t = (s["q"][at : at + n, j].double() @ kh.T / math.sqrt(d)).masked_fill(later, -math.inf)
                lse[at : at + n, j] = torch.logsumexp(t, 1)
                out[at : at + n, j] = torch.softmax(t, 1) @ vh
        at += n
    return [out, lse] if case["lse"] else out
