"""GPU tests of selected blocks (memstore_summarize_blocks, memstore_select_blocks, memstore_attend_blocks) against plain 64-bit
implementations, with the cases where such kernels go wrong."""
import math
import random

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    import drafts_ref as dr
    import serving_ref as ref
    from paper_2607_27090_b200.memstore import MemStore, MemStoreError, PagedCache
    from test_gpu_drafts import compare
    from test_gpu_serving import fill_cache, i32, paged, store

DEV = "cuda"
SHAPES = [
    # d, heads, kv heads, block size, 8-bit, layout
    (64, 4, 2, 16, False, "NHD"), (128, 32, 8, 16, False, "NHD"), (128, 40, 8, 32, False, "HND"), (128, 8, 8, 16, True, "NHD"), (64, 14, 2, 64, True, "HND"),
    (16, 2, 1, 16, False, "NHD"), (32, 3, 1, 8, False, "NHD"), (256, 8, 2, 16, False, "NHD"), (256, 4, 4, 16, True, "NHD"), (32, 4, 4, 16, True, "HND"),
    (16, 33, 3, 5, True, "NHD"), (128, 16, 1, 24, False, "NHD"), (64, 20, 1, 1, False, "HND"), (128, 7, 1, 128, True, "NHD")]  # fmt: skip


def token_major(cache, layer):
    x = cache.k[layer]
    return x.transpose(1, 2) if cache.layout == "HND" else x


# ------------------------------------------------------------------------------------------------ summaries
def check_summaries(ms, cache, lens, tables, new=None, layer=0, n_tokens=None):
    """All summaries of a layer after a call, bit for bit (zeros of either sign are equal), NaN for NaN."""
    hk, d, bs, nb = ms.n_kv_heads, ms.head_dim, cache.block_size, cache.num_blocks
    got = torch.full((nb, hk, 2, d), 7.0, dtype=torch.bfloat16, device=DEV)
    want = got.clone()
    x = token_major(cache, layer)
    x = x.view(ref.F8).float() if cache.fp8 else x.float()
    for r, n in enumerate(lens):
        m = n if new is None else new[r]
        if n < 0 or m <= 0:
            continue
        for b in range(max(0, n - m) // bs, min(-(-n // bs), tables.shape[1])):
            blk = int(tables[r, b])
            if 0 <= blk < nb:
                keys = x[blk, : min(bs, n - b * bs)]
                want[blk, :, 0], want[blk, :, 1] = keys.amin(0).to(torch.bfloat16), keys.amax(0).to(torch.bfloat16)  # (NaN goes through)
    q_start = None if new is None else i32([0] + [int(v) for v in np.cumsum(new)])
    kw = {} if n_tokens is None else {"n_tokens": n_tokens}
    ms.summarize_blocks(layer, cache, got, i32(lens), tables, q_start=q_start, **kw)
    torch.cuda.synchronize()
    nan = torch.isnan(want)
    assert torch.equal(torch.isnan(got), nan)
    assert torch.equal(got[~nan], want[~nan])
    return got


@pytest.mark.parametrize("d,hq,hk,bs,fp8,layout", SHAPES)
def test_summaries_against_the_definition(d, hq, hk, bs, fp8, layout):
    rng = random.Random(d + bs)
    ms = store(hk, d, 2)
    for nreq, hi in ((1, 1), (1, 700), (5, 90), (150, 60)):
        lens = [rng.choice([hi, 0, rng.randint(0, hi)]) if nreq > 1 else hi for _ in range(nreq)]
        new = [rng.choice([0, 1, n, n + 3, rng.randint(0, n)]) for n in lens]
        tables, nb = paged(rng, lens, bs)
        cache, _ = fill_cache(2, nb, bs, hk, d, fp8, layout, nreq)
        check_summaries(ms, cache, lens, tables, layer=1)
        check_summaries(ms, cache, lens, tables, new, layer=1, n_tokens=sum(new))
        check_summaries(ms, cache, lens, tables, new)
    ms.close()


@pytest.mark.parametrize("fp8", [False, True])
def test_summaries_of_holes_short_tables_and_values_that_are_not_finite(fp8):
    rng = random.Random(1)
    bs, lens = 16, [700, 500, 300, -5, 16, 17]
    tables, nb = paged(rng, lens, bs, width_extra=0)
    tables[0, 3], tables[1, 31], tables[1, 0] = nb, nb + 5, -(2**31)
    cache, _ = fill_cache(1, nb, bs, 3, 64, fp8, "NHD", 6)
    for e, x in ((0, math.nan), (9, math.inf), (33, -math.inf)):
        cache.k[0, int(tables[2, 4]), 7, 1, e] = 0x7F if fp8 else x
    cache.k[0, int(tables[5, 1]), 1:] = 0x7F if fp8 else math.nan  # behind the last key
    ms = store(3, 64)
    got = check_summaries(ms, cache, lens, tables)
    assert torch.isfinite(got[int(tables[5, 1])]).all() and torch.isnan(got[int(tables[2, 4]), 1, :, 0]).all()
    check_summaries(ms, cache, lens, tables[:, :20].contiguous())
    check_summaries(ms, cache, lens, tables, [700, 1, 17, 4, 0, 2])
    # ranges that are none
    keep = torch.full((nb, 3, 2, 64), 7.0, dtype=torch.bfloat16, device=DEV)
    s = keep.clone()
    ms.summarize_blocks(0, cache, s, i32([300]), tables[2:3], q_start=i32([5, 3]))
    ms.summarize_blocks(0, cache, s, i32([300]), tables[2:3], q_start=i32([-1, 3]))
    ms.summarize_blocks(0, cache, s, i32([300]), tables[2:3], q_start=i32([0, 9]), n_tokens=8)
    assert torch.equal(s, keep)
    assert ms.allocate_summaries(cache).shape == (1, nb, 3, 2, 64) and not ms.allocate_summaries(cache).any()
    with pytest.raises(ValueError):
        ms.summarize_blocks(0, cache, s[:-1], i32([300]), tables[2:3])
    with pytest.raises(TypeError):
        ms.summarize_blocks(0, cache, s.float(), i32([300]), tables[2:3])
    with pytest.raises(MemStoreError):
        ms.summarize_blocks(1, cache, s, i32([300]), tables[2:3])
    with pytest.raises(ValueError):
        ms.summarize_blocks(0, cache, s, i32([300]), tables[0])
    ms.close()


# ------------------------------------------------------------------------------------------------ selection
def run_select(ms, q, box, q_start, lens, tables, nb, bs, k, first, last, skip=(), want_scores=True):
    T, hq, d = q.shape
    hk = ms.n_kv_heads
    g, width = hq // hk, tables.shape[1]
    cache = PagedCache(torch.empty((1, 1, 1, hk, d), dtype=torch.bfloat16, device=DEV), torch.empty((1, 1, 1, hk, d), dtype=torch.bfloat16, device=DEV),
                       nb * bs * hk * d, bs * hk * d, hk * d, d, nb, bs)  # fmt: skip
    got = i32(np.full((T, hk, k), -3))
    sc = torch.full((T, hk, width), 9.0, device=DEV) if want_scores else None
    ms.select_blocks(q, cache, box, i32(q_start), i32(lens), tables, k, n_first=first, n_last=last, out_blocks=got, out_scores=sc)
    torch.cuda.synchronize()
    blocks, scores = got.cpu().numpy(), sc.cpu().numpy() if want_scores else None
    seen = np.zeros(T, bool)
    for r, n in enumerate(lens):
        a, b = q_start[r], q_start[r + 1]
        if r in skip:
            continue
        t_np = tables[r].cpu().numpy()
        for t in range(a, b):
            seen[t] = True
            pos = n - (b - a) + t - a
            every = pos // bs + 1 if pos >= 0 else 0
            m = min(every, width)
            named = (t_np[:m] >= 0) & (t_np[:m] < nb)
            safe = torch.as_tensor(np.where(named, t_np[:m], 0), device=DEV).long()
            for h in range(hk):
                want = dr.scores(q[t, h * g : (h + 1) * g], box[safe, h]) if m else torch.zeros(0, device=DEV)
                want32 = np.where(named, want.float().cpu().numpy(), -np.inf)
                if want_scores:
                    x = scores[t, h, :m]
                    assert np.array_equal(np.isnan(x), np.isnan(want32))
                    fin = np.isfinite(want32)
                    assert np.array_equal(x[~fin & ~np.isnan(x)], want32[~fin & ~np.isnan(x)])
                    # fp32 sums of exact products: head_dim / 8 matrix products one after another add 17 numbers each, cut off at 2^-23 of the largest
                    # or better; the three parts of P and N, the sum of three columns and the last rounding are off by 2^-24 four times
                    most = (d // 8 * 17 + 2) * 2.0**-23 * dr.magnitudes(q[t, h * g : (h + 1) * g], box[safe, h]).cpu().numpy() + 2.0**-140
                    assert (np.abs(x[fin] - want.cpu().numpy()[fin]) <= most[fin]).all()
                    assert (scores[t, h, m:] == 9.0).all()
                chosen = dr.choose(want32, named, k, first, last, every)
                assert blocks[t, h].tolist() == chosen + [-1] * (k - len(chosen)), (r, t, h)
    assert (blocks[~seen] == -3).all()
    return got


def boxes(gen, nb, hk, d, spread=1.0):
    mid = torch.randn((nb, hk, d), generator=gen, device=DEV)
    off = spread * torch.randn((nb, hk, d), generator=gen, device=DEV).abs()
    return torch.stack([mid - off, mid + off], 2).to(torch.bfloat16)


@pytest.mark.parametrize("d,hq,hk,bs,fp8,layout", SHAPES)
def test_selection_against_the_definition(d, hq, hk, bs, fp8, layout):
    rng = random.Random(d * 3 + bs)
    ms = store(hk, d)
    for nreq, n_hi, len_hi in ((1, 1, 1), (1, 1, 900), (4, 3, 400), (40, 1, 90)):
        new = [rng.randint(0 if nreq > 1 else 1, n_hi) for _ in range(nreq)]
        lens = [rng.choice([len_hi, max(0, n - 1), n, rng.randint(n, max(n, len_hi))]) for n in new]
        q_start = [0] + [int(x) for x in np.cumsum(new)]
        tables, nb = paged(rng, lens, bs)
        gen = torch.Generator(device=DEV).manual_seed(nreq)
        box = boxes(gen, nb, hk, d)
        q = torch.randn((q_start[-1] + 2, hq, d), generator=gen, device=DEV).to(torch.bfloat16)
        for k, first, last in ((1, 0, 0), (1, 0, 1), (7, 1, 2), (64, 2, 8), (3, 3, 0), (5, 0, 5)):
            run_select(ms, q, box, q_start, lens, tables, nb, bs, k, first, last, want_scores=rng.choice([True, False]))
    ms.close()


@pytest.mark.parametrize("n_blocks,k", [(255, 64), (256, 64), (257, 64), (2047, 1), (2049, 500), (8190, 64), (8193, 4000), (30000, 256), (49000, 9)])
def test_selection_over_long_contexts(n_blocks, k):
    """Few tokens over many blocks: a cluster of CTAs shares a token."""
    rng = random.Random(n_blocks)
    hk, hq, d, bs = 2, 6, 64, 4
    ms = store(hk, d)
    for nreq in (1, 3):
        lens = [n_blocks * bs - rng.randint(0, 3)] + [rng.randint(1, n_blocks * bs) for _ in range(nreq - 1)]
        tables, nb = paged(rng, lens, bs, width_extra=0)
        gen = torch.Generator(device=DEV).manual_seed(n_blocks)
        q = torch.randn((nreq, hq, d), generator=gen, device=DEV).to(torch.bfloat16)
        run_select(ms, q, boxes(gen, nb, hk, d), list(range(nreq + 1)), lens, tables, nb, bs, k, 1, min(4, k - 1))
    ms.close()


def test_selection_ties_infinities_and_nan():
    """Equal scores go to the lower block, zeros of either sign are equal, NaN ranks as plus infinity; also scores that agree in all but their last bits."""
    rng = random.Random(5)
    hk, hq, d, bs, n = 1, 2, 32, 8, 700
    lens = [n * bs]
    tables, nb = paged(rng, lens, bs)
    gen = torch.Generator(device=DEV).manual_seed(3)
    ms = store(hk, d)
    q = torch.randn((1, hq, d), generator=gen, device=DEV).to(torch.bfloat16)
    one = boxes(gen, 1, hk, d)
    row = tables[0, :n].long()
    for kind in range(6):
        box = one.expand(nb, hk, 2, d).clone()
        x = q.clone()
        if kind == 1:  # some are better, many equal
            box[row[100:300:7], 0, 1, 3] += 4.0
            x[..., 3] = 1.0
        elif kind == 2:
            box[row[50], 0, 1, 0], box[row[60], 0, 0, 1], box[row[70], 0, :, 2] = math.inf, -math.inf, math.nan
        elif kind == 3:  # zeros
            box.zero_()
            box[row[::2]] = -0.0
        elif kind == 4:  # all minus infinity
            x[:] = 1.0
            box[:, :, 0], box[:, :, 1] = 0.0, -math.inf
        elif kind == 5:  # steps of the last bit
            x.zero_()
            x[0, 0, 0], x[0, 0, 1] = 1.0, 2.0**-16
            box.zero_()
            box[row, 0, 1, 0] = 128.0
            box[row, 0, 1, 1] = (torch.arange(n, device=DEV) * 37 % 128).to(torch.bfloat16)
        for k in (1, 2, 3, 29, 300, 699, 700, 701):
            run_select(ms, x, box, [0, 1], lens, tables, nb, bs, k, min(1, k - 1), 0)
    ms.close()


def test_selection_holes_short_tables_and_refusals():
    rng = random.Random(6)
    bs, lens, q_start = 16, [700, 500, 300, 2, 90], [0, 1, 4, 4, 9, 10]
    hk, hq, d = 2, 8, 64
    tables, nb = paged(rng, lens, bs, width_extra=0)
    tables[0, 3], tables[0, 40], tables[1, 31], tables[1, 0], tables[1, 5] = -1, nb, nb + 5, -(2**31), 2**31 - 1
    gen = torch.Generator(device=DEV).manual_seed(3)
    ms = store(hk, d)
    box = boxes(gen, nb, hk, d)
    q = torch.randn((12, 12 * d), generator=gen, device=DEV).to(torch.bfloat16)[:, : hq * d].unflatten(1, (hq, d))  # a slice of a fused projection
    for k, first, last in ((5, 1, 2), (50, 3, 3), (2, 0, 2)):
        run_select(ms, q, box, q_start, lens, tables, nb, bs, k, first, last)
        run_select(ms, q, box, q_start, lens, tables[:, :9].contiguous(), nb, bs, k, first, last)
    # requests that are none: ranges outside the rows, a negative length
    run_select(ms, q, box, [0, 1, 4, 4, 9, 13], lens, tables, nb, bs, 5, 1, 1, skip=(4,))
    run_select(ms, q, box, q_start, [700, -1, 300, 2, 90], tables, nb, bs, 5, 1, 1, skip=(1,))
    cache = PagedCache.allocate(1, nb, bs, hk, d, DEV)
    args = (cache, box, i32(q_start), i32(lens), tables)
    for k, first, last in ((0, 0, 0), (-1, 0, 0), (3, 2, 2), (3, -1, 2), (3, 1, -1)):
        with pytest.raises(MemStoreError):
            ms.select_blocks(q, *args, k, n_first=first, n_last=last)
    with pytest.raises(MemStoreError):
        ms.select_blocks(q[:, :7], *args, 4)
    with pytest.raises(MemStoreError):
        ms.select_blocks(q, cache, box, i32(q_start), i32(lens), i32(np.zeros((5, 49153))), 4)
    with pytest.raises(ValueError):
        ms.select_blocks(q, cache, box[1:], i32(q_start), i32(lens), tables, 4)
    with pytest.raises(TypeError):
        ms.select_blocks(q.float(), *args, 4)
    with pytest.raises(ValueError):
        ms.select_blocks(q, *args, 4, out_blocks=i32(np.zeros((12, hk, 5))))
    with pytest.raises(ValueError):
        ms.select_blocks(q, *args, 4, out_scores=torch.zeros((12, hk, 5), device=DEV))
    got, none = ms.select_blocks(q[:0], cache, box, i32([0, 0]), i32([5]), tables[:1], 4)
    assert got.shape == (0, hk, 4) and none is None
    got, _ = ms.select_blocks(q, cache, box, i32([0, 12]), i32([90]), i32(np.zeros((1, 0))), 4)  # a table without entries
    assert (got == -1).all()
    ms.close()


# ------------------------------------------------------------------------------------------------ attention
def check_sparse(ms, cache, q, q_start, lens, tables, lists, layer=0, scale=0.0, want_status=None, **kw):
    T, hq, d = q.shape
    bs = cache.block_size
    out = torch.full((T, hq, d), 9.0, dtype=torch.bfloat16, device=DEV)
    lse = torch.full((T, hq), 9.0, device=DEV)
    status = i32([-5] * len(lens))
    ms.attend_blocks(layer, q, i32(lists), cache, i32(q_start), i32(lens), tables, scale=scale, out=out, out_lse=lse, out_status=status, **kw)
    torch.cuda.synchronize()

    def see(r, head, n):
        a, b = q_start[r], q_start[r + 1]
        rows = np.zeros((b - a, n), bool)
        for i in range(b - a):
            pos = n - (b - a) + i
            for x in lists[a + i, head, : -(-n // bs)]:
                if 0 <= x < tables.shape[1] and x * bs < n:
                    rows[i, x * bs : min(n, x * bs + bs, max(0, pos + 1))] = True
        return rows

    compare(out, lse, dr.attend_seen(q, cache, layer, q_start, lens, tables, ms.n_kv_heads, scale or 1.0 / math.sqrt(d), 9.0, see))
    assert status.tolist() == (want_status or [0] * len(lens))
    return out, lse


def lists_of(rng, q_start, lens, T, hk, bs, k, kind):
    """Blocks in rising order and -1 behind them, any order, none, or numbers that may be anything."""
    out = np.full((T, hk, k), -1, np.int64)
    for r, n in enumerate(lens):
        a, b = q_start[r], q_start[r + 1]
        for t in range(a, b):
            have = max(0, n - (b - a) + t - a) // bs + 1
            for h in range(hk):
                ids = rng.sample(range(have), min(k, have))
                if kind == "sorted":
                    ids.sort()
                elif kind == "none":
                    ids = []
                elif kind == "wild":
                    ids = [rng.choice([x, x, x, -1, -(2**31), 2**31 - 1, have + 5, have]) for x in ids]
                    ids = [x if x not in ids[:i] else -1 for i, x in enumerate(ids)]  # (each once)
                out[t, h, : len(ids)] = ids
    return out


@pytest.mark.parametrize("d,hq,hk,bs,fp8,layout", SHAPES)
@pytest.mark.parametrize("nreq,n_hi,len_hi,k,kind", [(1, 1, 1, 1, "sorted"), (5, 1, 700, 9, "sorted"), (4, 6, 333, 20, "wild"), (3, 40, 900, 3, "any"), (3, 2, 200, 70, "none"),
                                                     (2, 1, 5000, 64, "any")])  # fmt: skip
def test_sparse_attention_against_the_definition(d, hq, hk, bs, fp8, layout, nreq, n_hi, len_hi, k, kind):
    rng = random.Random(d * 7 + hq + nreq + k)
    new = [rng.choice([n_hi, 1, rng.randint(0, n_hi)]) for _ in range(nreq)]
    lens = [max(rng.randint(0, len_hi), rng.choice([n, n - 1 if n else 0])) for n in new]
    q_start = [0] + [int(x) for x in np.cumsum(new)]
    tables, nb = paged(rng, lens, bs)
    cache, gen = fill_cache(2, nb, bs, hk, d, fp8, layout, nreq)
    ms = store(hk, d, 2)
    x = (2.0 * torch.randn((q_start[-1] + 3, hq, d), generator=gen, device=DEV)).to(torch.bfloat16)  # rows behind the last request too
    lists = lists_of(rng, q_start, lens, q_start[-1] + 3, hk, bs, k, kind)
    out, lse = check_sparse(ms, cache, x, q_start, lens, tables, lists, layer=1)
    if kind == "none":
        assert (out[: q_start[-1]] == 0).all() and (lse[: q_start[-1]] == -math.inf).all()
    check_sparse(ms, cache, x, q_start, lens, tables, lists, layer=1, scale=0.9)
    ms.close()


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("bs,len_,k", [(16, 1, 4), (16, 16, 1), (16, 17, 2), (64, 64, 1), (64, 65, 2), (64, 129, 1), (48, 4000, 30), (128, 20001, 5), (16, 20001, 400), (1, 300, 130)])
def test_sparse_attention_lengths_around_tile_and_block_borders(fp8, bs, len_, k):
    rng = random.Random(len_ + bs)
    tables, nb = paged(rng, [len_], bs)
    cache, gen = fill_cache(1, nb, bs, 2, 128, fp8, "NHD", len_)
    for t in (cache.k, cache.v):  # behind the last token
        if len_ % bs:
            t[0, int(tables[0, len_ // bs]), len_ % bs :] = 0x7F if fp8 else math.nan
    ms = store(2, 128)
    for n in (1, 3):
        q = torch.randn((n, 8, 128), generator=gen, device=DEV).to(torch.bfloat16)
        lists = lists_of(rng, [0, n], [len_], n, 2, bs, k, "sorted")
        last = (len_ - 1) // bs
        for t in range(n):  # the block of the row itself among them, where it has one
            if len_ - n + t >= 0 and (len_ - n + t) // bs not in lists[t, 0]:
                lists[t, 0, 0] = (len_ - n + t) // bs
        assert last >= 0
        check_sparse(ms, cache, q, [0, n], [len_], tables, lists)
    ms.close()


@pytest.mark.parametrize("fp8", [False, True])
def test_sparse_attention_many_requests_equals_its_rows_alone(fp8):
    """200 ragged requests (more than a warp's line holds): a row's result is near the definition whatever else is in the call, and repeats to the bit."""
    rng = random.Random(3)
    new = [rng.choice([1, 1, 1, 0, 2]) for _ in range(200)]
    lens = [n + rng.choice([0, rng.randint(0, 50), rng.randint(0, 1500)]) for n in new]
    q_start = [0] + [int(x) for x in np.cumsum(new)]
    tables, nb = paged(rng, lens, 16)
    cache, gen = fill_cache(1, nb, 16, 2, 64, fp8, "NHD", 1)
    ms = store(2, 64)
    x = torch.randn((q_start[-1], 6, 64), generator=gen, device=DEV).to(torch.bfloat16)
    lists = lists_of(rng, q_start, lens, q_start[-1], 2, 16, 24, "sorted")
    a, la = check_sparse(ms, cache, x, q_start, lens, tables, lists)
    b, lb = check_sparse(ms, cache, x, q_start, lens, tables, lists)
    assert torch.equal(a, b) and torch.equal(la, lb)
    ms.close()


def test_sparse_attention_over_all_blocks_is_the_dense_one():
    rng = random.Random(7)
    lens = [900, 33, 2000]
    tables, nb = paged(rng, lens, 16)
    for fp8 in (False, True):
        cache, gen = fill_cache(1, nb, 16, 2, 128, fp8, "NHD", 3)
        ms = store(2, 128)
        q = torch.randn((3, 8, 128), generator=gen, device=DEV).to(torch.bfloat16)
        lists = np.tile(np.arange(126), (3, 2, 1))
        out, lse = check_sparse(ms, cache, q, [0, 1, 2, 3], lens, tables, lists)
        dense, dl, _ = ms.attend(0, q, cache, i32([0, 1, 2, 3]), i32(lens), tables, want_lse=True)
        assert torch.equal(out, dense) and torch.equal(lse, dl)  # the same tiles in the same order
        ms.close()


def test_sparse_attention_values_that_are_not_finite_and_refusals():
    rng = random.Random(9)
    lens, q_start = [700, 500, 300], [0, 1, 3, 4]
    tables, nb = paged(rng, lens, 16, width_extra=0)
    tables[0, 3], tables[1, 31], tables[1, 0] = -1, nb, -(2**31)
    cache, gen = fill_cache(1, nb, 16, 2, 128, False, "NHD", 6)
    ms = store(2, 128)
    q = torch.randn((4, 8, 128), generator=gen, device=DEV).to(torch.bfloat16)
    lists = lists_of(rng, q_start, lens, 4, 2, 16, 12, "sorted")
    lists[3] = np.arange(12)
    lists[0, :, :5] = [0, 1, 2, 3, 4]
    check_sparse(ms, cache, q, q_start, lens, tables, lists, want_status=[8, 8, 0])
    check_sparse(ms, cache, q, q_start, lens, tables[:, :30].contiguous(), lists, want_status=[12, 12, 0])
    # request 2 reads blocks 0 .. 11 only: what the others hold does not reach it, what these hold does
    for j in range(12, 19):
        cache.k[0, int(tables[2, j])], cache.v[0, int(tables[2, j])] = math.nan, math.inf
    out, _ = check_sparse(ms, cache, q, q_start, lens, tables, lists, want_status=[8, 8, 0])
    assert torch.isfinite(out[3]).all()
    cache.v[0, int(tables[2, 5]), 2, 0, 7] = math.inf
    out, _ = check_sparse(ms, cache, q, q_start, lens, tables, lists, want_status=[8, 8, 0])
    assert (out[3, :4, 7] == math.inf).all() and torch.isfinite(out[3, 4:]).all()
    good = dict(cache=cache, q_start=i32(q_start), seq_lens=i32(lens), block_tables=tables)
    for bad, err in ((i32(lists).long(), TypeError), (i32(lists)[:3], ValueError), (i32(lists)[:, :1].contiguous(), ValueError), (i32(lists)[0], ValueError),
                     (i32(lists)[:, :, :0].contiguous(), MemStoreError)):  # fmt: skip
        with pytest.raises(err):
            ms.attend_blocks(0, q, bad, **good)
    with pytest.raises(MemStoreError):
        ms.attend_blocks(1, q, i32(lists), **good)
    with pytest.raises(MemStoreError):
        ms.attend_blocks(0, q, i32(lists), scale=-1.0, **good)
    with pytest.raises(MemStoreError):
        ms.attend_blocks(0, q[:, :7], i32(lists), **good)
    # a block listed twice counts twice, and a list has no more entries than the request has blocks
    twice = np.full((4, 2, 12), -1)
    twice[3] = 4
    one = twice.copy()
    one[3, :, 1:] = -1
    a, la, _ = ms.attend_blocks(0, q, i32(twice), want_lse=True, **good)
    b, lb, _ = ms.attend_blocks(0, q, i32(one), want_lse=True, **good)
    assert ((la[3] - lb[3]) - math.log(12)).abs().max() < 1e-4
    ms.close()


def test_lists_and_tables_behind_32_bits():
    """Row numbers times K/V heads times list entries pass 2^31: lists of 2^23 rows, 4 heads, 80 entries."""
    rows, hk, k = (1 << 23) + 4, 4, 80
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("not enough memory")
    rng = random.Random(1)
    ms = store(hk, 16)
    tables, nb = paged(rng, [400], 16)
    cache, gen = fill_cache(1, nb, 16, hk, 16, False, "NHD", 1)
    lists = torch.full((rows, hk, k), -1, dtype=torch.int32, device=DEV)
    small = lists_of(rng, [0, 4], [400], 4, hk, 16, k, "sorted")
    lists[-4:] = i32(small)
    q = torch.zeros((rows, hk, 16), dtype=torch.bfloat16, device=DEV)
    q[-4:] = torch.randn((4, hk, 16), generator=gen, device=DEV).to(torch.bfloat16)
    out = torch.zeros_like(q)
    ms.attend_blocks(0, q, lists, cache, i32([rows - 4, rows]), i32([400]), tables, out=out)
    want, _ = check_sparse(ms, cache, q[-4:].clone(), [0, 4], [400], tables, small)
    assert torch.equal(out[-4:], want) and not out[:-4].any()
    box = boxes(gen, nb, hk, 16)
    got = torch.full((rows, hk, k), -7, dtype=torch.int32, device=DEV)
    ms.select_blocks(q, cache, box, i32([rows - 4, rows]), i32([400]), tables, k, out_blocks=got)
    few, _ = ms.select_blocks(q[-4:].clone(), cache, box, i32([0, 4]), i32([400]), tables, k)
    assert torch.equal(got[-4:], few) and bool((got[:-4] == -7).all())
    ms.close()


# ------------------------------------------------------------------------------------------------ together
@pytest.mark.parametrize("graph", [False, True])
@pytest.mark.parametrize("fp8", [False, True])
def test_a_decode_step_over_selected_blocks(fp8, graph):
    """Injection's summaries once, then steps of grow, append, summarize, select, attend: each against the definitions; with as many blocks as there are
    it is the dense attention.  Also captured and replayed while the requests grow."""
    L, hk, hq, d, bs, nb = 2, 2, 8, 64, 16, 200
    rng = random.Random(4)
    ms = MemStore(n_layers=L, n_kv_heads=hk, head_dim=d, emb_dim=64, max_facts_per_user=1, max_kv_tokens=0)
    cache = PagedCache.allocate(L, nb, bs, hk, d, DEV, fill_bits=0, fp8=fp8, k_scale=0.02, v_scale=0.02)
    box = ms.allocate_summaries(cache)
    prompt = [700, 40, 15, 333]
    n, width, steps, k = len(prompt), 50, 20, 6
    tables, free, taken = i32(np.full((n, width), -1)), i32(np.random.default_rng(0).permutation(nb)), i32([0])
    gen = torch.Generator(device=DEV).manual_seed(2)
    made = lambda T, h: torch.randn((T, h, d), generator=gen, device=DEV).to(torch.bfloat16)  # noqa: E731
    g = ms.grow_blocks(i32([0] * n), i32(prompt), tables, cache, free, taken, sum(prompt))
    for layer in range(L):
        ms.append(layer, None, made(sum(prompt), hk), made(sum(prompt), hk), g.positions, g.slots, cache)
        ms.summarize_blocks(layer, cache, box[layer], g.seq_lens, tables)
    lens = g.seq_lens.clone()
    taken.copy_(g.n_taken)
    one = i32([1] * n)
    ins = [[made(n, h) for h in (hq, hk, hk)] for _ in range(L)]
    result = {}

    def step():
        g = ms.grow_blocks(lens, one, tables, cache, free, taken, n)
        seen = []
        for layer in range(L):
            q = ms.append(layer, *ins[layer], g.positions, g.slots, cache)
            ms.summarize_blocks(layer, cache, box[layer], g.seq_lens, tables, q_start=g.q_start, n_tokens=n)
            lists, _ = ms.select_blocks(q, cache, box[layer], g.q_start, g.seq_lens, tables, k, n_first=1, n_last=2)
            out, lse, _ = ms.attend_blocks(layer, q, lists, cache, g.q_start, g.seq_lens, tables, want_lse=True)
            every, _ = ms.select_blocks(q, cache, box[layer], g.q_start, g.seq_lens, tables, width)
            full, _, _ = ms.attend_blocks(layer, q, every, cache, g.q_start, g.seq_lens, tables)
            dense, _, _ = ms.attend(layer, q, cache, g.q_start, g.seq_lens, tables)
            seen.append((q, lists, out, lse, full, dense))
        lens.copy_(g.seq_lens)
        taken.copy_(g.n_taken)
        result.update(seen=seen, status=g.status)

    replay = step
    if graph:
        keep = [x.clone() for x in (cache.k, cache.v, box, tables, free, taken, lens)]
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step()
        torch.cuda.current_stream().wait_stream(side)
        captured = torch.cuda.CUDAGraph()
        with torch.cuda.graph(captured):
            step()
        for x, y in zip((cache.k, cache.v, box, tables, free, taken, lens), keep):
            x.copy_(y)
        replay = captured.replay
    for i in range(steps):
        for layer in range(L):
            for x in ins[layer]:
                x.copy_(torch.randn(x.shape, generator=gen, device=DEV))
        replay()
        torch.cuda.synchronize()
        now = [p + i + 1 for p in prompt]
        assert lens.tolist() == now and result["status"].tolist() == [0] * n
        for layer, (q, lists, out, lse, full, dense) in enumerate(result["seen"]):
            assert torch.equal(full, dense)
            if i % 7 == 0:
                x = token_major(cache, layer)
                x = x.view(ref.F8).float() if fp8 else x.float()
                for r, m in enumerate(now):  # the summaries kept step by step are those of all keys
                    for b in range(-(-m // bs)):
                        keys = x[int(tables[r, b]), : min(bs, m - b * bs)]
                        assert torch.equal(box[layer, int(tables[r, b])], torch.stack([keys.amin(0), keys.amax(0)], 1).to(torch.bfloat16))
                run_select(ms, q, box[layer], list(range(n + 1)), now, tables, nb, bs, k, 1, 2)
                a, la = check_sparse(ms, cache, q, list(range(n + 1)), now, tables, lists.cpu().numpy().astype(np.int64), layer=layer)
                assert torch.equal(a, out) and torch.equal(la, lse)
    ms.close()


def test_selection_and_sparse_attention_on_another_stream_and_with_two_graphs_side_by_side():
    rng = random.Random(12)
    lens, bs = [9000, 300, 20000], 16
    tables, nb = paged(rng, lens, bs)
    cache, gen = fill_cache(1, nb, bs, 2, 128, False, "NHD", 4)
    ms = store(2, 128)
    box = ms.allocate_summaries(cache)[0]
    ms.summarize_blocks(0, cache, box, i32(lens), tables)
    qs = [torch.randn((3, 8, 128), generator=gen, device=DEV).to(torch.bfloat16) for _ in range(2)]
    q_start, ln = i32([0, 1, 2, 3]), i32(lens)

    def call(q, stream=None):
        lists, _ = ms.select_blocks(q, cache, box, q_start, ln, tables, 40, stream=stream)
        return lists, ms.attend_blocks(0, q, lists, cache, q_start, ln, tables, stream=stream)[0]

    want = [tuple(x.clone() for x in call(q)) for q in qs]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = call(qs[0], side)
    side.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(got, want[0]))
    graphs, outs = [], []
    for q in qs:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(call(q))
        graphs.append(g)
    for o in outs:
        o[1].zero_()
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(20):
        for g, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                g.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for o, w in zip(outs, want) for x, y in zip(o, w))
    ms.close()
