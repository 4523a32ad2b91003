"""GPU tests of drafted trees (memstore_plan_tree, memstore_attend_tree, memstore_accept) against plain 64-bit implementations, with the cases
where such kernels go wrong."""
import math
import random

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    import drafts_ref as dr
    import serving_ref as ref
    from paper_2607_27090_b200 import memstore as M
    from paper_2607_27090_b200.memstore import Accepted, MemStore, MemStoreError, PagedCache
    from test_gpu_serving import check_attend, fill_cache, i32, paged, store

DEV = "cuda"


# ------------------------------------------------------------------------------------------------ plan
def run_plan(ms, trees, words, starts, pad=0, in_place=False):
    q_start = [0] + [int(x) for x in np.cumsum([len(t) for t in trees])]
    T = q_start[-1] + pad
    parents = np.full(T, -7, np.int32)
    positions = np.full(T, -9, np.int32)
    want_pos, want_mask, want_st = positions.copy(), np.full((T, words), 77, np.int32), []
    for r, t in enumerate(trees):
        a, b = q_start[r], q_start[r + 1]
        parents[a:b] = t
        if len(t):
            positions[a] = starts[r]
    want_pos[:] = positions if in_place else -9
    for r, t in enumerate(trees):
        a, b = q_start[r], q_start[r + 1]
        if len(t) > 32 * words:
            want_st.append(256)
            continue
        made = dr.plan(t, words)
        want_st.append(0 if made else 512)
        want_pos[a:b] = -1 if made is None or (len(t) and starts[r] < 0) else np.array(made[0], np.int32) + (starts[r] if len(t) else 0)
        want_mask[a:b] = 0 if made is None else made[1]
    p, m, st = i32(positions), i32(np.full((T, words), 77)), i32([-5] * len(trees))
    o = p if in_place else i32(np.full(T, -9))
    ms.plan_tree(i32(parents), i32(q_start), p, out_positions=o, out_mask=m, out_status=st)
    torch.cuda.synchronize()
    assert np.array_equal(m.cpu().numpy(), want_mask)
    assert np.array_equal(o.cpu().numpy(), want_pos)
    assert st.tolist() == want_st


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("nreq,hi,words,chain", [(1, 1, 1, 0.0), (3, 32, 1, 0.3), (40, 33, 2, 0.0), (7, 700, 22, 0.2), (2, 4096, 128, 0.9), (200, 90, 3, 1.0),
                                                 (5, 300, 128, 0.5)])  # fmt: skip
def test_plan_against_the_definition(nreq, hi, words, chain, in_place):
    rng = random.Random(nreq * 100 + hi)
    ms = store()
    sizes = [rng.choice([hi, 1, 0, rng.randint(0, hi)]) if nreq > 1 else hi for _ in range(nreq)]
    trees = [dr.tree(rng, n, chain) if n else [] for n in sizes]
    run_plan(ms, trees, words, [rng.randrange(1 << 23) for _ in trees], pad=rng.choice([0, 5]), in_place=in_place)
    ms.close()


def test_plan_reports_what_it_refuses():
    ms = store()
    for in_place in (False, True):
        # a forest is fine; parents behind or on the node itself, below -1, far outside; too many nodes; a request that was refused blocks
        trees = [[-1, -1, 0, 1], [-1, 1, 0], [-1, 0, -2], [-1, 2, 0], [0, 0], [-1, 2**31 - 1], [-1] * 33, [-1, 0, 0], [-1]]
        run_plan(ms, trees, 1, [5, 6, 7, 8, 9, 10, 11, -1, 0], pad=2, in_place=in_place)
    # ranges outside the arrays
    parents, pos = i32([-1, 0, 1, 2]), i32([3, 3, 3, 3])
    st = i32([9] * 4)
    mask = i32(np.full((4, 1), 5))
    ms.plan_tree(parents, i32([2, 1, -1, 3, 5]), pos, out_positions=i32([0] * 4), out_mask=mask, out_status=st)
    assert st.tolist() == [256, 256, 256, 256] and (mask == 5).all()
    # new outputs: padding is -1 and 0
    p, m, s = ms.plan_tree(parents, i32([0, 2]), pos, 2)
    assert p.tolist() == [3, 4, -1, -1] and m.tolist() == [[1, 0], [3, 0], [0, 0], [0, 0]] and s is None
    for words in (0, -1):
        with pytest.raises(ValueError):
            ms.plan_tree(parents, i32([0, 2]), pos, words)
    with pytest.raises(MemStoreError):
        ms.plan_tree(parents, i32([0, 2]), pos, 129)
    with pytest.raises(ValueError):
        ms.plan_tree(parents, i32([0, 2]), pos[:3], 1)
    with pytest.raises(TypeError):
        ms.plan_tree(parents.long(), i32([0, 2]), pos, 1)
    ms.plan_tree(parents[:0], i32([0]), pos[:0], 1)  # nothing at all
    ms.close()


# ------------------------------------------------------------------------------------------------ attention
def check_tree(ms, cache, q, q_start, lens, tables, mask, layer=0, scale=0.0, max_q_len=0, want_status=None, wide=True, **kw):
    """Against the definition; with ``wide`` once more with tables of many more columns, which steers the call to the kernel for long contexts."""
    T, hq, d = q.shape
    if wide:
        pad = torch.full((tables.shape[0], 40000 // cache.block_size + 1000), -1, dtype=torch.int32, device=DEV)
        few = torch.tensor([st & 4 for st in want_status or []]).any().item()
        if not few:
            check_tree(ms, cache, q, q_start, lens, torch.cat([tables, pad], 1), mask, layer, scale, max_q_len, want_status, False, **kw)
    out = torch.full((T, hq, d), 9.0, dtype=torch.bfloat16, device=DEV)
    lse = torch.full((T, hq), 9.0, device=DEV)
    status = i32([-5] * len(lens))
    ms.attend_tree(layer, q, i32(mask), cache, i32(q_start), i32(lens), tables, scale=scale, max_q_len=max_q_len, out=out, out_lse=lse, out_status=status, **kw)
    torch.cuda.synchronize()

    def see(r, head, n):
        a, b = q_start[r], q_start[r + 1]
        if b - a > 32 * mask.shape[1]:
            return None
        bits, place = dr.bits_of(mask[a:b], b - a), np.arange(n) - (n - (b - a))
        return np.where(place[None] < 0, True, bits[:, np.clip(place, 0, b - a - 1)])

    compare(out, lse, dr.attend_seen(q, cache, layer, q_start, lens, tables, ms.n_kv_heads, scale or 1.0 / math.sqrt(d), 9.0, see))
    assert status.tolist() == (want_status or [0] * len(lens))
    return out, lse


def compare(out, lse, wanted):
    want, wl, tol, ltol = wanted
    fin = torch.isfinite(want)
    assert torch.equal(torch.isfinite(out.double()), fin) and torch.equal(torch.isnan(out.double()), torch.isnan(want))
    err = torch.where(fin, (out.double() - torch.where(fin, want, 0.0)).abs() - tol, 0.0)
    assert (err <= 0).all(), f"out: worst excess {err.max().item()} at {np.unravel_index(err.argmax().item(), err.shape)}"
    lf = torch.isfinite(wl)
    assert torch.equal(lse.double()[~lf], wl[~lf])
    le = torch.where(lf, (lse.double() - torch.where(lf, wl, 0.0)).abs() - ltol, 0.0)
    assert (le <= 0).all(), f"lse: worst excess {le.max().item()}"


def masks(rng, q, words, kind, pad=0):
    """Trees, any bits at all, or none."""
    rows = []
    for n in q:
        if kind == "tree":
            rows.append(dr.plan(dr.tree(rng, n), words)[1] if n else np.zeros((0, words), np.int32))
        elif kind == "any":
            rows.append(np.array([[rng.getrandbits(32) for _ in range(words)] for _ in range(n)], np.uint32).reshape(n, words).view(np.int32))
        else:
            rows.append(np.zeros((n, words), np.int32))
    return np.concatenate([*rows, np.full((pad, words), -1, np.int32)])


TREE_SHAPES = [
    # d, heads, kv heads, block size, 8-bit, layout
    (64, 4, 2, 16, False, "NHD"), (128, 32, 8, 16, False, "NHD"), (128, 40, 8, 32, False, "HND"), (128, 8, 8, 16, True, "NHD"), (64, 14, 2, 64, True, "HND"),
    (16, 2, 1, 16, False, "NHD"), (32, 3, 1, 8, False, "NHD"), (256, 8, 2, 16, False, "NHD"), (256, 4, 4, 16, True, "NHD"), (32, 4, 4, 16, True, "HND"),
    (16, 33, 3, 5, True, "NHD"), (128, 16, 1, 24, False, "NHD"), (64, 20, 1, 1, False, "HND"), (128, 7, 1, 128, True, "NHD")]  # fmt: skip


@pytest.mark.parametrize("d,hq,hk,bs,fp8,layout", TREE_SHAPES)
@pytest.mark.parametrize("kind,nreq,q_hi,len_hi", [("tree", 1, 1, 1), ("tree", 5, 9, 700), ("any", 6, 40, 333), ("tree", 3, 300, 900), ("none", 4, 70, 200)])
def test_tree_attention_against_the_definition(d, hq, hk, bs, fp8, layout, kind, nreq, q_hi, len_hi):
    rng = random.Random(d * 7 + hq + nreq)
    q = [rng.choice([q_hi, 1, rng.randint(0, q_hi)]) for _ in range(nreq)]
    lens = [max(rng.randint(0, len_hi), n) for n in q]
    q_start = [0] + [int(x) for x in np.cumsum(q)]
    tables, nb = paged(rng, lens, bs)
    cache, gen = fill_cache(2, nb, bs, hk, d, fp8, layout, nreq)
    ms = store(hk, d, 2)
    x = (2.0 * torch.randn((q_start[-1] + 3, hq, d), generator=gen, device=DEV)).to(torch.bfloat16)  # rows behind the last request too
    mask = masks(rng, q, max(1, -(-max(q) // 32)) + rng.choice([0, 1]), kind, pad=3)
    check_tree(ms, cache, x, q_start, lens, tables, mask, layer=1)
    check_tree(ms, cache, x, q_start, lens, tables, mask, layer=1, scale=0.9, max_q_len=max(q))
    ms.close()


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("n,len_", [(1, 1), (33, 33), (64, 65), (64, 127), (64, 192), (31, 4095), (64, 20001), (200, 150), (130, 0), (300, 257), (65, 128), (5, 3)])
def test_tree_attention_lengths_around_tile_and_word_borders(n, len_, fp8):
    """Masks whose first node lies anywhere in a tile and in a word; more nodes than tokens in the cache: the first nodes have no keys."""
    rng = random.Random(n * 1000 + len_)
    tables, nb = paged(rng, [len_], 16)
    cache, gen = fill_cache(1, nb, 16, 2, 128, fp8, "NHD", len_)
    ms = store(2, 128)
    q = torch.randn((n, 8, 128), generator=gen, device=DEV).to(torch.bfloat16)
    for kind in ("tree", "any", "none"):
        out, lse = check_tree(ms, cache, q, [0, n], [len_], tables, masks(rng, [n], -(-n // 32), kind))
        if kind == "none" and n >= len_:
            assert (out == 0).all() and (lse == -math.inf).all()
    ms.close()


@pytest.mark.parametrize("fp8,d", [(False, 64), (True, 64), (False, 128), (True, 128)])
@pytest.mark.parametrize("seed", range(6))
def test_tree_attention_random_batches(fp8, d, seed):
    rng = random.Random(1000 * d + 10 * seed + fp8)
    hk = rng.choice([1, 2, 3])
    hq = hk * rng.choice([1, 3, 4, 5, 7, 12, 16])
    nreq, bs = rng.choice([1, 2, 7, 19]), rng.choice([16, 16, 8, 24, 64, 11])
    q_hi = rng.choice([40, 300, 900]) if nreq < 7 else rng.choice([5, 60, 200])
    q = [rng.choice([0, 1, rng.randint(0, q_hi), rng.randint(0, q_hi)]) for _ in range(nreq)]
    lens = [rng.choice([n, n + rng.randint(0, 2500), max(0, n - rng.randint(0, 40))]) for n in q]
    q_start = [0] + [int(x) for x in np.cumsum(q)]
    tables, nb = paged(rng, lens, bs)
    cache, gen = fill_cache(1, nb, bs, hk, d, fp8, rng.choice(["NHD", "HND"]), seed)
    ms = store(hk, d)
    x = (rng.choice([0.3, 2.0, 6.0]) * torch.randn((q_start[-1] + 1, hq, d), generator=gen, device=DEV)).to(torch.bfloat16)
    mask = masks(rng, q, max(1, -(-max(q) // 32)), rng.choice(["tree", "any"]), pad=1)
    check_tree(ms, cache, x, q_start, lens, tables, mask, max_q_len=rng.choice([0, max(q), 1]))  # (the bound may be wrong)
    ms.close()


@pytest.mark.parametrize("fp8,d,hq,n", [(False, 128, 4, 5), (True, 128, 4, 5), (False, 128, 4, 90), (True, 128, 4, 90), (False, 64, 4, 90), (True, 64, 4, 90),
                                       (False, 32, 2, 40), (True, 256, 2, 20)])  # fmt: skip
def test_tree_attention_keeps_what_a_row_does_not_see_away_from_it(fp8, d, hq, n):
    """NaN and infinities in keys and values that some rows see and others do not, and behind the last token."""
    rng = random.Random(n + d)
    len_ = 300
    tables, nb = paged(rng, [len_], 16)
    cache, gen = fill_cache(1, nb, 16, 1, d, fp8, "NHD", 5, k_scale=0.05)
    q = torch.randn((n, hq, d), generator=gen, device=DEV).to(torch.bfloat16)
    mask = masks(rng, [n], -(-n // 32), "tree")
    ms = store(1, d)
    nan8, put = 0x7F, (lambda t, j, e, x: t[0, int(tables[0, j // 16]), j % 16, 0].__setitem__(e, x))
    pos0 = len_ - n
    # values: one node that few rows see, one of the context, and keys of nodes that nobody sees
    hidden = [1, n - 1]
    for j in hidden:
        mask[:, j // 32] &= ~np.int32(1 << (j % 32)) if j % 32 < 31 else np.int32(0x7FFFFFFF)
    for e, x in ((0, math.nan), (3, math.inf), (5, -math.inf)):
        put(cache.v, pos0 + 2, e, nan8 if fp8 else x)
        put(cache.v, pos0 - 1, (e + 7) % d, nan8 if fp8 else x)
    for j in hidden:
        put(cache.k, pos0 + j, slice(None), nan8 if fp8 else math.nan)
        put(cache.v, pos0 + j, slice(None), nan8 if fp8 else math.inf)
    blk = int(tables[0, len_ // 16])
    for t in (cache.k, cache.v):  # the rest of the last block
        t[0, blk, len_ % 16 :] = nan8 if fp8 else math.nan
    out, _ = check_tree(ms, cache, q, [0, n], [len_], tables, mask)
    saw = dr.bits_of(mask, n)[:, 2]
    assert torch.isfinite(out[:, :, 1]).all() and not torch.isfinite(out[torch.as_tensor(saw, device=DEV), :, 0]).any()
    assert torch.isfinite(out[torch.as_tensor(~saw, device=DEV), :, 0]).all()
    ms.close()


def test_tree_attention_with_a_chains_mask_is_the_causal_one():
    """A chain of nodes sees what causal attention shows it: both calls are near the same definition, on both kernels."""
    rng = random.Random(3)
    q = [1, 70, 7, 40]
    lens = [500, 700, 33, 2000]
    q_start = [0, 1, 71, 78, 118]
    for d, fp8 in ((128, False), (64, True), (32, False)):
        tables, nb = paged(rng, lens, 16)
        cache, gen = fill_cache(1, nb, 16, 2, d, fp8, "NHD", 3)
        ms = store(2, d)
        x = torch.randn((118, 8, d), generator=gen, device=DEV).to(torch.bfloat16)
        mask = np.concatenate([dr.plan([j - 1 for j in range(n)], 3)[1] for n in q])
        check_attend(ms, cache, x, q_start, lens, tables)
        check_tree(ms, cache, x, q_start, lens, tables, mask)
        ms.close()


def test_tree_attention_holes_strides_and_refusals():
    bs, lens, q_start = 16, [700, 500, 300, 90], [0, 40, 110, 120, 185]
    rng = random.Random(6)
    tables, nb = paged(rng, lens, bs, width_extra=0)
    tables[0, 3], tables[0, 40], tables[1, 31], tables[1, 0] = -1, nb, nb + 5, -(2**31)
    cache, gen = fill_cache(1, nb, bs, 2, 128, False, "NHD", 6)
    ms = store(2, 128)
    fused = torch.randn((185, 12 * 128), generator=gen, device=DEV).to(torch.bfloat16)
    q = fused[:, : 8 * 128].unflatten(1, (8, 128))  # a slice of a fused projection
    mask = masks(rng, [40, 70, 10, 65], 3, "tree")
    check_tree(ms, cache, q, q_start, lens, tables, mask, want_status=[8, 8, 0, 0])
    check_tree(ms, cache, q, q_start, lens, tables[:, :40].contiguous(), mask, want_status=[12, 8, 0, 0])
    # more nodes than the mask has bits: left out
    out, _ = check_tree(ms, cache, q, q_start, lens, tables, mask[:, :2].copy(), want_status=[8, 256, 0, 256])
    assert (out[40:110] == 9).all() and (out[120:] == 9).all()
    # in place
    want = ms.attend_tree(0, q, i32(mask), cache, i32(q_start), i32(lens), tables)[0]
    x = q.clone()
    assert ms.attend_tree(0, x, i32(mask), cache, i32(q_start), i32(lens), tables, out=x)[0] is x and torch.equal(x, want)
    good = dict(cache=cache, q_start=i32(q_start), seq_lens=i32(lens), block_tables=tables)
    for bad, err in ((i32(mask).long(), TypeError), (i32(mask)[:100], ValueError), (i32(mask)[:, 0], ValueError), (i32(np.zeros((185, 0))), MemStoreError),
                     (i32(np.zeros((185, 129))), MemStoreError), (torch.zeros((185, 3), dtype=torch.int32), TypeError)):  # fmt: skip
        with pytest.raises(err):
            ms.attend_tree(0, q, bad, **good)
    with pytest.raises(MemStoreError):
        ms.attend_tree(1, q, i32(mask), **good)
    with pytest.raises(MemStoreError):
        ms.attend_tree(0, q, i32(mask), scale=math.inf, **good)
    with pytest.raises(MemStoreError):
        ms.attend_tree(0, q, i32(mask), workspace=torch.empty(256, dtype=torch.uint8, device=DEV), **good)
    with pytest.raises(MemStoreError):
        ms.attend_tree(0, q[:, :7], i32(mask), **good)
    ms.close()


def test_tree_attention_reports_a_wait_that_ran_out_and_works_again():
    rng = random.Random(2)
    tables, nb = paged(rng, [900], 16, width_extra=8000)  # (as wide as for a long context, which steers the call to the kernel that waits)
    cache, gen = fill_cache(1, nb, 16, 2, 128, False, "NHD", 2)
    ms = store(2, 128)
    q = torch.randn((60, 8, 128), generator=gen, device=DEV).to(torch.bfloat16)
    mask = masks(rng, [60], 2, "tree")
    st = i32([0])
    ms.test_hooks(4096, True)
    ms.attend_tree(0, q, i32(mask), cache, i32([0, 60]), i32([900]), tables, out_status=st)
    torch.cuda.synchronize()
    assert st.tolist() == [32] and ms.stats()["kernel_timeouts"] == 1
    ms.test_hooks()
    check_tree(ms, cache, q, [0, 60], [900], tables, mask)
    assert ms.stats()["kernel_timeouts"] == 0
    ms.close()


# ------------------------------------------------------------------------------------------------ acceptance
def run_accept(rng, sizes, starts, layers=2, hk=2, d=64, bs=16, fp8=False, layout="NHD", hit=0.85, pad=0, stacked=False, shuffle_free=True, in_place=False,
               with_list=True, dup=0.3, break_=None, taken_extra=2):  # fmt: skip
    """One call against the rules; break_(state): spoils the inputs before the call (positions, lengths, tables ...)."""
    nreq = len(sizes)
    lens = [s + n for s, n in zip(starts, sizes)]
    tables, nb = paged(rng, lens, bs)
    tables = tables.cpu().numpy().copy()
    cache = PagedCache.allocate(layers, nb, bs, hk, d, DEV, layout=layout, stacked=stacked, fp8=fp8)
    gen = torch.Generator(device=DEV).manual_seed(rng.randrange(1 << 30))
    for t in (cache.k, cache.v):
        t.copy_(torch.randint(0, 256, t.shape, generator=gen, device=DEV).to(torch.uint8) if fp8 else torch.randn(t.shape, generator=gen, device=DEV).to(torch.bfloat16))
    q_start = [0] + [int(x) for x in np.cumsum(sizes)]
    T = q_start[-1] + pad
    s = dict(parents=np.full(T, -1, np.int64), tokens=np.zeros(T, np.int64), choices=np.zeros(T, np.int64), positions=np.full(T, -1, np.int64))
    for r, n in enumerate(sizes):
        a = q_start[r]
        s["parents"][a : a + n] = dr.tree(rng, n, 0.4) if n else []
        for i in range(n):
            p = s["parents"][a + i]
            twin = [j for j in range(1, i) if s["parents"][a + j] == p]
            s["tokens"][a + i] = s["tokens"][a + rng.choice(twin)] if twin and rng.random() < dup else rng.randrange(1 << 17)
            s["positions"][a + i] = starts[r] + i
        for i in range(n):
            kids = [j for j in range(i + 1, n) if s["parents"][a + j] == i]
            s["choices"][a + i] = s["tokens"][a + rng.choice(kids)] if kids and rng.random() < hit else rng.randrange(1 << 17, 1 << 18)
    free = list(range(1000, 1000 + sum(-(-n // bs) for n in lens) + taken_extra)) + [5, 6, 7]
    s.update(lens=list(lens), tables=tables, free=np.array(free), taken=len(free) - 3, q_start=list(q_start))
    if break_:
        break_(s)
    k0, v0 = (x.clone() for x in (cache.k, cache.v))
    want = dict(path=np.full(T, -3), a=[], said=[], lens=[], st=[], free=np.array(s["free"]).copy(), taken=s["taken"])
    planes = {"k": k0, "v": v0}
    at = lambda b, o: (slice(None), b, slice(None), o) if layout == "HND" else (slice(None), b, o)  # noqa: E731
    asked, ok_list = 0, 0 <= s["taken"] <= len(s["free"])
    for r in range(nreq):
        a, b, n = s["q_start"][r], s["q_start"][r + 1], s["lens"][r]
        st, way = 0, []
        if not (0 <= a <= b <= T):
            st, b = 256, a
        elif n < 0:
            st = 256
        elif b > a:
            first = int(s["positions"][a])
            st = 64 if first < 0 else 256 if first + (b - a) != n else 0
        if st == 0 and b > a:
            way = dr.walk(s["parents"][a:b].tolist(), s["tokens"][a:b].tolist(), s["choices"][a:b].tolist())
            name = lambda pos: int(s["tables"][r, pos // bs]) if pos // bs < s["tables"].shape[1] else None  # noqa: E731
            for i, c in enumerate(way):
                if c == i:
                    continue
                src, dst = name(first + c), name(first + i)
                for x in (src, dst):
                    st |= 4 if x is None else 0 if 0 <= x < nb else 8
                if all(x is not None and 0 <= x < nb for x in (src, dst)):
                    for t in planes.values():
                        t[at(dst, (first + i) % bs)] = t[at(src, (first + c) % bs)]
            end, width = first + len(way), s["tables"].shape[1]
            if with_list:
                going = s["tables"][r, min(-(-end // bs), width) : min(-(-n // bs), width)]
                ids = [x for x in going.tolist() if 0 <= x < nb]
                asked += len(ids)
                st |= 8 if len(ids) < len(going) else 0
                if ids and not (ok_list and asked <= s["taken"]):
                    st |= 128
                else:
                    want["taken"] -= len(ids)
                    lo = s["taken"] - asked
                    want["free"][lo : lo + len(ids)] = ids
        want["a"].append(len(way))
        want["said"].append(int(s["choices"][a + way[-1]]) if way else -1)
        want["lens"].append(first + len(way) if way else n)
        want["st"].append(st)
        if b > a:
            want["path"][a:b] = way + [-1] * (b - a - len(way))
    ms = store(hk, d, layers)
    f, t, ln = i32(s["free"]), i32([s["taken"]]), i32(s["lens"])
    fresh = lambda m: i32([-3] * m)  # noqa: E731
    out = Accepted(fresh(T), fresh(nreq), fresh(nreq), ln if in_place else fresh(nreq), (t if in_place else fresh(1)) if with_list else None, fresh(nreq))
    tab = i32(s["tables"])
    got = ms.accept(i32(s["parents"]), i32(s["tokens"]), i32(s["choices"]), i32(s["positions"]), i32(s["q_start"]), ln, tab, cache, f if with_list else None,
                    t if with_list else None, out=out)  # fmt: skip
    torch.cuda.synchronize()
    assert got is out
    assert out.path.tolist() == want["path"].tolist()
    assert out.n_accepted.tolist() == want["a"] and out.next_tokens.tolist() == want["said"]
    assert out.seq_lens.tolist() == want["lens"] and out.status.tolist() == want["st"]
    if with_list:
        assert f.tolist() == want["free"].tolist() and out.n_taken.tolist() == [want["taken"]]
    assert torch.equal(tab, i32(s["tables"]))
    for t1, t2 in ((cache.k, planes["k"]), (cache.v, planes["v"])):
        assert torch.equal(t1.contiguous().view(torch.uint8), t2.contiguous().view(torch.uint8))
    ms.close()
    return want


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("layers,hk,d,bs,fp8,layout,stacked", [(2, 2, 64, 16, False, "NHD", False), (1, 1, 16, 5, True, "NHD", False), (3, 8, 128, 16, False, "NHD", True),
                                                               (2, 3, 128, 1, True, "HND", False), (33, 4, 256, 32, False, "HND", True), (2, 1, 16, 64, False, "NHD", False)])  # fmt: skip
def test_accept_against_the_rules(layers, hk, d, bs, fp8, layout, stacked, in_place):
    rng = random.Random(layers * 100 + d + bs)
    for sizes in ([1], [26], [0], [5, 0, 64, 1, 33, 128, 2], [200, 129, 1, 300]):
        starts = [rng.choice([0, 1, bs - 1, rng.randrange(70)]) for _ in sizes]
        run_accept(rng, sizes, starts, layers, hk, d, bs, fp8, layout, stacked=stacked, in_place=in_place, pad=rng.choice([0, 3]), hit=rng.choice([0.5, 0.9, 1.0]))


def test_accept_many_requests_and_without_a_free_list():
    rng = random.Random(8)
    sizes = [rng.choice([0, 1, rng.randint(1, 30)]) for _ in range(700)]
    starts = [rng.randrange(40) for _ in sizes]
    want = run_accept(rng, sizes, starts, layers=1, hk=1, d=16)
    assert sum(a > 2 for a in want["a"]) > 100
    run_accept(rng, sizes[:9], starts[:9], with_list=False)
    run_accept(rng, [], [])


def test_accept_long_chains_and_whole_trees():
    rng = random.Random(9)

    def chain(s):
        n = len(s["parents"])
        s["parents"][:] = np.arange(n) - 1
        s["tokens"][:] = np.arange(n) + 50
        s["choices"][:] = np.arange(n) + 51

    for n in (2, 32, 128, 129, 700):
        want = run_accept(rng, [n], [13], break_=chain)
        assert want["a"] == [n]

    def comb(s):  # every second node is a dead end: everything moves
        n = len(s["parents"])
        for i in range(1, n):
            s["parents"][i] = i - 2 if i % 2 == 0 else i - 1
        s["tokens"][:] = [7 if i % 2 == 0 else 9 for i in range(n)]
        s["choices"][:] = 7

    for n in (3, 65, 200, 401):
        want = run_accept(rng, [n], [3], break_=comb, layers=2, hk=1, d=32)
        assert want["a"] == [(n + 1) // 2]


def test_accept_stays_inside_the_cache_where_rows_of_requests_overlap():
    """Two requests that share rows write their paths over one another's; no row is then read from a place in front of the cache's first."""
    ms, bs, n = store(1, 64, 1), 4, 10003
    row = bs * 64
    memory = torch.full((2, 10 * row), 3.0, dtype=torch.bfloat16, device=DEV)  # the cache is blocks 1 to 8 of this
    kv = memory[:, row : 9 * row]
    kv[:] = torch.arange(8 * bs, device=DEV).repeat_interleave(64).to(torch.bfloat16)
    cache = PagedCache(kv[0], kv[1], 8 * row, row, 64, 64, 8, bs)
    before = memory.clone()
    # request 0: rows 0 - 4, a chain that is accepted whole; request 2: from row 3 on, its root alone is accepted, after a look at all its nodes
    parents, tokens, choices, positions = np.zeros(n, np.int32), np.ones(n, np.int32), np.full(n, 9, np.int32), np.full(n, -1, np.int32)
    parents[:5], tokens[:5], choices[:5] = [-1, 0, 1, 2, 3], range(50, 55), range(51, 56)
    positions[0], positions[3] = 0, 100
    got = ms.accept(i32(parents), i32(tokens), i32(choices), i32(positions), i32([0, 5, 3, n]), i32([5, 7, 100 + n - 3]), i32([[0, 1], [2, 3], [4, 5]]), cache)
    torch.cuda.synchronize()
    assert got.n_accepted.tolist() == [5, 0, 1] and got.seq_lens.tolist() == [5, 7, 101] and got.status.tolist()[1] == M.REQ_BAD_LENGTH
    assert torch.equal(memory, before)


def test_accept_reports_what_it_refuses():
    rng = random.Random(10)
    sizes, starts = [12, 9, 20, 7, 15, 30, 11], [30, 31, 5, 0, 16, 3, 9]

    def spoil(s):
        q = s["q_start"]
        s["positions"][q[0]] = -1  # refused blocks: left as it is
        s["positions"][q[1]] += 1  # does not fit the length
        s["lens"][3] = -4
        s["tables"][2, 0] = 10**6
        s["tables"][4, 1] = -1
        s["tables"][5, 2] = -(2**31)

    run_accept(rng, sizes, starts, break_=spoil, hit=1.0)
    run_accept(rng, sizes, starts, break_=lambda s: s.update(tables=s["tables"][:, :2].copy()), hit=0.95)  # tables that are too short
    for taken in (-1, 10**6, 0, 1, 2, 3):  # counters that do not fit the list, or that the blocks do not fit in front of
        run_accept(rng, sizes, starts, bs=4, break_=lambda s: s.update(taken=taken), hit=0.6)  # noqa: B023

    run_accept(rng, [5, 5, 5, 5, 5, 5], [5] * 6, break_=lambda s: s.update(q_start=[0, 5, 40, 25, 25, 30, 29]))
    ms = store(2, 64, 2)
    cache = PagedCache.allocate(2, 8, 16, 2, 64, DEV)
    t = i32([[0, 1]])
    args = [i32([-1, 0]), i32([1, 2]), i32([2, 3]), i32([4, 5]), i32([0, 2]), i32([6]), t, cache]
    for i in range(6):
        bad = list(args)
        bad[i] = bad[i].long()
        with pytest.raises(TypeError):
            ms.accept(*bad)
    with pytest.raises(ValueError):
        ms.accept(*args, free_blocks=i32([1, 2]))
    with pytest.raises(ValueError):
        ms.accept(*args[:7], PagedCache.allocate(1, 8, 16, 2, 64, DEV))
    with pytest.raises(ValueError):
        ms.accept(*args[:6], i32([0, 1]), cache)
    ms.close()


# ------------------------------------------------------------------------------------------------ together
def loop_state(ms, nb, bs, d, hk, n_layers, lens):
    cache = PagedCache.allocate(n_layers, nb, bs, hk, d, DEV, fill_bits=0)
    tables = i32(np.full((len(lens), 40), -1))
    return cache, tables, i32(np.random.default_rng(1).permutation(nb)), i32([0])


@pytest.mark.parametrize("graph", [False, True])
def test_a_step_with_drafts_leaves_the_cache_as_steps_without_them_would(graph):
    """grow, plan, append, attend, accept: the cache of the accepted tokens is what appending those tokens alone writes, and a next step's attention is the
    same; also captured and replayed with other trees."""
    L, hk, hq, d, bs, nb = 2, 2, 8, 64, 16, 64
    rng = random.Random(4)
    ms = MemStore(n_layers=L, n_kv_heads=hk, head_dim=d, emb_dim=64, max_facts_per_user=1, max_kv_tokens=0, rope_theta=5.0e5)
    n_req, N, words = 3, 24, 1
    gen = torch.Generator(device=DEV).manual_seed(1)
    vocab = 40
    emb = {k: torch.randn((L, vocab, h, d), generator=gen, device=DEV).to(torch.bfloat16) for k, h in (("q", hq), ("k", hk), ("v", hk))}
    cache, tables, free, taken = loop_state(ms, nb, bs, d, hk, L, [0] * n_req)
    prompt = [rng.randint(20, 70) for _ in range(n_req)]
    lens = i32([0] * n_req)
    texts = [[rng.randrange(vocab) for _ in range(n)] for n in prompt]

    def feed(cache, g, toks):
        outs = []
        for layer in range(L):
            q = ms.append(layer, emb["q"][layer][toks], emb["k"][layer][toks], emb["v"][layer][toks], g.positions, g.slots, cache)
            outs.append(q)
        return outs

    g = ms.grow_blocks(lens, i32(prompt), tables, cache, free, taken, sum(prompt))
    feed(cache, g, torch.tensor(sum(texts, []), device=DEV))
    lens, taken = g.seq_lens, g.n_taken
    parents, tokens, choices = (torch.zeros(n_req * N, dtype=torch.int32, device=DEV) for _ in range(3))
    new = i32([N] * n_req)
    result = {}

    def step():
        g = ms.grow_blocks(lens, new, tables, cache, free, taken, n_req * N)
        pos, mask, _ = ms.plan_tree(parents, g.q_start, g.positions, words)
        grown = g._replace(positions=pos)
        qs = feed(cache, grown, tokens.long())
        outs = [ms.attend_tree(layer, qs[layer], mask, cache, g.q_start, g.seq_lens, tables)[0] for layer in range(L)]
        acc = ms.accept(parents, tokens, choices, pos, g.q_start, g.seq_lens, tables, cache, free, g.n_taken)
        lens.copy_(acc.seq_lens)
        taken.copy_(acc.n_taken)
        result.update(outs=outs, acc=acc, status=g.status)

    def fill():
        """Trees and choices of the next step; the accepted tokens by request."""
        p, t, c, got = [], [], [], []
        for _ in range(n_req):
            pr = dr.tree(rng, N, 0.3)
            tk = [rng.randrange(vocab) for _ in range(N)]
            ch = []
            for i in range(N):
                kids = [j for j in range(N) if pr[j] == i]
                ch.append(tk[rng.choice(kids)] if kids and rng.random() < 0.9 else rng.randrange(vocab))
            way = dr.walk(pr, tk, ch)
            got.append(([tk[i] for i in way], way))
            p, t, c = p + pr, t + tk, c + ch
        parents.copy_(i32(p))
        tokens.copy_(i32(t))
        choices.copy_(i32(c))
        return got

    graph_ = None
    if graph:
        keep = [x.clone() for x in (cache.k, cache.v, tables, free, taken, lens)]
        fill()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step()
        torch.cuda.current_stream().wait_stream(side)
        for x, y in zip((cache.k, cache.v, tables, free, taken, lens), keep):
            x.copy_(y)
        graph_ = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph_):
            step()
        for x, y in zip((cache.k, cache.v, tables, free, taken, lens), keep):
            x.copy_(y)
    for _ in range(5):
        before = [len(t) for t in texts]
        got = fill()
        if graph_:
            graph_.replay()
        else:
            step()
        torch.cuda.synchronize()
        assert result["status"].tolist() == [0] * n_req and result["acc"].status.tolist() == [0] * n_req
        assert result["acc"].n_accepted.tolist() == [len(w) for _, w in got]
        for r, (toks, way) in enumerate(got):
            texts[r] += toks
        # the same texts, fed token after token without drafts
        plain, ptables, pfree, ptaken = loop_state(ms, nb, bs, d, hk, L, [0] * n_req)
        size = [len(t) for t in texts]
        pg = ms.grow_blocks(i32([0] * n_req), i32(size), ptables, plain, pfree, ptaken, sum(size))
        pq = feed(plain, pg, torch.tensor(sum(texts, []), device=DEV))
        assert lens.tolist() == size and taken.item() == sum(-(-n // bs) for n in size)
        for r, n in enumerate(size):
            j = torch.arange(n, device=DEV)
            for x, y in ((cache.k, plain.k), (cache.v, plain.v)):
                mine, theirs = (t[:, tab[r, j // bs].long(), j % bs] for t, tab in ((x, tables), (y, ptables)))
                assert torch.equal(mine, theirs)
        q_start = [0] + [int(x) for x in np.cumsum(size)]
        for layer in range(L):
            ref_out, _, _ = ms.attend(layer, pq[layer], plain, i32(q_start), i32(size), ptables)
            for r, (toks, way) in enumerate(got):
                a = q_start[r] + before[r]
                x, y = result["outs"][layer][torch.tensor(way, device=DEV) + r * N].float(), ref_out[a : a + len(way)].float()
                # on either side an output is off by 2^-8 of itself and 2^-8 of the mean of |V| under its weights
                assert ((x - y).abs() <= 2.0**-7 * 1.1 * (y.abs() + emb["v"][layer].float().abs().max())).all()
    ms.close()


@pytest.mark.parametrize("bs", [8, 16, 32, 64, 128, 256, 384, 4, 24])
@pytest.mark.parametrize("fp8,d", [(False, 64), (True, 64), (False, 128), (True, 128)])
def test_tree_attention_with_every_way_to_fetch_a_tile(bs, fp8, d):
    """Block sizes that tensor copies take and others, strides with gaps between blocks, heads and tokens, tables with holes, units that the halves share (few
    rows) and others, a cache whose unused places hold NaN."""
    rng = random.Random(bs + d + fp8)
    hk, hq, q, lens = 2, 10, [9, 40, 25, 60, 1], [700, 1300, 90, 2500, 333]
    q_start = [0] + [int(x) for x in np.cumsum(q)]
    tables, nb = paged(rng, lens, bs)
    tables[1, 1], tables[3, 0] = nb + 3, -7
    dt = torch.uint8 if fp8 else torch.bfloat16
    gen = torch.Generator(device=DEV).manual_seed(bs)
    planes = []
    for scale in (0.02, 0.03):
        wide = torch.full((1, nb, bs, hk + 1, d + 16), 0x7F if fp8 else math.nan, device=DEV, dtype=dt)
        x = torch.randn((1, nb, bs, hk, d), generator=gen, device=DEV)
        wide[:, :, :, :hk, :d] = (x / scale).clamp(-448, 448).to(ref.F8).view(torch.uint8) if fp8 else x.to(torch.bfloat16)
        planes.append(wide[:, :, :, :hk, :d])
    row = (hk + 1) * (d + 16)
    cache = PagedCache(planes[0], planes[1], nb * bs * row, bs * row, row, d + 16, nb, bs, k_scale=0.02, v_scale=0.03)
    for r, n in enumerate(lens):  # behind the last tokens
        blk = int(tables[r, n // bs])
        if n % bs and 0 <= blk < nb:
            for t in planes:
                t[0, blk, n % bs :] = 0x7F if fp8 else math.nan
    ms = store(hk, d)
    x = torch.randn((q_start[-1], hq, d), generator=gen, device=DEV).to(torch.bfloat16)
    status = [8 if (r == 1 and lens[1] > bs) or r == 3 else 0 for r in range(5)]
    check_tree(ms, cache, x, q_start, lens, tables, masks(rng, q, 2, "tree"), want_status=status)
    check_attend(ms, cache, x, q_start, lens, tables, want_status=status)
    ms.close()


def test_drafts_on_another_stream_and_with_two_graphs_side_by_side():
    rng = random.Random(12)
    sizes, lens = [40, 7, 64], [900, 300, 1500]
    q_start = [0, 40, 47, 111]
    tables, nb = paged(rng, lens, 16)
    cache, gen = fill_cache(1, nb, 16, 2, 128, False, "NHD", 4)
    ms = store(2, 128)
    xs = [torch.randn((111, 8, 128), generator=gen, device=DEV).to(torch.bfloat16) for _ in range(2)]
    mask = i32(masks(rng, sizes, 2, "tree"))
    args = (cache, i32(q_start), i32(lens), tables)
    want = [ms.attend_tree(0, x, mask, *args)[0].clone() for x in xs]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = ms.attend_tree(0, xs[0], mask, *args, stream=side)[0]
    side.synchronize()
    assert torch.equal(got, want[0])
    graphs, outs = [], []
    for x in xs:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(ms.attend_tree(0, x, mask, *args)[0])
        graphs.append(g)
    streams = [torch.cuda.Stream() for _ in range(2)]
    for o in outs:
        o.zero_()
    torch.cuda.synchronize()
    for _ in range(20):
        for g, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                g.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(o, w) for o, w in zip(outs, want))
    ms.close()


def test_mask_words_behind_32_bits_of_rows():
    """Row numbers times mask words pass 2^31 elements: masks of 2^24 rows of 128 words."""
    rows, words = (1 << 24) + 8, 128
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("not enough memory")
    ms = store(1, 16)
    tables, nb = paged(random.Random(1), [40], 16)
    cache, gen = fill_cache(1, nb, 16, 1, 16, False, "NHD", 1)
    mask = torch.zeros((rows, words), dtype=torch.int32, device=DEV)
    q = torch.zeros((rows, 1, 16), dtype=torch.bfloat16, device=DEV)
    tail = torch.randn((8, 1, 16), generator=gen, device=DEV).to(torch.bfloat16)
    q[-8:] = tail
    small = masks(random.Random(2), [8], words, "tree")
    mask[-8:] = i32(small)
    out = torch.zeros_like(q)
    ms.attend_tree(0, q, mask, cache, i32([rows - 8, rows]), i32([40]), tables, out=out)
    want, _ = check_tree(ms, cache, tail, [0, 8], [40], tables, small)
    assert torch.equal(out[-8:], want) and not out[:-8].any()
    ms.close()
