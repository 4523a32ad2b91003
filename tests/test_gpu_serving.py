"""GPU tests of the serving calls around the paged cache: block tables and slot maps (memstore_grow_blocks,
memstore_release_blocks), the rotation and cache write of new tokens (memstore_append), and their attention over the cache
(memstore_attend), against plain 64-bit implementations, with the cases where such kernels go wrong."""
import math
import random

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    import serving_ref as ref
    from parity import to_dev
    from paper_2607_27090_b200 import memstore as M
    from paper_2607_27090_b200.memstore import GrownBlocks, MemStore, PagedCache

DEV = "cuda"


def store(n_kv=2, d=64, layers=1, **kw):
    return MemStore(n_layers=layers, n_kv_heads=n_kv, head_dim=d, emb_dim=64, max_facts_per_user=1, max_kv_tokens=0, **kw)


def i32(x):
    return torch.tensor(np.asarray(x, np.int32), device=DEV)


def geometry(num_blocks, bs):
    return PagedCache.allocate(1, num_blocks, bs, 1, 16, DEV)


# ------------------------------------------------------------------------------------------------ block tables
def run_grow(ms, start, new, tables, free, taken, bs, num_blocks, capacity, in_place=False, max_position=1 << 24):
    cache = geometry(num_blocks, bs)
    t = i32(tables)
    s, n, f, k = i32(start), i32(new), i32(free), i32([taken])
    want = ref.grow(start, new, t.cpu().numpy(), free, taken, bs, num_blocks, capacity, max_position, t.shape[1])
    out = None
    if in_place:
        e = lambda m, dt=torch.int32: torch.full((m,), -77, dtype=dt, device=DEV)  # noqa: E731
        out = GrownBlocks(e(len(start) + 1), s, e(capacity), e(capacity, torch.int64), k, e(len(start)))
    g = ms.grow_blocks(s, n, t, cache, f, k, capacity, out=out)
    torch.cuda.synchronize()
    assert np.array_equal(t.cpu().numpy(), want[0])
    assert g.q_start.tolist() == want[1] and g.seq_lens.tolist() == want[2]
    assert np.array_equal(g.positions.cpu().numpy(), want[3]) and np.array_equal(g.slots.cpu().numpy(), want[4])
    assert g.n_taken.tolist() == [want[5]] and g.status.tolist() == want[6]
    if not in_place:
        assert s.tolist() == list(start) and k.tolist() == [taken]
    return g


def random_requests(rng, nreq, bs, start_hi, new_hi, width_extra=2):
    start = [rng.randint(0, start_hi) for _ in range(nreq)]
    new = [rng.choice([0, 1, rng.randint(0, new_hi)]) for _ in range(nreq)]
    held = [-(-s // bs) for s in start]
    width = max(-(-(s + n) // bs) for s, n in zip(start, new)) + width_extra
    used = sum(held)
    need = sum(-(-(s + n) // bs) - h for s, n, h in zip(start, new, held))
    ids = list(range(used + need + 7))
    rng.shuffle(ids)
    tables, at = np.full((nreq, width), -1, np.int64), 0
    for r, h in enumerate(held):
        tables[r, :h] = ids[at : at + h]
        at += h
    return start, new, tables, ids[at:], need, len(ids)


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("nreq,bs,start_hi,new_hi", [(1, 16, 0, 1), (1, 16, 40, 3), (7, 1, 9, 5), (100, 16, 300, 2), (33, 24, 100, 700), (1500, 16, 64, 9),
                                                     (40, 128, 5000, 900), (300, 7, 50, 100), (3, 16, 100, 9000)])  # fmt: skip
def test_grow_against_the_sequential_rule(nreq, bs, start_hi, new_hi, in_place):
    rng = random.Random(nreq * 1000 + bs)
    ms = store()
    start, new, tables, free, need, nb = random_requests(rng, nreq, bs, start_hi, new_hi)
    total = sum(new)
    for taken, capacity in ((0, total), (4, total + 37), (7, total + 9000)):
        run_grow(ms, start, new, tables, [0] * taken + free[taken:] if taken else free, taken, bs, nb, capacity, in_place)
    ms.close()


def test_grow_without_enough_blocks_serves_a_prefix_and_whoever_needs_none():
    ms = store()
    bs = 16
    start, new = [16, 15, 0, 3, 30, 0, 16], [17, 1, 40, 2, 1, 1, 0]
    tables = np.full((7, 6), -1, np.int64)
    for r, s in enumerate(start):
        for j in range(-(-s // bs)):
            tables[r, j] = 40 + 3 * r + j
    for n_free in range(0, 8):
        run_grow(ms, start, new, tables, list(range(n_free)), 0, bs, 64, sum(new) + 3)
        run_grow(ms, start, new, tables, list(range(n_free)), min(2, n_free), bs, 64, sum(new))
    for taken in (-1, 9):  # no valid counter: only requests that need nothing
        run_grow(ms, start, new, tables, list(range(8)), taken, bs, 64, sum(new))
    ms.close()


def test_grow_reports_what_it_refuses():
    ms = store(max_position=1000)
    bs = 16
    start, new = [-1, 5, 990, 0, 10, 0, 3, 60], [3, -2, 11, 200, 4, 0, 5, 4]
    tables = np.full((8, 7), -1, np.int64)
    tables[1, 0], tables[4, 0], tables[6, 0] = 3, 99, 4  # request 4 holds a block that the cache does not have
    tables[7, :4] = [5, 6, 7, -5]  # request 7's last, half full block is unknown
    g = run_grow(ms, start, new, tables, [8, 9, 10, 11] + list(range(12, 40)), 0, bs, 40, 1000, max_position=1000)
    assert g.status.tolist() == [64, 256, 16 | 4, 4, 8, 0, 0, 8]
    # the free list names a block outside the cache: that block's tokens are left out
    run_grow(ms, [0, 3], [40, 20], np.array([[-1, -1, -1], [2, -1, -1]]), [5, 1000, 6, -3, 7], 0, bs, 40, 60)
    # tokens behind the capacity of the arrays
    for cap in (0, 1, 39, 40, 41, 59):
        g = run_grow(ms, [0, 3], [40, 20], np.array([[-1, -1, -1], [2, -1, -1]]), [5, 6, 7, 8], 0, bs, 40, cap)
        assert g.status[1].item() == 256
    # no requests at all
    g = run_grow(ms, [], [], np.zeros((0, 3)), [1, 2], 1, bs, 40, 5)
    assert g.q_start.tolist() == [0] and g.slots.tolist() == [-1] * 5
    ms.close()


def test_grow_far_positions_and_sums_behind_32_bits():
    ms = store()
    bs = 16
    top = 1 << 24
    width = top // bs
    tables = np.full((2, width), -1, np.int64)
    tables[0, : width - 1] = np.arange(width - 1) % 100
    run_grow(ms, [top - 20, 0], [20, 1], tables, [7, 8, 9, 10], 0, bs, 100, 32)
    # 300 requests of 2^24 tokens each: their sum is beyond 2^31
    run_grow(ms, [0] * 300, [top] * 300, np.full((300, 2), -1), [7, 8], 0, bs, 100, 64)
    ms.close()


def test_release_gives_the_blocks_back_and_grow_takes_them_again():
    ms = store()
    bs, nb = 16, 64
    cache = geometry(nb, bs)
    tables = i32(np.full((4, 8), -1))
    free, taken = i32(np.random.default_rng(0).permutation(nb)), i32([0])
    lens = i32([0, 0, 0, 0])
    g = ms.grow_blocks(lens, i32([100, 1, 0, 33]), tables, cache, free, taken, 200)
    held = {r: [b for b in tables[r].tolist() if b >= 0] for r in range(4)}
    assert [len(held[r]) for r in range(4)] == [7, 1, 0, 3] and g.n_taken.item() == 11
    before = free.clone()
    status = i32([-1] * 4)
    lens, taken = g.seq_lens, g.n_taken
    ms.release_blocks(lens, tables, cache, free, taken, release=i32([1, 0, 1, 7]), out_status=status)
    assert taken.item() == 1 and lens.tolist() == [0, 1, 0, 0] and status.tolist() == [0, 0, 0, 0]
    assert (tables[0] == -1).all() and (tables[3] == -1).all() and tables[1].tolist() == [held[1][0]] + [-1] * 7
    assert free[4:11].tolist() == held[0] and free[1:4].tolist() == held[3] and free[11:].tolist() == before[11:].tolist()
    g = ms.grow_blocks(lens, i32([160, 16, 16, 16]), tables, cache, free, taken, 300)  # everything that is free is handed out once
    used = [b for b in tables.flatten().tolist() if b >= 0]
    assert g.status.tolist() == [4, 0, 0, 0]  # ten blocks do not fit the table
    assert len(set(used)) == len(used) == 4
    # blocks that the cache does not have are dropped, requests without room keep theirs
    tables = i32([[1, 99, 2, -1], [3, 4, 5, -1], [6, -1, -1, -1], [-1, -1, -1, -1]])
    lens, taken, free = i32([40, 48, 1, 0]), i32([3]), i32([0] * 6)
    ms.release_blocks(lens, tables, cache, free, taken, out_status=status)
    assert status.tolist() == [8, 128, 128, 0] and lens.tolist() == [0, 48, 1, 0] and taken.item() == 1 and free.tolist() == [0, 1, 2, 0, 0, 0]
    assert tables.tolist() == [[-1, -1, -1, -1], [3, 4, 5, -1], [6, -1, -1, -1], [-1] * 4]
    ms.close()


# ------------------------------------------------------------------------------------------------ append
@pytest.mark.parametrize("d,hq,hk,rotary,style,fp8,layout", [
    (64, 4, 2, 0, 0, False, "NHD"), (128, 32, 8, 0, 0, False, "HND"), (128, 5, 1, 64, 1, True, "NHD"), (256, 3, 3, 0, 1, False, "NHD"),
    (16, 6, 2, 0, 0, True, "HND"), (32, 8, 8, 16, 0, False, "NHD"), (128, 40, 8, 0, 0, True, "NHD"), (64, 0, 2, 0, 1, False, "HND")])  # fmt: skip
@pytest.mark.parametrize("T", [1, 37])
def test_append_rotates_and_writes(d, hq, hk, rotary, style, fp8, layout, T):
    theta, bs, nb, L = 5.0e5, 16, 12, 2
    ms = store(hk, d, L, rope_theta=theta, rope_style=style, rotary_dim=rotary)
    R = rotary or d
    freq = (theta ** (-2.0 * np.arange(R // 2) / R)).astype(np.float32)
    gen = torch.Generator(device=DEV).manual_seed(T * d)
    cache = PagedCache.allocate(L, nb, bs, hk, d, DEV, layout=layout, fill_bits=0x5A if fp8 else 0xC2F2, fp8=fp8, k_scale=0.03, v_scale=0.9)
    qkv = torch.randn((T, (hq + 2 * hk) * d + 8), generator=gen, device=DEV, dtype=torch.bfloat16)  # rows of a fused projection, padded
    q = qkv[:, : hq * d].unflatten(1, (hq, d)) if hq else None
    k, v = (qkv[:, (hq + i * hk) * d : (hq + (i + 1) * hk) * d].unflatten(1, (hk, d)) for i in (0, 1))
    positions = torch.randint(0, 1 << 24, (T,), generator=gen, device=DEV, dtype=torch.int32)
    slots = torch.randperm(nb * bs, generator=gen, device=DEV)[:T]
    status = i32([-9] * T)
    bad = {}
    if T > 8:
        positions[1], positions[2], slots[3], slots[4], slots[5] = -1, 1 << 24, -1, nb * bs, 1 << 40
        bad = {1: 64, 2: 16, 3: 8, 4: 8, 5: 8}
    q_out = torch.full((T, hq, d), 7.0, dtype=torch.bfloat16, device=DEV) if hq else None
    before = [x.clone() for x in (cache.k, cache.v)]
    r = ms.append(1, q, k, v, positions, slots, cache, q_out=q_out, out_status=status)
    torch.cuda.synchronize()
    assert (r is q_out) and status.tolist() == [bad.get(i, 0) for i in range(T)]
    live = torch.tensor([bad.get(i, 0) in (0, 8) for i in range(T)], device=DEV)
    stay = torch.tensor([i not in bad for i in range(T)], device=DEV)

    def near(got, x):  # parity rule of the injection tests: one rounding, fp32 rotation
        want = ref.rotate(x, positions, freq, R, style == 1)
        norm = torch.sqrt(want[..., :R].square().sum(-1, keepdim=True)) if R else 0.0
        assert ((got.double() - want).abs() <= 2.0**-7 * torch.maximum(want.abs(), 2.0**-10 * norm)).all()

    if hq:
        assert (q_out[~live] == 7.0).all()
        near(q_out[live], q[live]) if live.all() else near_masked(q_out, q, positions, freq, R, style, live)
    planes = [x[1].transpose(1, 2) if layout == "HND" else x[1] for x in (cache.k, cache.v)]
    old = [x[1].transpose(1, 2) if layout == "HND" else x[1] for x in before]
    blk, off = slots.clamp(0, nb * bs - 1) // bs, slots.clamp(0, nb * bs - 1) % bs
    gk, gv = planes[0][blk, off], planes[1][blk, off]
    if fp8:  # byte for byte what the rule makes of the bf16 value
        kb = ms_rotated_bf16(ms, k, positions, slots, L, nb, bs, hk, d)
        assert torch.equal(gk[stay], e4m3(kb, 0.03)[stay])
        assert torch.equal(gv[stay], e4m3(v, 0.9)[stay])
    else:
        near_masked(gk, k, positions, freq, R, style, stay)
        assert torch.equal(gv[stay], v[stay])
    # nothing else was written
    for new, was, vals in ((planes[0], old[0], gk), (planes[1], old[1], gv)):
        expect = was.clone()
        expect[blk[stay], off[stay]] = vals[stay]
        assert torch.equal(new, expect)
    for x, y in zip((cache.k, cache.v), before):
        assert torch.equal(x[0], y[0])
    if hq:  # in place
        q2 = q.clone() if q.is_contiguous() else q
        want = q_out.clone()
        want[~live] = q2[~live]
        assert ms.append(1, q2, k, v, positions, slots, cache, q_out=q2) is q2
        assert torch.equal(q2, want)
    ms.close()


def e4m3(x, scale):
    """Codes of x / scale with IEEE division (torch multiplies by the reciprocal when the divisor is a scalar: another quotient for some values)."""
    return (x.float() / torch.full(x.shape, scale, device=x.device)).clamp(-448, 448).to(ref.F8).view(torch.uint8)


def near_masked(got, x, positions, freq, R, style, keep):
    want = ref.rotate(x, positions, freq, R, style == 1)[keep]
    norm = torch.sqrt(want[..., :R].square().sum(-1, keepdim=True))
    assert ((got[keep].double() - want).abs() <= 2.0**-7 * torch.maximum(want.abs(), 2.0**-10 * norm)).all()


def ms_rotated_bf16(ms, k, positions, slots, L, nb, bs, hk, d):
    """The same keys appended to a bf16 cache."""
    c = PagedCache.allocate(L, nb, bs, hk, d, DEV)
    ms.append(1, None, k, k, positions, slots, c)
    s = slots.clamp(0, nb * bs - 1)
    return c.k[1][s // bs, s % bs]


@pytest.mark.parametrize("fp8", [False, True])
def test_append_writes_the_bytes_of_an_injection(fp8):
    """A fact injected at a position and the same keys and values appended there leave identical caches."""
    L, hk, d, n, bs, nb, start = 2, 2, 128, 50, 16, 8, 77
    ms = MemStore(n_layers=L, n_kv_heads=hk, head_dim=d, emb_dim=64, max_facts_per_user=2, max_kv_tokens=64, rope_theta=5.0e5)
    k, v = (torch.randn((L, n, hk, d), device=DEV).to(torch.bfloat16) for _ in range(2))
    fid = ms.add_fact(torch.randn(64, device=DEV).half(), k, v)
    caches = [PagedCache.allocate(L, nb, bs, hk, d, DEV, fill_bits=3, fp8=fp8, k_scale=0.011, v_scale=0.007) for _ in range(2)]
    table = i32([[5, 0, 3, 7, 1, 2, 6, 4]])
    ms.inject(i32([[fid]]), i32([start]), table, caches[0])
    g = ms.grow_blocks(i32([start]), i32([n]), i32(np.pad(table.cpu().numpy()[:, :5], ((0, 0), (0, 3)))), caches[1], i32([2, 6, 4]), i32([0]), n)
    for layer in range(L):
        ms.append(layer, None, k[layer], v[layer], g.positions, g.slots, caches[1])
    torch.cuda.synchronize()
    assert torch.equal(caches[0].k.view(torch.uint8), caches[1].k.view(torch.uint8)) and torch.equal(caches[0].v.view(torch.uint8), caches[1].v.view(torch.uint8))
    ms.close()


# ------------------------------------------------------------------------------------------------ attention
def fill_cache(L, nb, bs, hk, d, fp8, layout, seed, k_scale=0.02, v_scale=0.03):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    cache = PagedCache.allocate(L, nb, bs, hk, d, DEV, layout=layout, fp8=fp8, k_scale=k_scale, v_scale=v_scale)
    for t, s in ((cache.k, k_scale), (cache.v, v_scale)):
        x = torch.randn(t.shape, generator=gen, device=DEV)
        t.copy_((x / s).clamp(-448, 448).to(ref.F8).view(torch.uint8) if fp8 else x.to(torch.bfloat16))
    return cache, gen


def check_attend(ms, cache, q, q_start, lens, tables, layer=0, scale=0.0, max_q_len=0, want_status=None, **kw):
    T, hq, d = q.shape
    out = torch.full((T, hq, d), 9.0, dtype=torch.bfloat16, device=DEV)
    lse = torch.full((T, hq), 9.0, device=DEV)
    status = i32([-5] * len(lens))
    ms.attend(layer, q, cache, i32(q_start), i32(lens), tables, scale=scale, max_q_len=max_q_len, out=out, out_lse=lse, out_status=status, **kw)
    torch.cuda.synchronize()
    sc = scale or 1.0 / math.sqrt(d)
    want, wl, tol, ltol = ref.attend(q, cache, layer, q_start, lens, tables, ms.n_kv_heads, sc, 9.0)
    fin = torch.isfinite(want)
    assert torch.equal(torch.isfinite(out.double()), fin) and torch.equal(torch.isnan(out.double()), torch.isnan(want))
    err = torch.where(fin, (out.double() - torch.where(fin, want, 0.0)).abs() - tol, 0.0)
    assert (err <= 0).all(), f"out: worst excess {err.max().item()} at {np.unravel_index(err.argmax().item(), err.shape)}"
    lf = torch.isfinite(wl)
    assert torch.equal(lse.double()[~lf], wl[~lf]) or torch.isnan(wl[~lf]).any()
    le = torch.where(lf, (lse.double() - torch.where(lf, wl, 0.0)).abs() - ltol, 0.0)
    assert (le <= 0).all(), f"lse: worst excess {le.max().item()}"
    assert status.tolist() == (want_status or [0] * len(lens))
    return out, lse


def paged(rng, lens, bs, extra_blocks=3, width_extra=2):
    need = [-(-max(n, 0) // bs) for n in lens]
    nb = sum(need) + extra_blocks
    ids = list(range(nb))
    rng.shuffle(ids)
    t = np.full((len(lens), max(need + [0]) + width_extra), -1, np.int64)
    at = 0
    for r, n in enumerate(need):
        t[r, :n] = ids[at : at + n]
        at += n
    return i32(t), nb


def random_case(rng, nreq, q_hi, len_hi):
    q = [rng.choice([1, 1, rng.randint(0, q_hi)]) for _ in range(nreq)]
    lens = [max(rng.randint(0, len_hi), n) for n in q]
    return [0] + list(np.cumsum(q)), lens


ATTEND_SHAPES = [
    # d, heads, kv heads, block size, 8-bit, layout
    (64, 4, 2, 16, False, "NHD"), (128, 32, 8, 16, False, "NHD"), (128, 40, 8, 32, False, "HND"), (128, 8, 8, 16, True, "NHD"),
    (64, 14, 2, 64, True, "HND"), (16, 2, 1, 16, False, "NHD"), (32, 3, 1, 8, False, "NHD"), (256, 8, 2, 16, False, "NHD"),
    (256, 4, 4, 16, True, "NHD"), (32, 4, 4, 16, True, "HND"), (16, 33, 3, 5, True, "NHD"), (128, 16, 1, 24, False, "NHD"),
    (64, 20, 1, 1, False, "HND"), (128, 7, 1, 128, True, "NHD")]  # fmt: skip


@pytest.mark.parametrize("d,hq,hk,bs,fp8,layout", ATTEND_SHAPES)
@pytest.mark.parametrize("nreq,q_hi,len_hi", [(1, 1, 1), (5, 1, 700), (6, 40, 333), (3, 300, 900)])
def test_attend_against_the_definition(d, hq, hk, bs, fp8, layout, nreq, q_hi, len_hi):
    rng = random.Random(d * 7 + hq + nreq)
    q_start, lens = random_case(rng, nreq, q_hi, len_hi)
    tables, nb = paged(rng, lens, bs)
    cache, gen = fill_cache(2, nb, bs, hk, d, fp8, layout, nreq)
    ms = store(hk, d, 2)
    q = (2.0 * torch.randn((q_start[-1] + 3, hq, d), generator=gen, device=DEV)).to(torch.bfloat16)  # rows behind the last request too
    check_attend(ms, cache, q, q_start, lens, tables, layer=1)
    check_attend(ms, cache, q, q_start, lens, tables, layer=1, scale=0.9, max_q_len=max(np.diff(q_start)))
    ms.close()


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("len_", [1, 15, 16, 17, 63, 64, 65, 127, 128, 129, 4095, 20001])
@pytest.mark.parametrize("n", [1, 2, 5])
def test_attend_lengths_around_tile_borders(fp8, len_, n):
    hk, d, hq = 2, 128, 8
    tables, nb = paged(random.Random(len_), [len_], 16)
    cache, gen = fill_cache(1, nb, 16, hk, d, fp8, "NHD", len_)
    ms = store(hk, d)
    q = torch.randn((n, hq, d), generator=gen, device=DEV).to(torch.bfloat16)
    check_attend(ms, cache, q, [0, n], [len_], tables)  # n > len_: the first rows have no keys
    ms.close()


@pytest.mark.parametrize("fp8,d", [(False, 64), (True, 64), (False, 128), (True, 128)])
@pytest.mark.parametrize("seed", range(6))
def test_attend_random_batches(fp8, d, seed):
    """Seeded batches of chunks and single tokens: many and few units, group sizes that divide 256 and that do not, pages of any size,
    units that several CTAs share."""
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
    check_attend(ms, cache, x, q_start, lens, tables, max_q_len=rng.choice([0, max(q), 1]))  # (the bound may be wrong)
    ms.close()


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("n,len_", [(200, 150), (300, 0), (130, 129), (64, 1), (40, 40), (700, 3), (65, 128), (257, 129)])
def test_attend_chunks_whose_first_rows_have_no_keys(fp8, n, len_):
    hk, d, hq = 2, 128, 8
    tables, nb = paged(random.Random(n), [len_], 16)
    cache, gen = fill_cache(1, nb, 16, hk, d, fp8, "NHD", n)
    ms = store(hk, d)
    q = torch.randn((n, hq, d), generator=gen, device=DEV).to(torch.bfloat16)
    out, lse = check_attend(ms, cache, q, [0, n], [len_], tables)
    assert (out[: max(0, n - len_)] == 0).all() and (lse[: max(0, n - len_)] == -math.inf).all()
    ms.close()


def test_attend_chunks_over_tables_with_holes():
    bs, lens, q_start = 16, [700, 500, 300], [0, 90, 290, 300]
    tables, nb = paged(random.Random(6), lens, bs, width_extra=0)
    tables[0, 3], tables[0, 40], tables[1, 31], tables[1, 0] = -1, nb, nb + 5, -(2**31)
    short = tables[:, :40].contiguous()  # request 0 has 44 blocks
    cache, gen = fill_cache(1, nb, bs, 2, 128, False, "NHD", 6)
    ms = store(2, 128)
    q = torch.randn((300, 8, 128), generator=gen, device=DEV).to(torch.bfloat16)
    check_attend(ms, cache, q, q_start, lens, tables, want_status=[8, 8, 0])
    check_attend(ms, cache, q, q_start, lens, short, want_status=[12, 8, 0])
    ms.close()


def test_attend_scores_that_grow_along_the_keys():
    """Every tile raises the running maximum (by far more than the weights' slack), or lowers it: accumulators are rescaled each time."""
    n, len_, hk, d = 70, 1500, 1, 128
    for fp8 in (False, True):
        for sign in (1.0, -1.0):
            tables, nb = paged(random.Random(8), [len_], 16)
            cache, gen = fill_cache(1, nb, 16, hk, d, fp8, "NHD", 3, k_scale=1.0, v_scale=0.03)
            q = torch.zeros((n, 4, d), device=DEV)
            q[..., 0] = 1.0 + torch.arange(n, device=DEV)[:, None] / n
            for j in range(len_):
                blk, off = int(tables[0, j // 16]), j % 16
                val = round(sign * (j - 750) / 4.0)
                k = torch.zeros(d, device=DEV)
                k[0] = val
                cache.k[0, blk, off, 0] = k.to(ref.F8).view(torch.uint8) if fp8 else k.to(torch.bfloat16)
            ms = store(hk, d)
            check_attend(ms, cache, q.to(torch.bfloat16), [0, n], [len_], tables, scale=1.0)
            check_attend(ms, cache, q[:2].to(torch.bfloat16), [0, 2], [len_], tables, scale=1.0)
            ms.close()


def test_attend_reports_a_wait_that_ran_out_and_works_again():
    """The chunk kernel's loading role issues nothing and every wait gives up after a few thousand polls: the call returns, the status
    says so, and the next call is right."""
    lens, q_start = [700, 50], [0, 100, 101]
    tables, nb = paged(random.Random(9), lens, 16)
    cache, gen = fill_cache(1, nb, 16, 2, 128, False, "NHD", 9)
    ms = store(2, 128)
    q = torch.randn((101, 8, 128), generator=gen, device=DEV).to(torch.bfloat16)
    status = i32([0, 0])
    ms.test_hooks(wait_poll_limit=3000, mute_producers=True)
    ms.attend(0, q, cache, i32(q_start), i32(lens), tables, out_status=status)
    torch.cuda.synchronize()
    assert status.tolist() == [32, 0]  # (the single token is served by the other kernel)
    ms.test_hooks()
    check_attend(ms, cache, q, q_start, lens, tables)
    ms.close()


def test_attend_many_requests_and_empty_ones():
    rng = random.Random(3)
    q_start, lens = random_case(rng, 700, 3, 90)
    lens = [0 if rng.random() < 0.1 else n for n in lens]  # rows without any key
    tables, nb = paged(rng, lens, 16)
    cache, gen = fill_cache(1, nb, 16, 2, 64, False, "NHD", 1)
    ms = store(2, 64)
    q = torch.randn((q_start[-1], 6, 64), generator=gen, device=DEV).to(torch.bfloat16)
    check_attend(ms, cache, q, q_start, lens, tables)
    ms.close()


def poison(cache, tables, lens, bs, codes=(0x7FC0, 0x7F80, 0xFF80)):
    """NaN and infinities in every cache row that no request's tokens use."""
    used = set()
    for r, n in enumerate(lens):
        for j in range(n):
            used.add(int(tables[r, j // bs]) * bs + j % bs)
    dead = torch.tensor([i for i in range(cache.num_blocks * bs) if i not in used], device=DEV)
    for t in (cache.k, cache.v):
        p = t[0].transpose(1, 2) if cache.layout == "HND" else t[0]
        bits = p.view(torch.int16) if not cache.fp8 else p
        for i, c in enumerate(codes):
            d = dead[i :: len(codes)]
            bits[d // bs, d % bs] = 0x7F if cache.fp8 else (c - 0x10000 if c >= 0x8000 else c)


@pytest.mark.parametrize("fp8,layout", [(False, "NHD"), (True, "HND")])
@pytest.mark.parametrize("d", [64, 128])
def test_attend_never_sees_what_lies_behind_the_last_key(fp8, layout, d):
    lens, q_start = [5, 100, 31, 257], [0, 2, 42, 43, 300]
    tables, nb = paged(random.Random(1), lens, 16)
    tables[tables < 0] = 0  # entries behind the last block name a real block
    cache, gen = fill_cache(1, nb, 16, 2, d, fp8, layout, 4)
    poison(cache, tables.cpu().numpy(), lens, 16)
    ms = store(2, d)
    q = torch.randn((300, 8, d), generator=gen, device=DEV).to(torch.bfloat16)
    out, lse = check_attend(ms, cache, q, q_start, lens, tables)
    assert torch.isfinite(out).all() and torch.isfinite(lse).all()
    ms.close()


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("d,n", [(128, 3), (128, 200), (64, 130), (256, 9)])
def test_attend_later_tokens_that_are_not_finite_do_not_reach_earlier_rows(fp8, d, n):
    """NaN and infinities in keys and values of a chunk's later tokens: earlier rows stay as they are, later rows get them."""
    bs, hk, hq, len_ = 16, 2, 4, 40 + n
    tables, nb = paged(random.Random(n), [len_], bs)
    cache, gen = fill_cache(1, nb, bs, hk, d, fp8, "NHD", 9)
    nan, inf = (0x7F, 0x7F) if fp8 else (0x7FC0, 0x7F80)
    for tok, head, plane, col, code in ((40 + n - 1, 0, 1, 3, inf), (40 + n // 2, 1, 1, 5, nan), (40 + n // 2, 1, 0, 7, nan)):
        t = (cache.k, cache.v)[plane][0]
        t = t if fp8 else t.view(torch.int16)
        t[tables[0, tok // bs].long(), tok % bs, head, col] = code
    ms = store(hk, d)
    q = torch.randn((n, hq, d), generator=gen, device=DEV).to(torch.bfloat16)
    check_attend(ms, cache, q, [0, n], [len_], tables)
    ms.close()


def test_attend_rows_with_extreme_queries():
    """A NaN row, an infinite one and rows of the largest and smallest values stand beside ordinary ones."""
    for fp8 in (False, True):
        tables, nb = paged(random.Random(2), [300], 16)
        cache, gen = fill_cache(1, nb, 16, 1, 128, fp8, "NHD", 5)
        ms = store(1, 128)
        q = torch.randn((9, 4, 128), generator=gen, device=DEV).to(torch.bfloat16)
        clean, _, _ = ms.attend(0, q, cache, i32([0, 9]), i32([300]), tables)
        x = q.clone()
        x[1, 0, 3], x[2, 1, 5], x[3, 2], x[4, 3] = math.nan, math.inf, 1e-38, 0.0
        out, lse, _ = ms.attend(0, x, cache, i32([0, 9]), i32([300]), tables, want_lse=True)
        assert torch.isnan(out[1, 0]).all() and torch.isnan(out[2, 1]).all()
        same = torch.ones((9, 4), dtype=torch.bool, device=DEV)
        for a, b in ((1, 0), (2, 1), (3, 2), (4, 3)):
            same[a, b] = False
        assert torch.equal(out[same], clean[same])
        assert abs(lse[4, 3].item() - math.log(296)) < 1e-5 and abs(lse[3, 2].item() - math.log(295)) < 1e-5  # all weights alike
        ms.close()


def test_attend_tables_that_do_not_name_every_block():
    bs = 16
    lens, q_start = [100, 80, 64, 33, -3, 20], [0, 3, 4, 5, 6, 7, 9]
    tables, nb = paged(random.Random(5), [100, 80, 64, 33, 0, 20], bs, width_extra=0)
    t = tables[:, :5].contiguous()  # request 0 needs seven blocks
    t[1, 2], t[1, 4], t[2, 0] = nb, -7, 2**30
    t[3, :] = -1
    cache, gen = fill_cache(1, nb, bs, 2, 64, False, "NHD", 6)
    ms = store(2, 64)
    q = torch.randn((9, 4, 64), generator=gen, device=DEV).to(torch.bfloat16)
    out, lse = check_attend(ms, cache, q, q_start, lens, t, want_status=[4, 8, 8, 8, 256, 0])
    assert (out[5] == 0).all() and (lse[5] == -math.inf).all()  # no key is left
    # ranges that are no ranges: that request's rows stay as they were
    status = i32([0] * 3)
    out = torch.full((9, 4, 64), 9.0, dtype=torch.bfloat16, device=DEV)
    ms.attend(0, q, cache, i32([4, 2, 5, 12]), i32([50, 20, 20]), t[:3], out=out, out_status=status)
    assert status.tolist() == [256, 0, 256]  # (20 tokens need the first two blocks of request 1, which are good)
    assert (out[:2] == 9).all() and (out[5:] == 9).all() and not (out[2:5] == 9).any()
    # no blocks at all
    out, lse, _ = ms.attend(0, q, cache, i32([0, 9]), i32([20]), torch.empty((1, 0), dtype=torch.int32, device=DEV), want_lse=True)
    assert (out == 0).all() and (lse == -math.inf).all()
    ms.close()


def test_attend_strided_queries_and_outputs_in_place():
    bs, hk, hq, d = 16, 2, 6, 128
    lens, q_start = [50, 700], [0, 1, 30]
    tables, nb = paged(random.Random(7), lens, bs)
    cache, gen = fill_cache(1, nb, bs, hk, d, False, "HND", 7)
    ms = store(hk, d)
    qkv = torch.randn((30, (hq + 2 * hk) * d + 8), generator=gen, device=DEV).to(torch.bfloat16)
    q = qkv[:, : hq * d].unflatten(1, (hq, d))
    want, _, _ = ms.attend(0, q.contiguous(), cache, i32(q_start), i32(lens), tables)
    head_major = torch.empty((hq, 30, d), dtype=torch.bfloat16, device=DEV).transpose(0, 1)
    ms.attend(0, q, cache, i32(q_start), i32(lens), tables, out=head_major)
    assert torch.equal(head_major, want)
    rest = qkv[:, hq * d :].clone()
    ms.attend(0, q, cache, i32(q_start), i32(lens), tables, out=q)  # in place, inside the projection's rows
    assert torch.equal(q, want) and torch.equal(qkv[:, hq * d :], rest)
    ms.close()


def test_attend_a_cache_plane_beyond_32_bits():
    """Blocks more than 2^32 elements into the cache."""
    hk, d, bs = 1, 128, 16
    nb = (1 << 32) // (bs * d) + 40  # 2^32 elements and a little, 8.6 GB a plane
    cache = PagedCache.allocate(1, nb, bs, hk, d, DEV)
    blocks = [nb - 1, 0, nb - 30, 5, nb - 17]
    gen = torch.Generator(device=DEV).manual_seed(0)
    small = PagedCache.allocate(1, 5, bs, hk, d, DEV)
    for t, u in ((cache.k, small.k), (cache.v, small.v)):
        u.copy_(torch.randn(u.shape, generator=gen, device=DEV))
        t[0, torch.tensor(blocks, device=DEV)] = u[0]
    ms = store(hk, d)
    for n in (2, 70):
        q = torch.randn((n, 4, d), generator=gen, device=DEV).to(torch.bfloat16)
        a, _, _ = ms.attend(0, q, cache, i32([0, n]), i32([79]), i32([blocks]))
        b, _, _ = ms.attend(0, q, small, i32([0, n]), i32([79]), i32([[0, 1, 2, 3, 4]]))
        assert torch.equal(a, b)
    pos = i32([0, 1])
    ms.append(0, None, small.k[0, 0, :2], small.v[0, 0, :2], pos, torch.tensor([nb * bs - 1, nb * bs - 500], device=DEV), cache)
    torch.cuda.synchronize()
    assert torch.equal(cache.v[0, nb - 1, bs - 1], small.v[0, 0, 0])
    ms.close()


def test_attend_is_the_same_on_every_run_and_on_other_streams():
    rng = random.Random(11)
    q_start, lens = random_case(rng, 40, 70, 3000)
    tables, nb = paged(rng, lens, 16)
    cache, gen = fill_cache(1, nb, 16, 4, 128, False, "NHD", 11)
    ms = store(4, 128)
    q = torch.randn((q_start[-1], 16, 128), generator=gen, device=DEV).to(torch.bfloat16)
    qs, ln = i32(q_start), i32(lens)
    first, l1, _ = ms.attend(0, q, cache, qs, ln, tables, want_lse=True)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    outs = []
    for rep in range(4):
        for st in streams:
            outs.append(ms.attend(0, q, cache, qs, ln, tables, want_lse=True, stream=st))
    torch.cuda.synchronize()
    for o, l, _ in outs:
        assert torch.equal(o, first) and torch.equal(l, l1)
    ms.close()


# ------------------------------------------------------------------------------------------------ the calls as a serving loop makes them
@pytest.mark.parametrize("fp8", [False, True])
def test_a_serving_loop_from_injection_to_release(fp8):
    """Facts are injected, the question is appended and attended to, tokens follow one by one, the blocks go back; every step's
    attention is compared with the definition on what the cache holds."""
    L, hk, hq, d, bs, nb = 2, 2, 8, 64, 16, 64
    ms = MemStore(n_layers=L, n_kv_heads=hk, head_dim=d, emb_dim=64, max_facts_per_user=8, max_kv_tokens=400, rope_theta=1.0e4)
    gen = torch.Generator(device=DEV).manual_seed(0)
    bf = lambda *shape: torch.randn(shape, generator=gen, device=DEV).to(torch.bfloat16)  # noqa: E731
    emb = torch.nn.functional.normalize(torch.randn((8, 64), generator=gen, device=DEV), dim=1).half()
    ms.add_facts(emb, [40] * 8, bf(L, 320, hk, d), bf(L, 320, hk, d))
    cache = PagedCache.allocate(L, nb, bs, hk, d, DEV, fp8=fp8, k_scale=0.02, v_scale=0.02)
    for t in (cache.k, cache.v):
        t.view(torch.uint8).fill_(0x7F)  # NaN wherever nothing was written
    free, taken = i32(np.random.default_rng(1).permutation(nb)), i32([0])
    tables, lens = i32(np.full((3, 20), -1)), i32([0, 0, 0])
    # blocks for the facts (two, three and no facts), then their injection
    g = ms.grow_blocks(lens, i32([80, 120, 0]), tables, cache, free, taken, 200)
    ids = i32([[0, 1, -1], [2, 3, 4], [-1, -1, -1]])
    ms.inject(ids, i32([0, 0, 0]), tables, cache)
    lens, taken = g.seq_lens, g.n_taken
    for step, new in enumerate(([7, 33, 5], [1, 1, 1], [1, 0, 1], [1, 1, 1])):
        T = sum(new) + 2  # padded as in a captured step
        g = ms.grow_blocks(lens, i32(new), tables, cache, free, taken, T)
        assert g.status.tolist() == [0, 0, 0]
        for layer in range(L):
            q, k, v = bf(T, hq, d), bf(T, hk, d), bf(T, hk, d)
            ms.append(layer, q, k, v, g.positions, g.slots, cache, q_out=q)
            check_attend(ms, cache, q, g.q_start.tolist(), g.seq_lens.tolist(), tables, layer=layer, max_q_len=max(new))
        lens, taken = g.seq_lens, g.n_taken
    assert lens.tolist() == [90, 155, 8]
    ms.release_blocks(lens, tables, cache, free, taken)
    torch.cuda.synchronize()
    assert taken.item() == 0 and sorted(free.tolist()) == list(range(nb)) and (tables == -1).all()
    ms.close()


def test_a_decode_step_in_a_graph_replayed_between_eager_calls():
    """grow -> append -> attend captured once, with its state updated in place; two graphs of one store share nothing."""
    hk, hq, d, bs, nb, nreq = 2, 8, 128, 16, 200, 5
    ms = store(hk, d)
    gen = torch.Generator(device=DEV).manual_seed(3)

    def make():
        cache = PagedCache.allocate(1, nb, bs, hk, d, DEV)
        for t in (cache.k, cache.v):
            t.zero_()
        s = {"cache": cache, "tables": i32(np.full((nreq, 30), -1)), "lens": i32([0] * nreq), "free": i32(np.arange(nb)), "taken": i32([0]),
             "new": i32([100, 3, 0, 17, 200]), "q": torch.randn((320, hq, d), generator=gen, device=DEV).to(torch.bfloat16),
             "k": torch.randn((320, hk, d), generator=gen, device=DEV).to(torch.bfloat16)}  # fmt: skip
        e = lambda m, dt=torch.int32: torch.empty((m,), dtype=dt, device=DEV)  # noqa: E731
        s["g"] = GrownBlocks(e(nreq + 1), s["lens"], e(320), e(320, torch.int64), s["taken"], e(nreq))
        s["out"] = torch.zeros((320, hq, d), dtype=torch.bfloat16, device=DEV)
        s["qr"] = torch.empty_like(s["q"])
        return s

    def step(s):
        g = ms.grow_blocks(s["lens"], s["new"], s["tables"], s["cache"], s["free"], s["taken"], 320, out=s["g"])
        ms.append(0, s["q"], s["k"], s["k"], g.positions, g.slots, s["cache"], q_out=s["qr"])
        ms.attend(0, s["qr"], s["cache"], g.q_start, g.seq_lens, s["tables"], out=s["out"])

    a, b = make(), make()
    graphs = []
    for s in (a, b):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step(s)
        graphs.append(graph)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    news = ([100, 3, 0, 17, 200], [1, 1, 1, 1, 1], [1, 20, 1, 0, 1])
    for new in news:
        for s in (a, b):
            s["new"].copy_(i32(new))
        torch.cuda.synchronize()
        for graph, st in zip(graphs, streams):  # both at once
            with torch.cuda.stream(st):
                graph.replay()
        torch.cuda.synchronize()
    eager = [make(), make()]
    for s, e in zip((a, b), eager):
        e["q"], e["k"] = s["q"], s["k"]
        for new in news:
            e["new"].copy_(i32(new))
            step(e)
        torch.cuda.synchronize()
        n = int(s["g"].q_start[-1])
        for name in ("lens", "taken", "tables"):
            assert torch.equal(s[name], e[name])
        assert torch.equal(s["out"][:n], e["out"][:n]) and torch.equal(s["cache"].k, e["cache"].k)
    ms.close()


# ------------------------------------------------------------------------------------------------ refusals
def test_refusals():
    ms = store(2, 64, 2)
    cache = PagedCache.allocate(2, 4, 16, 2, 64, DEV)
    q, k = torch.zeros((3, 4, 64), dtype=torch.bfloat16, device=DEV), torch.zeros((3, 2, 64), dtype=torch.bfloat16, device=DEV)
    pos, slots = i32([0, 1, 2]), torch.zeros(3, dtype=torch.int64, device=DEV)
    qs, ln, tb = i32([0, 3]), i32([3]), i32([[0]])

    def refused(f, *a, code=1, **kw):
        with pytest.raises(M.MemStoreError) as e:
            f(*a, **kw)
        assert e.value.code == code and str(e.value)

    for layer in (-1, 2):
        refused(ms.append, layer, q, k, k, pos, slots, cache)
        refused(ms.attend, layer, q, cache, qs, ln, tb)
    refused(ms.attend, 0, q[:, :3], cache, qs, ln, tb)  # 3 query heads for 2 K/V heads
    for scale in (-1.0, math.nan, math.inf):
        refused(ms.attend, 0, q, cache, qs, ln, tb, scale=scale)
    refused(ms.attend, 0, q, cache, qs, ln, tb, max_q_len=-1)
    refused(ms.attend, 0, q, cache, qs, ln, tb, workspace=torch.empty(100, dtype=torch.uint8, device=DEV))
    refused(ms.attend, 0, q, cache, qs, ln, tb, out=q[:1].expand(3, 4, 64))
    wide = torch.zeros((3, 4 * 64 + 4), dtype=torch.bfloat16, device=DEV)
    refused(ms.attend, 0, wide[:, : 4 * 64].unflatten(1, (4, 64)), cache, qs, ln, tb)  # rows not 16-byte aligned
    refused(ms.attend, 0, wide[:, 4:].unflatten(1, (4, 64)), cache, qs, ln, tb)
    odd = PagedCache.allocate(2, 4, 16, 2, 64, DEV)
    odd.token_stride = 132
    refused(ms.append, 0, q, k, k, pos, slots, odd)
    refused(ms.attend, 0, q, odd, qs, ln, tb)
    f8 = PagedCache.allocate(2, 4, 16, 2, 64, DEV, fp8=True, k_scale=0.0)
    refused(ms.attend, 0, q, f8, qs, ln, tb)
    f8 = PagedCache.allocate(2, 4, 16, 2, 64, DEV, fp8=True)
    f8.head_stride = 72
    refused(ms.attend, 0, q, f8, qs, ln, tb, code=2)
    refused(ms.grow_blocks, ln, ln, tb, cache, ln, ln, -1, out=GrownBlocks(qs, ln, None, None, ln, ln))
    with pytest.raises(TypeError):
        ms.append(0, q.float(), k, k, pos, slots, cache)
    with pytest.raises(TypeError):
        ms.append(0, q, k, k, pos.long(), slots, cache)
    with pytest.raises(TypeError):
        ms.attend(0, q.cpu(), cache, qs, ln, tb)
    with pytest.raises(ValueError):
        ms.append(0, q, k[:2], k, pos, slots, cache)
    with pytest.raises(ValueError):
        ms.attend(0, q, cache, i32([0, 1, 3]), ln, tb)
    with pytest.raises(ValueError):
        ms.attend(0, q, cache, qs, ln, i32([0]))
    with pytest.raises(ValueError):
        ms.attend(0, q, cache, qs, ln, tb, out=torch.zeros((3, 4, 128), dtype=torch.bfloat16, device=DEV)[..., ::2])
    assert ms.attend(0, q[:0], cache, i32([0, 0]), ln, tb)[0].shape == (0, 4, 64)
    ms.append(0, q[:0], k[:0], k[:0], pos[:0], slots[:0], cache)
    torch.cuda.synchronize()
    ms.close()


def test_counts_that_would_wrap_are_refused():
    """Loops over counts near 2^31 would wrap; such calls are refused before anything is launched."""
    ms = store(2, 64, 2)
    cache = PagedCache.allocate(2, 4, 16, 2, 64, DEV)
    ln, tb, qs, big = i32([3]), i32([[0]]), i32([0, 3]), (1 << 30) + 1
    out, c = GrownBlocks(qs, ln, None, None, ln, ln), cache._struct()
    for capacity in (big, 2**31 - 1):
        with pytest.raises(M.MemStoreError) as e:
            ms.grow_blocks(ln, ln, tb, cache, ln, ln, capacity, out=out)
        assert e.value.code == 2 and "2^30" in str(e.value)
    lib, h, at = ms._lib, ms._h, ln.data_ptr()
    x = M._Heads(torch.zeros(3 * 4 * 64, dtype=torch.bfloat16, device=DEV).data_ptr(), 256, 64)
    work = torch.empty(ms.attend_workspace_bytes(), dtype=torch.uint8, device=DEV)
    assert lib.memstore_release_blocks(h, None, at, 1, at, big, c, at, 1, at, None, 0) == 2
    assert lib.memstore_release_blocks(h, None, at, big, at, 1, c, at, 1, at, None, 0) == 2
    assert lib.memstore_append(h, 0, None, 0, x, x, at, at, big, c, None, None, 0) == 2
    for n_tokens, nreq, blocks in ((big, 1, 1), (big // 2 + 1, 1, 1), (3, big, 1), (3, 1, big)):
        assert lib.memstore_attend(h, 0, x, 4, n_tokens, at, at, nreq, at, blocks, c, 0.0, 0, x, None, None, work.data_ptr(), work.numel(), 0) == 2
    torch.cuda.synchronize()
    ms.close()


@pytest.mark.parametrize("d,hq,hk,fp8", [(128, 8, 2, False), (128, 16, 1, True), (64, 4, 1, False), (64, 20, 4, True)])
@pytest.mark.parametrize("nreq,lens_hi", [(1, 2500), (5, 900), (90, 300)])
def test_attend_rows_on_both_sides_of_the_choice_of_kernels(d, hq, hk, fp8, nreq, lens_hi):
    """Requests of 16, 17, 32, 33 and more rows, in batches that leave SMs without a unit and in batches that do not."""
    rng, group = random.Random(nreq * d + hq), hq // hk
    ns = [rows // group + extra for rows in (16, 32) for extra in (0, 1)] + [1, 64 // group]
    ms = store(hk, d)
    for shift in range(1 if nreq > 1 else len(ns)):
        n = [ns[(r + shift) % len(ns)] for r in range(nreq)]
        lens = [m + rng.randint(0, lens_hi) for m in n]
        tables, nb = paged(rng, lens, 16)
        cache, gen = fill_cache(1, nb, 16, hk, d, fp8, "NHD", nreq)
        q_start = [0] + [int(x) for x in np.cumsum(n)]
        q = torch.randn((q_start[-1], hq, d), generator=gen, device=DEV).to(torch.bfloat16)
        for bound in (0, max(n)):
            check_attend(ms, cache, q, q_start, lens, tables, max_q_len=bound)
    ms.close()


def test_attend_from_two_threads_and_two_graphs_at_once():
    """Calls that overlap on the GPU: two host threads on streams of their own, then two captured graphs replayed side by side."""
    import threading

    rng = random.Random(5)
    ms = store(4, 128)
    work = []
    for i in range(2):
        q_start, lens = random_case(rng, 30, 90, 2500)
        tables, nb = paged(rng, lens, 16)
        cache, gen = fill_cache(1, nb, 16, 4, 128, bool(i), "NHD", 50 + i)
        q = torch.randn((q_start[-1], 16, 128), generator=gen, device=DEV).to(torch.bfloat16)
        a = (0, q, cache, i32(q_start), i32(lens), tables)
        want, lse = check_attend(ms, cache, q, q_start, lens, tables)
        work.append((a, want, lse, torch.cuda.Stream()))
    torch.cuda.synchronize()
    got = [[], []]

    def serve(i):
        a, _, _, st = work[i]
        with torch.cuda.stream(st):
            for _ in range(20):
                got[i].append(ms.attend(*a, want_lse=True))

    threads = [threading.Thread(target=serve, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    for i in range(2):
        assert len(got[i]) == 20 and all(torch.equal(o, work[i][1]) and torch.equal(l, work[i][2]) for o, l, _ in got[i])
    graphs = []
    for a, *_ in work:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out, lse, _ = ms.attend(*a, want_lse=True)
        graphs.append((g, out, lse))
    for _ in range(10):
        for (g, out, lse), w in zip(graphs, work):
            with torch.cuda.stream(w[3]):
                out.zero_()
                g.replay()
    torch.cuda.synchronize()
    for (g, out, lse), w in zip(graphs, work):
        assert torch.equal(out, w[1]) and torch.equal(lse, w[2])
    ms.close()
