"""GPU tests of the serving calls where several things meet: units with and without keys in one CTA's share, long tails of small
weights, scales at the ends of their range, calls back to back on one stream, time-outs that nobody asked about."""
import math
import random

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    import serving_ref as ref
    from paper_2607_27090_b200 import memstore as M
    from test_gpu_serving import DEV, check_attend, fill_cache, i32, paged, store


# ------------------------------------------------------------------------------------------------ units without keys
@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("first,empty", [([(65, 128)], 12), ([(65, 128)], 3), ([(65, 256), (200, 200), (97, 128), (33, 384)], 30)])
def test_attend_chunks_without_keys_behind_chunks_whose_last_tile_every_row_sees(fp8, d, first, empty):
    """Prompts that found no blocks (their rows see no key) beside a chunk whose last unit ends with a tile that all its rows see."""
    hk, hq = 8, 32
    q = [n for n, _ in first] + [1000] * empty
    lens = [n for _, n in first] + [0] * empty
    q_start = [0] + [int(x) for x in np.cumsum(q)]
    tables, nb = paged(random.Random(d), lens, 16)
    cache, gen = fill_cache(1, nb, 16, hk, d, fp8, "NHD", d)
    ms = store(hk, d)
    x = torch.randn((q_start[-1], hq, d), generator=gen, device=DEV).to(torch.bfloat16)
    out, lse = check_attend(ms, cache, x, q_start, lens, tables)
    a = q_start[len(first)]
    assert (out[a:] == 0).all() and (lse[a:] == -math.inf).all()
    ms.close()


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("d", [64, 128])
def test_attend_chunks_without_keys_behind_chunks_with_short_tables(fp8, d):
    """The table ends long before the rows' positions, so that every tile of the unit is one that all rows see."""
    hk, hq, bs = 4, 16, 16
    q, lens = [70, 600, 600, 64, 600, 600, 600, 600], [900, 0, 0, 800, 0, 0, 0, 0]
    q_start = [0] + [int(x) for x in np.cumsum(q)]
    tables, nb = paged(random.Random(d), lens, bs)
    cache, gen = fill_cache(1, nb, bs, hk, d, fp8, "NHD", d + 1)
    ms = store(hk, d)
    x = torch.randn((q_start[-1], hq, d), generator=gen, device=DEV).to(torch.bfloat16)
    for width in (8, 16, 31):
        check_attend(ms, cache, x, q_start, lens, tables[:, :width].contiguous(), want_status=[4, 0, 0, 4, 0, 0, 0, 0])
    ms.close()


@pytest.mark.parametrize("fp8,d", [(False, 64), (True, 64), (False, 128), (True, 128)])
@pytest.mark.parametrize("seed", range(4))
def test_attend_random_batches_with_many_units_without_keys(fp8, d, seed):
    rng = random.Random(7000 + 10 * seed + d + fp8)
    hk = rng.choice([1, 2, 4])
    hq = hk * rng.choice([1, 4, 6, 64 // hk**2])
    q, lens = [], []
    for _ in range(rng.choice([6, 40, 140])):  # (more than 128 requests are located by the whole block)
        n = rng.choice([1, 33, 65, 97, 129, 200])
        q.append(n)
        lens.append(rng.choice([0, 0, 0, 0, n, n + 63, 128 * rng.randint(1, 5)]))
    q_start = [0] + [int(x) for x in np.cumsum(q)]
    tables, nb = paged(rng, lens, 16)
    cache, gen = fill_cache(1, nb, 16, hk, d, fp8, rng.choice(["NHD", "HND"]), seed)
    ms = store(hk, d)
    x = torch.randn((q_start[-1], hq, d), generator=gen, device=DEV).to(torch.bfloat16)
    check_attend(ms, cache, x, q_start, lens, tables)
    ms.close()


def test_attend_two_chunks_with_many_requests_between_them():
    """The unit after the first chunk's last one belongs to the last of 200,000 requests (no tokens in between, then a few); far more are refused."""
    nreq, hk, hq, d, bs, n = 200_000, 2, 8, 128, 128, 700
    cache, gen = fill_cache(1, 12, bs, hk, d, False, "NHD", 1)
    tables = torch.full((nreq, 6), -1, dtype=torch.int32, device=DEV)
    tables[0], tables[-1] = torch.arange(6, device=DEV), torch.arange(6, 12, device=DEV)
    ms = store(hk, d)
    for middle in ({}, {70_000: 1, 70_031: 600, 70_032: 2, 130_000: 40}):
        new = torch.zeros(nreq, dtype=torch.int64)
        new[0] = new[-1] = n
        for r, k in middle.items():
            new[r] = k
            tables[r] = torch.tensor([r % 12, 3, 5, 7, 9, 11], device=DEV)
        lens = i32(torch.where(new > 0, torch.minimum(new + 60, torch.tensor(768)), 0).numpy())
        q_start = torch.cat([torch.zeros(1, dtype=torch.int64), new.cumsum(0)])
        q = torch.randn((int(q_start[-1]), hq, d), generator=gen, device=DEV).to(torch.bfloat16)
        some = sorted([0, nreq - 1, *middle])
        out, _, _ = ms.attend(0, q, cache, q_start.int().cuda(), lens, tables)
        exact, _, tol, _ = ref.attend(q, cache, 0, [0, *new[some].cumsum(0).tolist()], lens[some].tolist(), tables[some], hk, 1.0 / math.sqrt(d), 9.0)
        assert ((out.double() - exact).abs() <= tol).all()
    torch.cuda.synchronize()
    assert ms.stats()["kernel_timeouts"] == 0
    x = M._Heads(q.data_ptr(), hq * d, d)
    work = torch.empty(ms.attend_workspace_bytes(), dtype=torch.uint8, device=DEV)
    at, c = lens.data_ptr(), cache._struct()
    assert ms._lib.memstore_attend(ms._h, 0, x, hq, n, at, at, (1 << 26) + 1, at, 1, c, 0.0, 0, x, None, None, work.data_ptr(), work.numel(), 0) == 2
    ms.close()


# ------------------------------------------------------------------------------------------------ time-outs
@pytest.mark.parametrize("nreq", [1, 2])
def test_attend_counts_a_wait_that_ran_out_when_nobody_asks_for_the_status(nreq):
    q_start, lens = [0, 100, 101][: nreq + 1], [700, 50][:nreq]
    tables, nb = paged(random.Random(9), lens, 16)
    cache, gen = fill_cache(1, nb, 16, 2, 128, False, "NHD", 9)
    ms = store(2, 128)
    q = torch.randn((q_start[-1], 8, 128), generator=gen, device=DEV).to(torch.bfloat16)
    assert ms.stats()["kernel_timeouts"] == 0
    ms.attend(0, q, cache, i32(q_start), i32(lens), tables)
    torch.cuda.synchronize()
    assert ms.stats()["kernel_timeouts"] == 0
    ms.test_hooks(wait_poll_limit=3000, mute_producers=True)
    ms.attend(0, q, cache, i32(q_start), i32(lens), tables)
    torch.cuda.synchronize()
    assert ms.stats()["kernel_timeouts"] == 1
    ms.attend(0, q[-1:], cache, i32([0, 1]), i32([50]), tables[-1:])  # (no kernel with waits of its own: the word stays)
    torch.cuda.synchronize()
    assert ms.stats()["kernel_timeouts"] == 1
    ms.test_hooks()
    assert ms.stats()["kernel_timeouts"] == 0
    check_attend(ms, cache, q, q_start, lens, tables)
    assert ms.stats()["kernel_timeouts"] == 0
    ms.close()


# ------------------------------------------------------------------------------------------------ long tails of small weights
@pytest.mark.parametrize("d,n", [(16, 1), (128, 1), (128, 3), (256, 2), (64, 70), (128, 70), (128, 300)])
@pytest.mark.parametrize("drop", [12.0, 16.6, 18.3])
def test_attend_small_weights_behind_large_ones_count_in_an_8_bit_cache(d, n, drop):
    """Eight keys far above 8,000 others, whose weights are 2^-17 to 2^-26 of theirs: the others decide the output, because the large
    keys' values are zero.  300 requests over the same blocks, so that whole units stay in one CTA.

    Bound: an fp16 weight is off by 2^-11 of itself (2^-12 would do) or, below 2^-14, by 2^-25. The exponents are lifted by 14 in the
    kernel for few rows and by 4 in the one for chunks, so the row's largest weight is at least 2^14 or 2^4, and that is 2^-39 or 2^-29 of
    it a key. Beside it the fp32 errors of a score (ds) and the rounding of the output."""
    hk, hq, bs, len_, nreq = 1, 4, 16, 8000 + n, 300
    tables, nb = paged(random.Random(d + n), [len_], bs)
    cache, gen = fill_cache(1, nb, bs, hk, d, True, "NHD", 3, k_scale=1.0, v_scale=0.03)
    # keys: the first coordinate carries the score, the others are noise that only small elements of q look at
    k = torch.randn((nb, bs, hk, d), generator=gen, device=DEV)
    v = 8.0 + 4.0 * torch.rand((nb, bs, hk, d), generator=gen, device=DEV)
    k[..., 0] = 0.0
    for page in tables[0, :8].tolist():  # (a key of every warp's share of a tile)
        k[page, 5] = 0.0
        k[page, 5, 0, 0] = 16.0
        v[page, 5] = 0.0
    cache.k[0], cache.v[0] = k.to(ref.F8).view(torch.uint8), v.to(ref.F8).view(torch.uint8)
    q = (0.02 * torch.randn((n, hq, d), generator=gen, device=DEV)).to(torch.bfloat16)
    q[..., 0] = drop / 16.0
    ms = store(hk, d)
    out, lse, _ = ms.attend(0, q.repeat(nreq, 1, 1), cache, i32(range(0, n * nreq + 1, n)), i32([len_] * nreq), tables.repeat(nreq, 1), scale=1.0,
                            want_lse=True)  # fmt: skip
    step = 2.0**-29 if n >= 70 else 2.0**-39
    out, lse = out.unflatten(0, (nreq, n)).double(), lse.unflatten(0, (nreq, n)).double()
    kk, vv, _ = ref.cache_rows(cache, 0, tables[0], len_, nb)
    see = torch.arange(len_, device=DEV)[None] <= torch.arange(len_ - n, len_, device=DEV)[:, None]
    for h in range(hq):
        s = torch.where(see, q[:, h].double() @ kk[:, 0].T, -math.inf)
        m = s.amax(1, keepdim=True)
        w = torch.exp(s - m)
        l = w.sum(1, keepdim=True)
        want = (w @ vv[:, 0]) / l
        ds = (q[:, h].double().abs() @ kk[:, 0].abs().T).amax() * (d + 8) * ref.U_F32 + 2.0**-20
        tol = 2.0**-8 * want + (2.0**-11 + 3 * ds) * want + step * (see.double() @ vv[:, 0]) / l
        err = (out[:, :, h] - want).abs().amax(0)
        assert (err <= tol).all(), (h, (err / tol).max().item(), (err / want).max().item())
        want_lse = (m + torch.log(l))[:, 0]
        assert ((lse[:, :, h] - want_lse).abs().amax(0) <= 2 * ds + 4 * ref.U_F32 * want_lse.abs() + 2.0**-20).all()
    ms.close()


# ------------------------------------------------------------------------------------------------ calls back to back
@pytest.mark.parametrize("fp8,d", [(False, 128), (True, 128), (False, 64)])
def test_layers_back_to_back_read_what_the_calls_before_them_wrote(fp8, d):
    """Mixed batches (both attention kernels) layer after layer on one stream, nothing waited for in between: lengths, tables, queries and
    cache rows of a call are written by the calls just before it, into buffers that the call before read.  The same steps with a
    synchronise after every call give the same bits; eagerly and from a replayed graph."""
    L, hk, hq, bs, steps = 4, 4, 16, 16, 3
    rng = random.Random(d + fp8)
    new = [[rng.choice([1, 1, 2, rng.randint(30, 200)]) for _ in range(20)] for _ in range(steps)]
    T = max(sum(n) for n in new)
    total = [sum(x) for x in zip(*new)]
    width = max(-(-t // bs) for t in total) + 1
    nb = sum(-(-t // bs) for t in total) + 5
    gen = torch.Generator(device=DEV).manual_seed(11)
    qkv = torch.randn((steps, L, T, (hq + 2 * hk) * d), generator=gen, device=DEV).to(torch.bfloat16)
    news = [i32(n) for n in new]
    ms = store(hk, d, L)

    def run(wait, graph=False):
        from paper_2607_27090_b200.memstore import GrownBlocks, PagedCache

        cache = PagedCache.allocate(L, nb, bs, hk, d, DEV, fp8=fp8, k_scale=0.02, v_scale=0.03)
        tables, free, taken = i32(np.full((20, width), -1)), i32(rng_ids), i32([0])
        lens = i32([0] * 20)
        g = GrownBlocks(i32([0] * 21), lens, i32([0] * T), torch.zeros(T, dtype=torch.int64, device=DEV), taken, i32([0] * 20))
        buf, q, out = torch.zeros_like(qkv[0, 0]), torch.zeros((T, hq, d), dtype=torch.bfloat16, device=DEV), torch.zeros((steps, L, T, hq, d), dtype=torch.bfloat16, device=DEV)
        workspace = torch.full((ms.attend_workspace_bytes(),), 255, dtype=torch.uint8, device=DEV)  # (any contents will do)

        def body():
            for s in range(steps):
                ms.grow_blocks(lens, news[s], tables, cache, free, taken, T, out=g)
                for layer in range(L):
                    buf.copy_(qkv[s, layer])
                    h = buf.unflatten(1, (hq + 2 * hk, d))
                    ms.append(layer, h[:, :hq], h[:, hq : hq + hk], h[:, hq + hk :], g.positions, g.slots, cache, q_out=q)
                    ms.attend(layer, q, cache, g.q_start, g.seq_lens, tables, out=out[s, layer], workspace=workspace)
                    if wait:
                        torch.cuda.synchronize()

        if graph:
            cg = torch.cuda.CUDAGraph()
            with torch.cuda.graph(cg):
                body()
            for t, v in ((tables, -1), (taken, 0), (lens, 0)):
                t.fill_(v)
            cg.replay()
        else:
            body()
        torch.cuda.synchronize()
        return out

    rng_ids = list(range(nb))
    rng.shuffle(rng_ids)
    want = run(True)
    assert want.float().abs().amax(dim=(2, 3, 4)).min() > 0
    for _ in range(4):
        assert torch.equal(run(False), want)
    assert torch.equal(run(False, graph=True), want)
    ms.close()


# ------------------------------------------------------------------------------------------------ scales
@pytest.mark.parametrize("n", [3, 100])
@pytest.mark.parametrize("fp8", [False, True])
def test_attend_scales_at_the_ends_of_their_range(fp8, n):
    """Scales (and 8-bit scales) whose product with the powers of two inside leaves fp32: far too small ones give every key a row sees the
    same weight, far too large ones give the key with the largest score all of it."""
    hk, hq, d, len_ = 1, 4, 128, 300
    tables, nb = paged(random.Random(2), [len_], 16)
    cache, gen = fill_cache(1, nb, 16, hk, d, fp8, "NHD", 5, k_scale=1.0)
    q = torch.randn((n, hq, d), generator=gen, device=DEV).to(torch.bfloat16)
    q[0, 0] = 0.0  # (a row of zeros scales by the largest power of two)
    q[1, 1] *= 2.0**-90
    ms = store(hk, d)
    qs, ln = i32([0, n]), i32([len_])
    k, v, _ = ref.cache_rows(cache, 0, tables[0], len_, nb)
    seen = torch.arange(len_ - n + 1, len_ + 1, device=DEV).double()
    mean = torch.cumsum(v[:, 0], 0)[len_ - n :] / seen[:, None]
    for scale, k_scale in ((1e-36, 1.0), (1.0e-44, 1.0)) + (((1e-30, 1e-20), (1e-20, 1e-38)) if fp8 else ()):
        cache.k_scale = k_scale
        out, lse, _ = ms.attend(0, q, cache, qs, ln, tables, scale=scale, want_lse=True)
        # weights of one: fp32 sums of at most 300 values of magnitude 14 (0.03 * 448), one rounding to bf16
        assert ((out.double() - mean[:, None]).abs() <= 2.0**-8 * mean[:, None].abs() + 300 * 14 * 2.0**-24).all()
        assert ((lse.double() - seen.log()[:, None]).abs() <= 2.0**-18).all()
    # every score of one tile's rows is infinite or zero: the row of zeros still sees all keys alike
    cache.k_scale = 1.0
    out, lse, _ = ms.attend(0, q, cache, qs, ln, tables, scale=3.0e38, want_lse=True)
    assert ((out[0, 0].double() - mean[0]).abs() <= 2.0**-8 * mean[0].abs() + 300 * 14 * 2.0**-24).all()
    assert abs(lse[0, 0].item() - math.log(len_ - n + 1)) <= 2.0**-18
    ms.close()


# ------------------------------------------------------------------------------------------------ workspaces
def test_attend_on_an_external_stream_keeps_no_workspace_for_it():
    import ctypes

    driver = ctypes.CDLL("libcuda.so.1")
    lens, q_start = [700, 50], [0, 100, 101]
    tables, nb = paged(random.Random(9), lens, 16)
    cache, gen = fill_cache(1, nb, 16, 2, 128, False, "NHD", 9)
    ms = store(2, 128)
    q = torch.randn((101, 8, 128), generator=gen, device=DEV).to(torch.bfloat16)
    qs, ln = i32(q_start), i32(lens)
    want, _, _ = ms.attend(0, q, cache, qs, ln, tables)
    torch.cuda.synchronize()
    kept = len(ms._workspaces)
    with torch.cuda.stream(torch.cuda.Stream()):
        assert torch.equal(ms.attend(0, q, cache, qs, ln, tables)[0], want)
    assert len(ms._workspaces) == kept + 1  # one of torch's own streams
    torch.cuda.synchronize()
    for _ in range(3):
        handle = ctypes.c_void_p()
        assert driver.cuStreamCreate(ctypes.byref(handle), 1) == 0
        with torch.cuda.stream(torch.cuda.ExternalStream(handle.value)):
            outs = [ms.attend(0, q, cache, qs, ln, tables)[0] for _ in range(3)]
        torch.cuda.synchronize()
        assert driver.cuStreamDestroy_v2(handle) == 0
        assert all(torch.equal(o, want) for o in outs) and len(ms._workspaces) == kept + 1
    ms.close()
