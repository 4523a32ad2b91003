"""Operators around the paged KV cache that spend fewer passes or fewer bytes per token, with their plain forms in elementary torch operations.

Drafted trees (several guesses of the next tokens checked in one pass):
  plan       positions and visibility masks of drafted trees from their parents
  verify     attention of the drafted nodes over the cache: the context, and among the nodes what the mask names
  accept     the drafted tokens that the model confirms: their path, the cache put in order, blocks behind it back to the free list
Selected blocks (long contexts of which a token reads a part):
  summarize  smallest and largest key of every cache block, coordinate by coordinate
  select     each token's best blocks by an upper bound of their scores
  sparse     attention of each token over its selected blocks

With ``own`` false ``run`` computes the plain forms, with ``own`` true it calls the library.
"""
import math
import random

import numpy as np
import torch

own = False

_FP8 = torch.float8_e4m3fn
_KS, _VS = 0.02, 0.015  # scales of the 8-bit caches
_VOCAB = 128256


# ------------------------------------------------------------------------------------------------ cases
def _plan(name, nreq, nodes, shape_seed, pad=0):
    return {"name": name, "op": "plan", "nreq": nreq, "n_lo": nodes[0], "n_hi": nodes[1], "pad": pad, "shape_seed": shape_seed}


def _verify(name, nreq, heads, kv_heads, dim, block_size, fp8, ctx, nodes, shape_seed, lse=False, head_major=False):
    return {"name": name, "op": "verify", "nreq": nreq, "heads": heads, "kv_heads": kv_heads, "dim": dim, "block_size": block_size, "fp8": fp8,
            "ctx_lo": ctx[0], "ctx_hi": ctx[1], "n_lo": nodes[0], "n_hi": nodes[1], "lse": lse, "head_major": head_major, "shape_seed": shape_seed}  # fmt: skip


def _accept(name, nreq, layers, kv_heads, dim, block_size, fp8, ctx, nodes, shape_seed, head_major=False):
    return {"name": name, "op": "accept", "nreq": nreq, "layers": layers, "kv_heads": kv_heads, "dim": dim, "block_size": block_size, "fp8": fp8,
            "ctx_lo": ctx[0], "ctx_hi": ctx[1], "n_lo": nodes[0], "n_hi": nodes[1], "head_major": head_major, "shape_seed": shape_seed}  # fmt: skip


def _summarize(name, nreq, kv_heads, dim, block_size, fp8, ctx, new, shape_seed, head_major=False):
    return {"name": name, "op": "summarize", "nreq": nreq, "kv_heads": kv_heads, "dim": dim, "block_size": block_size, "fp8": fp8, "ctx_lo": ctx[0],
            "ctx_hi": ctx[1], "new": new, "head_major": head_major, "shape_seed": shape_seed}  # fmt: skip


def _select(name, nreq, heads, kv_heads, dim, block_size, ctx, new, select, first, last, shape_seed):
    return {"name": name, "op": "select", "nreq": nreq, "heads": heads, "kv_heads": kv_heads, "dim": dim, "block_size": block_size, "ctx_lo": ctx[0],
            "ctx_hi": ctx[1], "new": new, "select": select, "first": first, "last": last, "shape_seed": shape_seed}  # fmt: skip


def _sparse(name, nreq, heads, kv_heads, dim, block_size, fp8, ctx, new, select, shape_seed, lse=False, head_major=False):
    return {"name": name, "op": "sparse", "nreq": nreq, "heads": heads, "kv_heads": kv_heads, "dim": dim, "block_size": block_size, "fp8": fp8,
            "ctx_lo": ctx[0], "ctx_hi": ctx[1], "new": new, "select": select, "lse": lse, "head_major": head_major, "shape_seed": shape_seed}  # fmt: skip


def listed():
    return [
        # one user's draft of 26 nodes
        _plan("plan one tree", 1, (26, 26), 1),
        # wide drafts of a full batch, packed arrays padded to a bucket
        _plan("plan 256 trees", 256, (40, 255), 2, pad=333),
        # one user's draft after 50 injected facts, Llama-3.1-8B heads
        _verify("verify one draft", 1, 32, 8, 128, 16, False, (2033, 2033), (26, 26), 3),
        # a batch's drafts over long contexts in an 8-bit cache, 14B-class heads
        _verify("verify 40 drafts 8-bit", 40, 40, 8, 128, 32, True, (700, 9000), (17, 61), 4, lse=True),
        # one user's draft: three tokens or so move in each of 32 layers
        _accept("accept one draft", 1, 32, 8, 128, 16, False, (700, 700), (26, 26), 5),
        # a batch's drafts, short contexts, 32 layers
        _accept("accept 90 drafts", 90, 32, 8, 128, 16, False, (9, 70), (20, 60), 6),
        # the new token of each of 100 users: its block's summary is formed again
        _summarize("summarize decode 100 users", 100, 8, 128, 16, False, (500, 1300), 1, 7),
        # contexts of injected facts, every block
        _summarize("summarize 32 contexts", 32, 8, 128, 32, False, (1900, 13700), 0, 8),
        # one user's token over 131,000 others
        _select("select one long context", 1, 32, 8, 128, 16, (131001, 131001), 1, 64, 1, 4, 9),
        # a decode step of 60 users over ragged contexts, 14B-class heads
        _select("select 60 users", 60, 40, 8, 128, 16, (3000, 32700), 1, 128, 1, 8, 10),
        # the same token over its 64 blocks
        _sparse("sparse one long context", 1, 32, 8, 128, 16, False, (131001, 131001), 1, 64, 11, lse=True),
        # the decode step of 60 users, 128 blocks each, 8-bit cache
        _sparse("sparse 60 users 8-bit", 60, 40, 8, 128, 16, True, (3000, 16300), 1, 128, 12),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["plan", "verify", "verify", "accept", "summarize", "select", "sparse", "sparse"])
    shape_seed = rng.randrange(1 << 30)
    block_size = rng.choice([16, 16, 32, 64])
    top = max(_cost(x) for x in listed() if x["op"] == op)
    while True:
        nreq = _log(rng, 1, 128)
        heads, kv_heads = rng.choice([(32, 8), (40, 8), (16, 4), (8, 8), (28, 4), (16, 1)])
        dim = rng.choice([64, 128, 128, 128])
        hi = _log(rng, 16, 32000)
        ctx = (rng.randint(1, hi), hi)
        n_hi = _log(rng, 1, 255)
        nodes = (rng.randint(1, n_hi), n_hi)
        fp8, lse, head_major = (rng.choice([False, True]) for _ in range(3))
        new = rng.choice([1, 1, 1, 2, rng.randint(1, 9)])
        if op == "plan":
            c = _plan("", nreq, nodes, shape_seed, rng.choice([0, 5, 600]))
        elif op == "verify":
            c = _verify("", nreq, heads, kv_heads, dim, block_size, fp8, ctx, nodes, shape_seed, lse, head_major)
        elif op == "accept":
            c = _accept("", nreq, rng.choice([1, 16, 32, 48]), kv_heads, dim, block_size, fp8, (ctx[0] % 60, 60 + ctx[0] % 7), (min(nodes[0], 60), min(n_hi, 60)),
                        shape_seed, head_major)  # fmt: skip
        elif op == "summarize":
            c = _summarize("", nreq, kv_heads, dim, block_size, fp8, ctx, rng.choice([0, 1, new, 61]), shape_seed, head_major)
        else:
            k = _log(rng, 1, 256)
            first = rng.randint(0, min(2, k - 1))
            if op == "select":
                c = _select("", nreq, heads, kv_heads, dim, block_size, ctx, new, k, first, rng.randint(0, min(8, k - first)), shape_seed)
            else:
                c = _sparse("", nreq, heads, kv_heads, dim, block_size, fp8, ctx, new, k, shape_seed, lse, head_major)
        if _cost(c) <= top and _padded(c) <= 1.2e9:
            break
    del c["name"]
    return c


def _cost(case):
    w = work(case)
    return max(w["bytes"], w["flops"] / 100)


def _padded(case):
    """Elements that the plain form holds at once."""
    op, n = case["op"], case["nreq"]
    if op == "plan":
        return n * case["n_hi"] ** 2
    ctx = case["ctx_hi"] + case.get("n_hi", 0)
    if op == "verify":
        return max(n * case["n_hi"] * ctx * case["heads"], 2 * n * ctx * case["kv_heads"] * case["dim"])
    if op == "accept":
        return n * ctx * case["layers"] * case["kv_heads"] * case["dim"]
    if op == "summarize":
        return 2 * n * ctx * case["kv_heads"] * case["dim"]
    if op == "select":
        return n * case["new"] * ctx // case["block_size"] * case["kv_heads"] * case["dim"] * 4
    return max(n * ctx * case["kv_heads"] * case["dim"], 2 * n * case["new"] * case["kv_heads"] * min(case["select"] * case["block_size"], ctx) * case["dim"])


# ------------------------------------------------------------------------------------------------ lengths (by the case alone)
def _blocks(n, bs):
    return -(-n // bs)


def _lengths(case):
    """New tokens and tokens in the cache (the new ones among them) of every request."""
    r = random.Random(case["shape_seed"])
    ctx = [r.randint(case.get("ctx_lo", 0), case.get("ctx_hi", 0)) for _ in range(case["nreq"])]
    if "n_lo" in case:
        new = [r.randint(case["n_lo"], case["n_hi"]) for _ in range(case["nreq"])]
        return new, [c + n for c, n in zip(ctx, new)]
    ctx = [max(c, 1) for c in ctx]
    return [min(case["new"] or c, c) for c in ctx], ctx


def _words(case):
    return _blocks(case["n_hi"], 32)


# ------------------------------------------------------------------------------------------------ inputs
def _generator(seed, case):
    return torch.Generator(device="cuda").manual_seed(int(seed) * 1000003 + case["shape_seed"])


def _store(layers, case):
    """The handle that a user's program keeps."""
    from paper_2607_27090_b200.memstore import MemStore

    return MemStore(n_layers=layers, n_kv_heads=case.get("kv_heads", 1), head_dim=case.get("dim", 64), emb_dim=64, max_facts_per_user=1, max_kv_tokens=0)


def _paged(case, s):
    """The description of the cache that a user's program keeps."""
    from paper_2607_27090_b200.memstore import PagedCache

    h, d, bs, nb = case["kv_heads"], case["dim"], case["block_size"], s["num_blocks"]
    k = s.get("k_cache")
    if k is None:  # selecting takes no more of the cache than its geometry
        k = torch.empty((1, 1, bs, h, d), dtype=torch.bfloat16, device="cuda")
    token, head = (d, bs * d) if case.get("head_major") else (h * d, d)
    return PagedCache(k, s.get("v_cache", k), nb * bs * h * d, bs * h * d, token, head, nb, bs, k_scale=_KS, v_scale=_VS)


def _cache(case, num_blocks, gen, layers=1):
    """K and V of a paged cache, filled as after earlier writes: [layers, blocks, bs, h, d] or [layers, blocks, h, bs, d]."""
    bs, h, d = case["block_size"], case["kv_heads"], case["dim"]
    shape = (layers, num_blocks, h, bs, d) if case["head_major"] else (layers, num_blocks, bs, h, d)
    x = [torch.randn(shape, generator=gen, device="cuda", dtype=torch.bfloat16) for _ in range(2)]
    return [(t.float() / c).clamp_(-448, 448).to(_FP8).view(torch.uint8) if case["fp8"] else t for t, c in zip(x, (_KS, _VS))]


def _tables(case, lens, gen):
    """Block tables of random blocks, their number, and the ids that are left over."""
    bs, dev = case["block_size"], {"device": "cuda"}
    used = torch.tensor([_blocks(n, bs) for n in lens], **dev)
    num_blocks = sum(_blocks(n, bs) for n in lens) + 9
    ids = torch.randperm(num_blocks, generator=gen, **dev).to(torch.int32)
    col = torch.arange(max(_blocks(n, bs) for n in lens) + 2, **dev)
    at = (used.cumsum(0) - used)[:, None] + col
    return torch.where(col < used[:, None], ids[at.clamp(max=num_blocks - 1)], 0), num_blocks, ids[num_blocks - 9 :]


def _starts(new):
    return torch.tensor([0, *np.cumsum(new)], dtype=torch.int32, device="cuda")


def _local(new, pad=0):
    """Request of every packed token, and its place in the request; padding behind the last one belongs to none (-1)."""
    n = torch.tensor(new, device="cuda")
    r = torch.repeat_interleave(torch.arange(len(new), device="cuda"), n)
    i = torch.arange(len(r), device="cuda") - (n.cumsum(0) - n)[r]
    none = torch.full((pad,), -1, device="cuda")
    return torch.cat([r, none]), torch.cat([i, none])


def _parents(i, gen):
    """Random trees: node 0 is the root, node i hangs on one of the nodes before it."""
    u = torch.rand(i.shape, generator=gen, device="cuda", dtype=torch.float64)
    return torch.where(i > 0, (u * i).long().clamp(max=i - 1), -1).int()


def prepare(case, seed):
    gen = _generator(seed, case)
    i32 = {"dtype": torch.int32, "device": "cuda"}
    op = case["op"]
    new, lens = _lengths(case)
    s = {"case": case, "q_start": _starts(new), "seq_lens": torch.tensor(lens, **i32), "max_new": max(new), "max_len": max(lens)}
    s["request"], s["place"] = _local(new, case.get("pad", 0))
    T = len(s["place"])
    if op == "plan":
        s["parents"] = _parents(s["place"], gen)
        start = torch.randint(0, 9000, (case["nreq"],), generator=gen, device="cuda")
        s["positions"] = torch.where(s["place"] >= 0, start[s["request"]] + s["place"], -1).int()
        s["out_positions"], s["mask"] = torch.full((T,), -1, **i32), torch.zeros((T, _words(case)), **i32)
        if own:
            s["store"] = _store(1, case)
        return s
    s["tables"], s["num_blocks"], spare = _tables(case, lens, gen)
    if op != "select":
        s["k_cache"], s["v_cache"] = _cache(case, s["num_blocks"], gen, case.get("layers", 1))
    if op == "verify":
        s["parents"] = _parents(s["place"], gen)
        s["mask"] = _pack(_ancestors(s), _words(case))[s["request"], s["place"]]
    elif op == "accept":
        s["parents"] = p = _parents(s["place"], gen)
        s["positions"] = (s["seq_lens"] - s["q_start"].diff())[s["request"]] + s["place"].int()
        s["tokens"] = torch.randint(0, _VOCAB, (T,), generator=gen, **i32)
        # what the model says behind each node: mostly the token of its last child, where that is not one of the first nodes
        first = s["q_start"][s["request"]].long()
        child = torch.full((T,), -1, device="cuda").scatter_reduce(0, (first + p).clamp(min=0), torch.where(p >= 0, s["place"], -1), "amax")
        late = (child > s["q_start"].diff()[s["request"]] // 3) & (torch.rand(T, generator=gen, device="cuda") < 0.9)
        other = torch.randint(0, _VOCAB, (T,), generator=gen, **i32)
        s["choices"] = torch.where(late, s["tokens"][first + child.clamp(min=0)], other)
        s["free_blocks"] = torch.cat([torch.zeros(sum(_blocks(n, case["block_size"]) for n in lens), **i32), spare])
        s["n_taken"] = torch.tensor([s["free_blocks"].numel() - spare.numel()], **i32)
    elif op in ("select", "summarize"):
        shape = (s["num_blocks"], case["kv_heads"], 2, case["dim"])
        s["summaries"] = torch.zeros(shape, dtype=torch.bfloat16, device="cuda")
        if op == "select":  # smallest and largest key of each block
            mid = 0.6 * torch.randn(shape[:2] + shape[3:], generator=gen, device="cuda")
            off = 1.5 + 0.4 * torch.randn(mid.shape, generator=gen, device="cuda").abs()
            s["summaries"][:, :, 0], s["summaries"][:, :, 1] = mid - off, mid + off
            s["blocks"] = torch.full((T, case["kv_heads"], case["select"]), -1, **i32)
            s["scores"] = torch.zeros((T, case["kv_heads"], s["tables"].shape[1]), device="cuda")
    elif op == "sparse":
        s["blocks"] = _some_blocks(case, s, gen)
    if op in ("verify", "select", "sparse"):
        s["q"] = (1.5 * torch.randn((T, case["heads"], case["dim"]), generator=gen, device="cuda")).to(torch.bfloat16)
    if own:
        s["store"], s["cache"] = _store(case.get("layers", 1), case), _paged(case, s)
    return s


def _held(case, s):
    """Blocks that each token may read."""
    pos = (s["seq_lens"] - s["q_start"].diff())[s["request"]] + s["place"]
    return pos // case["block_size"] + 1


def _some_blocks(case, s, gen):
    """Lists as a selection gives them: the first block, the last ones, others at random; ascending, -1 behind the end."""
    nb, k = _held(case, s), case["select"]
    col = torch.arange(_blocks(s["max_len"], case["block_size"]), device="cuda")
    u = torch.rand((len(nb), case["kv_heads"], len(col)), generator=gen, device="cuda")
    u = torch.where(col == 0, 2.0, u)
    u = torch.where(col >= nb[:, None, None] - min(4, k), 3.0, u)
    u = torch.where(col < nb[:, None, None], u, -1.0)
    best = u.topk(min(k, len(col)), dim=2)
    ids = torch.where(best.values >= 0, best.indices, 1 << 30).sort(2).values
    ids = torch.where(ids < 1 << 30, ids, -1).int()
    return torch.nn.functional.pad(ids, (0, k - ids.shape[2]), value=-1).contiguous()


# ------------------------------------------------------------------------------------------------ the passes
def run(state):
    case = state["case"]
    if own:
        return _run_own(case, state)
    forms = {"plan": _plain_plan, "verify": _plain_verify, "accept": _plain_accept, "summarize": _plain_summarize, "select": _plain_select, "sparse": _plain_sparse}
    return forms[case["op"]](case, state)


def _run_own(case, s):
    op, store = case["op"], s["store"]
    if op == "plan":
        positions, mask, _ = store.plan_tree(s["parents"], s["q_start"], s["positions"], out_positions=s["out_positions"], out_mask=s["mask"])
        return {"positions": positions, "mask": mask}
    if op == "accept":
        a = store.accept(s["parents"], s["tokens"], s["choices"], s["positions"], s["q_start"], s["seq_lens"], s["tables"], s["cache"], s["free_blocks"],
                         s["n_taken"])  # fmt: skip
        return {"path": a.path, "n_accepted": a.n_accepted, "next": a.next_tokens, "seq_lens": a.seq_lens, "n_taken": a.n_taken, "free": s["free_blocks"],
                **_stored(case, s)}  # fmt: skip
    if op == "summarize":
        store.summarize_blocks(0, s["cache"], s["summaries"], s["seq_lens"], s["tables"], q_start=s["q_start"] if case["new"] else None, n_tokens=len(s["place"]))
        return s["summaries"]
    if op == "select":
        store.select_blocks(s["q"], s["cache"], s["summaries"], s["q_start"], s["seq_lens"], s["tables"], case["select"], n_first=case["first"],
                            n_last=case["last"], out_blocks=s["blocks"], out_scores=s["scores"])  # fmt: skip
        return {"blocks": s["blocks"], "scores": s["scores"]}
    if op == "verify":
        out, lse, _ = store.attend_tree(0, s["q"], s["mask"], s["cache"], s["q_start"], s["seq_lens"], s["tables"], max_q_len=s["max_new"], want_lse=case["lse"])
    else:
        out, lse, _ = store.attend_blocks(0, s["q"], s["blocks"], s["cache"], s["q_start"], s["seq_lens"], s["tables"], want_lse=case["lse"])
    return [out, lse] if case["lse"] else out


def _stored(case, s):
    return {n: s[n].view(_FP8) if case["fp8"] else s[n] for n in ("k_cache", "v_cache")}


def _ancestors(s):
    """[requests, nodes, nodes]: whether the second node is the first one or lies above it (roads of doubled length)."""
    n, N = s["seq_lens"].numel(), s["max_new"]
    live = s["place"] >= 0
    r, i, p = s["request"][live], s["place"][live], s["parents"][live].long()
    up = torch.zeros((n, N, N), device=p.device)
    up[r, i, p.clamp(min=0)] = (p >= 0).float()
    up[r, i, i] = 1.0
    for _ in range(max(1, (N - 1).bit_length())):
        up = torch.matmul(up, up).clamp_(max=1.0)
    return up


def _pack(see, words):
    """32 truth values to a word, the lowest bit first."""
    bits = torch.nn.functional.pad(see, (0, 32 * words - see.shape[-1])).unflatten(-1, (words, 32)).long()
    w = (bits << torch.arange(32, device=see.device)).sum(-1)
    return torch.where(w >= 1 << 31, w - (1 << 32), w).int()


def _plain_plan(case, s):
    see = _ancestors(s)
    live = s["place"] >= 0
    r, i = s["request"][live], s["place"][live]
    depth = see.sum(-1)[r, i].int() - 1
    s["mask"][live] = _pack(see, s["mask"].shape[1])[r, i]
    s["out_positions"][live] = s["positions"][s["q_start"][:-1].long()][r] + depth
    return {"positions": s["out_positions"], "mask": s["mask"]}


def _token_major(case, x):
    """[blocks, bs, h, d] of one layer."""
    return x[0].transpose(1, 2) if case["head_major"] else x[0]


def _values(case, x, scale):
    return x.view(_FP8).float() * scale if case["fp8"] else x.float()


def _plain_verify(case, s):
    n, hq, hk, d, bs = case["nreq"], case["heads"], case["kv_heads"], case["dim"], case["block_size"]
    g, qmax, kmax = hq // hk, s["max_new"], s["max_len"]
    dev = s["q"].device
    q_start, lens = s["q_start"].long(), s["seq_lens"].long()
    q_lens = q_start.diff()
    key = torch.arange(kmax, device=dev)
    index = s["tables"].long()[:, (key // bs).clamp(max=s["tables"].shape[1] - 1)]
    k, v = (_values(case, _token_major(case, s[c])[index, key % bs], sc).transpose(1, 2) for c, sc in (("k_cache", _KS), ("v_cache", _VS)))
    i = torch.arange(qmax, device=dev)
    row = (q_start[:-1, None] + i).clamp(max=s["q"].shape[0] - 1)  # padded to the largest tree
    q = s["q"][row].float().unflatten(2, (hk, g)).permute(0, 2, 3, 1, 4).reshape(n, hk, g * qmax, d)
    scores = torch.matmul(q, k.transpose(2, 3)).view(n, hk, g, qmax, kmax).mul_(1.0 / math.sqrt(d))
    bit = (key - (lens - q_lens)[:, None])[:, None].expand(n, qmax, kmax)  # the node that a key belongs to, negative: context
    word = s["mask"][row].gather(2, (bit // 32).clamp(0, s["mask"].shape[1] - 1))
    see = (bit < 0) | ((bit < q_lens[:, None, None]) & ((word >> (bit % 32)) & 1).bool())
    scores.masked_fill_(~see[:, None, None], -math.inf)
    m = scores.amax(-1, keepdim=True)
    p = scores.sub_(m).exp_()
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p.view(n, hk, g * qmax, kmax), v).view(n, hk, g, qmax, d) / total
    has = i[None] < q_lens[:, None]
    out = out.permute(0, 3, 1, 2, 4).reshape(n, qmax, hq, d)[has].to(torch.bfloat16)
    return [out, (m + total.log())[..., 0].permute(0, 3, 1, 2).reshape(n, qmax, hq)[has]] if case["lse"] else out


def _plain_accept(case, s):
    n, T, bs = case["nreq"], len(s["place"]), case["block_size"]
    r, i, p, tok = s["request"], s["place"], s["parents"].long(), s["tokens"]
    first = s["q_start"].long()[r]
    above = (first + p).clamp(min=0)
    match = (p >= 0) & (tok == s["choices"][above])
    winner = torch.full((T,), T, device=p.device).scatter_reduce(0, above, torch.where(match, i, T), "amin")
    good = (i == 0) | (match & (winner[above] == i))
    jump = torch.where(i == 0, first, above)
    for _ in range(max(1, (s["max_new"] - 1).bit_length())):  # whether all nodes up to the root are good
        good, jump = good & good[jump], jump[jump]
    a = torch.zeros(n, dtype=torch.int64, device=p.device).scatter_add(0, r, good.long())
    rank = good.long().cumsum(0) - 1 - (a.cumsum(0) - a)[r]
    path = torch.full((T,), -1, device=p.device).scatter(0, torch.where(good, first + rank, 0), torch.where(good, i, 0))  # (entry 0 is node 0 of request 0)
    last = path[s["q_start"].long()[:-1] + a - 1] + s["q_start"].long()[:-1]
    lens = s["seq_lens"].long()
    start = lens - s["q_start"].long().diff()
    src, dst = start[r] + torch.where(path >= 0, path, i), start[r] + i
    tables = s["tables"].long()
    move = [(tables[r, x // bs], x % bs) for x in (src, dst)]
    for c in ("k_cache", "v_cache"):
        x = s[c].transpose(2, 3) if case["head_major"] else s[c]
        x[:, move[1][0], move[1][1]] = x[:, move[0][0], move[0][1]]
    # blocks behind the new end: request 0's in front of the free part, the next request's in front of them
    held, kept = (lens + bs - 1) // bs, (start + a + bs - 1) // bs
    back = held - kept
    upto = back.cumsum(0)
    col = torch.arange(tables.shape[1], device=p.device)[None]
    at = s["n_taken"] - upto[:, None] + col - kept[:, None]
    going = (col >= kept[:, None]) & (col < held[:, None])
    s["free_blocks"][at[going]] = s["tables"][going]
    return {"path": path.int(), "n_accepted": a.int(), "next": s["choices"][last], "seq_lens": (start + a).int(), "n_taken": (s["n_taken"] - upto[-1]).int(),
            "free": s["free_blocks"], **_stored(case, s)}  # fmt: skip


def _plain_summarize(case, s):
    bs = case["block_size"]
    lens = s["seq_lens"].long()
    start = lens - s["q_start"].long().diff() if case["new"] else torch.zeros_like(lens)
    col = torch.arange(_blocks(s["max_len"], bs), device=lens.device)
    touched = (col >= start[:, None] // bs) & (col < (lens[:, None] + bs - 1) // bs)
    r, b = touched.nonzero(as_tuple=True)
    block = s["tables"].long()[r, b]
    x = _values(case, _token_major(case, s["k_cache"])[block], 1.0)  # (8-bit caches: of the codes' values)
    dead = (b[:, None] * bs + torch.arange(bs, device=lens.device) >= lens[r, None])[:, :, None, None]
    s["summaries"][block, :, 0] = x.masked_fill(dead, math.inf).amin(1).to(torch.bfloat16)
    s["summaries"][block, :, 1] = x.masked_fill(dead, -math.inf).amax(1).to(torch.bfloat16)
    return s["summaries"]


def _plain_select(case, s):
    """Sums of 64 bits: a list changes where two scores are as near as 32-bit sums err."""
    hk, k = case["kv_heads"], case["select"]
    q = s["q"].double().unflatten(1, (hk, -1))
    q = torch.stack([q.clamp(max=0).sum(2), q.clamp(min=0).sum(2)], 2)  # against smallest and largest keys
    nb = _held(case, s)[:, None, None]
    col = torch.arange(_blocks(s["max_len"], case["block_size"]), device=q.device)
    block = s["tables"].long()[:, : len(col)]
    one = case["new"] == 1  # (several tokens of a request read the same summaries)
    x = s["summaries"][block].permute(0, 2, 1, 3, 4).flatten(3).double()
    x = x if one else x[s["request"]]
    score = torch.matmul(x, q.flatten(2)[..., None])[..., 0].float()
    s["scores"][:, :, : len(col)] = torch.where(col < nb, score, s["scores"][:, :, : len(col)])
    forced = (col < case["first"]) | (col >= nb - case["last"])
    score = torch.where(forced, math.inf, score).masked_fill(col >= nb, -math.inf)
    best = score.sort(dim=2, descending=True, stable=True).indices[:, :, :k]
    ids = torch.where(best < nb, best, 1 << 30).sort(dim=2).values
    s["blocks"][:, :, : ids.shape[2]] = torch.where(ids < 1 << 30, ids, -1).int()
    return {"blocks": s["blocks"], "scores": s["scores"]}


def _plain_sparse(case, s):
    hq, hk, d, bs = case["heads"], case["kv_heads"], case["dim"], case["block_size"]
    T = s["q"].shape[0]
    pos = (s["seq_lens"] - s["q_start"].diff())[s["request"]] + s["place"]
    slots = s["blocks"].long()[:, :, : _blocks(s["max_len"], bs)]
    key = (slots[..., None] * bs + torch.arange(bs, device=pos.device)).flatten(2)  # [T, hk, keys]
    live = (slots >= 0).repeat_interleave(bs, 2) & (key <= pos[:, None, None])
    key = key.clamp(min=0)
    index = s["tables"].long()[s["request"][:, None, None], (key // bs).clamp(max=s["tables"].shape[1] - 1)]
    head = torch.arange(hk, device=pos.device)[None, :, None]
    k, v = (_values(case, _token_major(case, s[c])[index, key % bs, head], sc) for c, sc in (("k_cache", _KS), ("v_cache", _VS)))
    q = s["q"].float().unflatten(1, (hk, -1))
    scores = torch.matmul(q, k.transpose(2, 3)).mul_(1.0 / math.sqrt(d)).masked_fill_(~live[:, :, None], -math.inf)
    m = scores.amax(-1, keepdim=True)
    p = scores.sub_(m).exp_()
    total = p.sum(-1, keepdim=True)
    out = (torch.matmul(p, v) / total).reshape(T, hq, d).to(torch.bfloat16)
    return [out, (m + total.log()).reshape(T, hq)] if case["lse"] else out


# ------------------------------------------------------------------------------------------------ what a pass cannot do without
def work(case):
    op = case["op"]
    new, lens = _lengths(case)
    T, bs = sum(new), case.get("block_size", 1)
    if op == "plan":
        return {"bytes": T * (8 + 4 * _words(case)) + 8 * case["nreq"], "flops": T}
    hk, d, row = case["kv_heads"], case["dim"], case["kv_heads"] * case["dim"] * (1 if case.get("fp8") else 2)
    if op == "accept":  # about three tokens of a draft are taken, the first of which stays where it is
        moved = sum(min(2, n - 1) for n in new)
        return {"bytes": moved * case["layers"] * 4 * row + 20 * T + 16 * case["nreq"], "flops": T}
    if op == "summarize":
        touched = [(_blocks(n, bs) - (n - a) // bs, n - (n - a) // bs * bs) for a, n in zip(new, lens)]
        return {"bytes": sum(k for _, k in touched) * row + sum(b for b, _ in touched) * (hk * d * 4 + 4), "flops": 2 * sum(k for _, k in touched) * hk * d}
    hq = case["heads"]
    if op == "verify":
        pairs = sum(n * (c - n) + n * 6 for n, c in zip(new, lens))
        kv = sum(lens) * 2 * row + 4 * sum(_blocks(c, bs) for c in lens)
        return {"bytes": kv + T * hq * (4 * d + (4 if case["lse"] else 0)) + 4 * T * _words(case), "flops": 4 * pairs * hq * d}
    if op == "select":  # several tokens of a request read the same summaries
        nb = sum(_blocks(c, bs) for c in lens)
        every = sum(n * _blocks(c, bs) for n, c in zip(new, lens))
        return {"bytes": nb * (hk * d * 4 + 4) + T * (2 * hq * d + 4 * hk * case["select"]) + 4 * every * hk, "flops": 4 * every * hk * d}
    keys = sum(n * min(case["select"] * bs, c) for n, c in zip(new, lens))
    return {"bytes": keys * 2 * row + T * (hq * (4 * d + (4 if case["lse"] else 0)) + 4 * hk * case["select"]), "flops": 4 * keys * hq * d}


# ------------------------------------------------------------------------------------------------ the definitions in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    forms = {"plan": _exact_plan, "verify": _exact_verify, "accept": _exact_accept, "summarize": _exact_summarize, "select": _exact_select, "sparse": _exact_sparse}
    return forms[case["op"]](case, s)


def _spans(s):
    q = s["q_start"].tolist()
    return list(zip(range(len(q) - 1), q, q[1:], s["seq_lens"].tolist()))


def _exact_plan(case, s):
    """Node after node: a node sees itself and what its parent sees."""
    parents, positions, out, mask = (s[n].cpu().numpy().copy() for n in ("parents", "positions", "out_positions", "mask"))
    for _, a, b, _ in _spans(s):
        sees = []
        for i in range(b - a):
            p = int(parents[a + i])
            sees.append((sees[p] if p >= 0 else 0) | 1 << i)
            out[a + i] = positions[a] + bin(sees[i]).count("1") - 1
            mask[a + i] = np.array([sees[i] >> 32 * w & 0xFFFFFFFF for w in range(mask.shape[1])], np.uint32).view(np.int32)
    return {"positions": torch.from_numpy(out), "mask": torch.from_numpy(mask)}


def _request_rows(case, s, r, n):
    """K and V of a request's first n tokens in 64 bits: [n, h, d]."""
    table = s["tables"][r, : _blocks(n, case["block_size"])].long()
    out = []
    for c, scale in (("k_cache", _KS), ("v_cache", _VS)):
        x = _token_major(case, s[c])[table].flatten(0, 1)[:n]
        out.append(x.view(_FP8).float().double() * float(np.float32(scale)) if case["fp8"] else x.double())
    return out


def _exact_rows(q, k, v, see, d):
    t = (q.double() @ k.T / math.sqrt(d)).masked_fill(~see, -math.inf)
    return torch.softmax(t, 1) @ v, torch.logsumexp(t, 1)


def _exact_verify(case, s):
    """Request by request and head by head."""
    hq, hk, d = case["heads"], case["kv_heads"], case["dim"]
    if work(case)["flops"] > 2e12:
        return None
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(s["q"].shape[:2], dtype=torch.float64, device="cuda")
    for r, a, b, n in _spans(s):
        k, v = _request_rows(case, s, r, n)
        words = s["mask"][a:b].cpu().numpy().view(np.uint32).view(np.uint8)
        bits = np.unpackbits(words, axis=1, bitorder="little")[:, : b - a].astype(bool)
        see = torch.cat([torch.ones((b - a, n - (b - a)), dtype=torch.bool), torch.from_numpy(bits)], 1).cuda()
        for h in range(hq):
            out[a:b, h], lse[a:b, h] = _exact_rows(s["q"][a:b, h], k[:, h * hk // hq], v[:, h * hk // hq], see, d)
    return [out, lse] if case["lse"] else out


def _exact_accept(case, s):
    """A walk down every tree, then row after row."""
    bs = case["block_size"]
    parents, tokens, choices = (s[n].tolist() for n in ("parents", "tokens", "choices"))
    tables, free, taken = s["tables"].cpu().numpy(), s["free_blocks"].cpu().numpy().copy(), s["n_taken"].item()
    caches = {n: x.clone() for n, x in _stored(case, s).items()}
    at = (lambda b, o: (slice(None), b, slice(None), o)) if case["head_major"] else (lambda b, o: (slice(None), b, o))
    path, counts, ends, said = [], [], [], []
    for r, a, b, n in _spans(s):
        way = [0]
        while True:
            here = way[-1]
            to = [c for c in range(here + 1, b - a) if parents[a + c] == here and tokens[a + c] == choices[a + here]]
            if not to:
                break
            way.append(to[0])
        first = n - (b - a)
        for i, c in enumerate(way):
            if c != i:
                x, y = first + c, first + i
                for t in caches.values():
                    t[at(int(tables[r, y // bs]), y % bs)] = t[at(int(tables[r, x // bs]), x % bs)]
        end = first + len(way)
        going = tables[r, _blocks(end, bs) : _blocks(n, bs)]
        free[taken - len(going) : taken] = going
        taken -= len(going)
        path += way + [-1] * (b - a - len(way))
        counts.append(len(way))
        ends.append(end)
        said.append(choices[a + way[-1]])
    i32 = lambda x: torch.tensor(np.asarray(x, np.int32))  # noqa: E731
    return {"path": i32(path), "n_accepted": i32(counts), "next": i32(said), "seq_lens": i32(ends), "n_taken": i32([taken]), "free": torch.from_numpy(free), **caches}


def _exact_summarize(case, s):
    bs, out = case["block_size"], s["summaries"].double()
    for r, a, b, n in _spans(s):
        first = (n - (b - a)) // bs if case["new"] else 0
        table = s["tables"][r, first : _blocks(n, bs)].long()
        x = _token_major(case, s["k_cache"])[table]
        x = x.view(_FP8).float().double() if case["fp8"] else x.double()
        full = (n - first * bs) // bs
        out[table[:full], :, 0], out[table[:full], :, 1] = x[:full].min(1).values, x[:full].max(1).values
        if full < len(table):
            rest = x[full, : n % bs]
            out[table[full], :, 0], out[table[full], :, 1] = rest.min(0).values, rest.max(0).values
    return out


def _exact_select(case, s):
    """Token by token: the largest possible sum of the group's scores, coordinate by coordinate."""
    bs, hk, k = case["block_size"], case["kv_heads"], case["select"]
    blocks, scores = s["blocks"].cpu().numpy().copy(), s["scores"].double()
    for r, a, b, n in _spans(s):
        for t in range(a, b):
            nb = (n - (b - a) + t - a) // bs + 1
            box = s["summaries"][s["tables"][r, :nb].long()].double()
            score = torch.zeros(nb, hk, dtype=torch.float64, device="cuda")
            for q in s["q"][t].double().unflatten(0, (hk, -1)).unbind(1):
                score += torch.maximum(q * box[:, :, 0], q * box[:, :, 1]).sum(-1)
            scores[t, :, :nb] = score.T
            score = score.float().cpu().numpy()
            must = [j for j in range(nb) if j < case["first"] or j >= nb - case["last"]]
            for h in range(hk):
                rest = np.argsort(-score[:, h], kind="stable")
                rest = rest[~np.isin(rest, must)]
                ids = np.sort(np.concatenate([np.array(must, np.int64), rest[: max(0, k - len(must))]]))
                blocks[t, h] = -1
                blocks[t, h, : len(ids)] = ids
    return {"blocks": torch.from_numpy(blocks), "scores": scores}


def _exact_sparse(case, s):
    """Token by token and K/V head by K/V head."""
    hq, hk, d, bs = case["heads"], case["kv_heads"], case["dim"], case["block_size"]
    g = hq // hk
    if len(s["place"]) * hk > 6000:
        return None
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(s["q"].shape[:2], dtype=torch.float64, device="cuda")
    lists = s["blocks"].cpu().numpy()
    for r, a, b, n in _spans(s):
        k, v = _request_rows(case, s, r, n)
        for t in range(a, b):
            for h in range(hk):
                keys = [j * bs + o for j in lists[t, h].tolist() if j >= 0 for o in range(bs)]
                keys = torch.tensor([j for j in keys if j <= n - (b - a) + t - a], device="cuda")
                see = torch.ones((g, len(keys)), dtype=torch.bool, device="cuda")
                x = slice(h * g, (h + 1) * g)
                out[t, x], lse[t, x] = _exact_rows(s["q"][t, x], k[keys, h], v[keys, h], see, d)
    return [out, lse] if case["lse"] else out
