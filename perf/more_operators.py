"""More operators of a serving step, as a serving program calls them: norms of the queries and keys of every head together with
the rotary embedding and the write to the cache; requests that branch, are cut back or move to another pool (forks, copies, freed
pages, compaction); penalties, biases and grammar masks on the logits of packed rows.

Sizes follow the repository's own workloads (the 0.5B, 1.5B and 3B shapes in bfloat16, the small shape in float32; contexts of
512 to 8192 tokens, up to 33 rows of drafts, batches of 16 sequences, pages of 64 tokens in random order).  A layer's pages have
the layout that include/vf.h states; the plain form takes it apart with views.
"""
import math
import random
from types import SimpleNamespace

import torch

DEV = "cuda:0"
own = False
PAGE = 64

# q heads, kv heads, head_dim, layers, vocabulary, dtype
SHAPES = {
    "0.5b": (14, 2, 64, 24, 151936, "bf16"),
    "1.5b": (12, 2, 128, 28, 151936, "bf16"),
    "3b": (24, 8, 128, 28, 128256, "bf16"),
    "tiny": (4, 4, 64, 2, 4096, "f32"),
}


def listed():
    return [
        # a decoding step of 16 users of a model with norms of q and k: one token each
        {"name": "norm_rotary_1.5b_16", "op": "norm", "shape": "1.5b", "seqs": 16, "held": 2048, "new": 1, "pairs": "half",
         "part": 1.0, "gains": "shared", "layout": 5},
        # float32: some prompts of odd lengths; interleaved pairs in half of each head, gains of their own for every head
        {"name": "norm_rotary_tiny_1100", "op": "norm", "shape": "tiny", "seqs": 5, "held": 0, "new": 219, "pairs": "interleaved",
         "part": 0.5, "gains": "heads", "layout": 3},
        # a long prompt of the widest shape behind a cached prefix
        {"name": "norm_rotary_3b_8192", "op": "norm", "shape": "3b", "seqs": 1, "held": 65, "new": 8192, "pairs": "half",
         "part": 1.0, "gains": "shared", "layout": 1},
        # four samples of one prompt: latency
        {"name": "fork_0.5b_4", "op": "fork", "shape": "0.5b", "parents": 1, "children": 4, "keys": 1000, "prefix": 1.0,
         "room": 1.5, "keep": 0.0, "layout": 4},
        # each of eight requests tries three continuations and gives them up: their pages go back
        {"name": "branch_1.5b_24", "op": "branch", "shape": "1.5b", "parents": 8, "children": 3, "keys": 1024, "prefix": 1.0,
         "room": 1.3, "keep": 0.0, "layout": 15},
        # 64 branches of 16 long contexts, cut back into pages that they share, in a pool with too little room for all
        {"name": "branch_3b_64", "op": "branch", "shape": "3b", "parents": 16, "children": 4, "keys": 1500, "prefix": 0.9,
         "room": 0.9, "keep": 0.7, "layout": 64},
        # a small batch moves to a smaller pool
        {"name": "compact_0.5b_5", "op": "compact", "shape": "0.5b", "parents": 3, "children": 1, "keys": 400, "spread": 2.0, "layout": 7},
        # a full batch with shared prefixes moves to a pool of its own
        {"name": "compact_1.5b_32", "op": "compact", "shape": "1.5b", "parents": 16, "children": 1, "keys": 2048, "spread": 1.5, "layout": 11},
        # one user, one token: the penalties of an ordinary sampler
        {"name": "logits_0.5b_1", "op": "logits", "vocab": 151936, "dtype": "f32", "seqs": 1, "rows": "one", "history": 1024,
         "penalties": True, "biases": 0, "allowed": 1.0, "layout": 1},
        # 16 drafts of one request under a grammar that leaves few tokens
        {"name": "logits_1.5b_17", "op": "logits", "vocab": 151936, "dtype": "f32", "seqs": 1, "rows": "draft16", "history": 2048,
         "penalties": True, "biases": 40, "allowed": 0.02, "layout": 3},
        # 70 users, one token each, logits in bfloat16, a vocabulary of another size, biases
        {"name": "logits_3b_70", "op": "logits", "vocab": 128256, "dtype": "bf16", "seqs": 70, "rows": "one", "history": 1500,
         "penalties": True, "biases": 300, "allowed": 1.0, "layout": 70},
        # the drafts of 16 users, 2 to 33 rows each, with everything at once
        {"name": "logits_1.5b_drafts", "op": "logits", "vocab": 151936, "dtype": "f32", "seqs": 16, "rows": "drafts", "history": 2048,
         "penalties": True, "biases": 100, "allowed": 0.6, "layout": 15312},
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm", "fork", "branch", "compact", "logits", "logits"])
    layout = rng.randint(1, 1 << 20)
    if op == "norm":
        new = rng.choice([1, _log_uniform(rng, 2, 8192)])
        return {"op": op, "shape": rng.choice(["0.5b", "1.5b", "3b", "tiny"]),
                "seqs": _log_uniform(rng, 1, 300) if new == 1 else _log_uniform(rng, 1, max(1, min(16, 5000 // new))),
                "held": rng.choice([0, _log_uniform(rng, 1, 4096)]), "new": new, "pairs": rng.choice(["half", "interleaved"]),
                "part": rng.choice([0.25, 0.5, 1.0]), "gains": rng.choice(["shared", "heads", "none"]), "layout": layout}
    if op == "logits":
        rows, dtype = rng.choice(["one", "one", "draft16", "drafts"]), rng.choice(["f32", "f32", "bf16"])
        vocab = rng.choice([151936, 128256, 4096, _log_uniform(rng, 500, 151936)])
        return {"op": op, "vocab": vocab, "dtype": dtype, "seqs": _log_uniform(rng, 1, {"one": 200, "draft16": 15, "drafts": 11}[rows]), "rows": rows,
                "history": _log_uniform(rng, 1, 8192), "penalties": rng.random() < 0.8, "biases": rng.choice([0, _log_uniform(rng, 1, 400)]),
                "allowed": rng.choice([1.0, 1.0, rng.random()]), "layout": layout}
    shape = rng.choice(["0.5b", "1.5b", "tiny"])
    if op == "compact":
        parents = _log_uniform(rng, 1, 16)
        return {"op": op, "shape": shape, "parents": parents, "children": rng.choice([0, 1, 3]),
                "keys": _log_uniform(rng, 16, min(4096, 16384 // parents)), "spread": rng.choice([1.0, 1.3, 2.0]), "layout": layout}
    parents = _log_uniform(rng, 1, 16)
    return {"op": op, "shape": shape, "parents": parents, "children": rng.randint(1, 4), "keys": _log_uniform(rng, 16, min(4096, 16384 // parents)),
            "prefix": rng.choice([1.0, 1.0, 0.9, 0.3]), "room": rng.choice([0.5, 0.9, 1.0, 1.5]),
            "keep": rng.choice([0.0, 0.7, 0.9]) if op == "branch" else 0.0, "layout": layout}


# ---- what a call is made of --------------------------------------------------------------------

def _around(rng, middle, sigma, least, most):
    return int(min(max(middle * math.exp(rng.gauss(0.0, sigma)), least), most))


def _pages(tokens):
    return -(-tokens // PAGE)


def _new_rows(case):
    """norm: per sequence (tokens in the cache before the step, tokens of the step).  Part of the case, not of the seed."""
    rng, out = random.Random(case["layout"]), []
    for _ in range(case["seqs"]):
        new = case["new"] if case["new"] == 1 or case["seqs"] == 1 else _around(rng, case["new"], 0.5, 1, 8192)
        held = case["held"] if case["seqs"] == 1 else _around(rng, case["held"], 0.6, 0, 8192)
        out.append((held, new))
    return out


def _family(case):
    """fork, branch, compact: the parents' lengths, and per child (parent, tokens that it takes over: -1 all, tokens that it keeps)."""
    rng, lens, children = random.Random(case["layout"]), [], []
    for _ in range(case["parents"]):
        lens.append(case["keys"] if case["parents"] == 1 else _around(rng, case["keys"], 0.5, 1, min(8192, 2 * case["keys"])))
    for i in range(case["parents"] * case["children"]):
        p, prefix = i % case["parents"], case.get("prefix", 1.0)
        n = -1 if prefix == 1.0 else int(lens[p] * prefix * rng.uniform(0.9, 1.0))
        t = lens[p] if n < 0 else n
        children.append((p, n, min(int(t * case.get("keep", 0.0) * rng.uniform(0.9, 1.0)), t - t % PAGE)))   # none of its own page
    return lens, children


def _logit_rows(case):
    """Per sequence (tokens of its prompt, tokens of its history, rows of the step, biases)."""
    rng, out = random.Random(case["layout"]), []
    for _ in range(case["seqs"]):
        n = case["history"] if case["seqs"] == 1 else _around(rng, case["history"], 0.6, 0, 8192)
        rows = {"one": 1, "draft16": 17, "drafts": rng.randint(2, 33)}[case["rows"]]
        out.append((int(n * rng.uniform(0.3, 1.0)), n, rows, rng.randint(0, 2 * case["biases"])))
    return out


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def _zeros(*shape):
    return torch.zeros(shape, dtype=torch.int32, device=DEV)


def _angles(rotary_dim, positions):
    """cos and sin of the rotary angles, [positions, rotary_dim / 2, 2], angles taken in 64 bits: the plan a program keeps."""
    freq = 1e6 ** (-torch.arange(0, rotary_dim, 2, dtype=torch.float64, device=DEV) / rotary_dim)
    a = torch.arange(positions, dtype=torch.float64, device=DEV)[:, None] * freq
    return torch.stack((a.cos(), a.sin()), -1).float().contiguous()


def _prepare_norm(case, s, rng, gen):
    reqs = _new_rows(case)
    s.total, s.eps = sum(w for _, w in reqs), 1e-6
    s.hq, s.hkv, s.hd, _, _, dtype = SHAPES[case["shape"]]
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    pages = sum(_pages(h + w) for h, w in reqs)
    perm = list(range(pages))
    rng.shuffle(perm)

    def normal(*shape, std):
        return torch.empty(shape, dtype=dt, device=DEV).normal_(0.0, std, generator=gen)

    def gain(heads):
        if case["gains"] == "none":
            return None
        return 1.0 + 0.2 * torch.randn((heads, s.hd) if case["gains"] == "heads" else (s.hd,), generator=gen, device=DEV)
    s.pool = normal(pages, 2, s.hkv, PAGE * s.hd, std=1.5)
    # q, k and v are the columns of one matrix, as the projection leaves them
    qkv = normal(s.total, (s.hq + 2 * s.hkv) * s.hd, std=1.5).view(s.total, s.hq + 2 * s.hkv, s.hd)
    s.q, s.k, s.v = qkv[:, :s.hq], qkv[:, s.hq:s.hq + s.hkv], qkv[:, s.hq + s.hkv:]
    s.q_gain, s.k_gain = gain(s.hq), gain(s.hkv)
    s.q_out = torch.empty((s.total, s.hq, s.hd), dtype=dt, device=DEV)
    s.rotary_dim, s.pairs = int(s.hd * case["part"]), case["pairs"]
    s.angles = _angles(s.rotary_dim, max(h + w for h, w in reqs))
    pos, slot, first = [], [], 0
    for h, w in reqs:
        pos += range(h, h + w)
        slot += [PAGE * perm[first + t // PAGE] + t % PAGE for t in range(h, h + w)]
        first += _pages(h + w)
    s.pos, s.slot = _i32(pos), _i32(slot)


def _prepare_pages(case, s, rng, gen):
    hq, hkv, hd, layers, _, dtype = SHAPES[case["shape"]]
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    lens, children = _family(case)
    n, held = len(lens) + len(children), sum(_pages(h) for h in lens)
    width = _pages(max(lens)) + 1
    if s.op == "compact":       # the children share their parents' full pages and have their own last ones
        own_pages = sum(lens[p] % PAGE > 0 for p, _, _ in children)
        pages = int((held + own_pages) * case["spread"])
        perm = list(range(pages))
        rng.shuffle(perm)
        rows, shares = [], [0] * pages
        for h in lens:
            rows.append(perm[:_pages(h)])
            del perm[:_pages(h)]
        for p, _, _ in children:
            rows.append(rows[p][:lens[p] // PAGE] + perm[:lens[p] % PAGE > 0])
            del perm[:lens[p] % PAGE > 0]
            for page in rows[p][:lens[p] // PAGE]:
                shares[page] += 1
        lens = lens + [lens[p] for p, _, _ in children]
        s.lens, s.shares, s.table = _i32(lens), _i32(shares), _i32([r + [-1] * (width - len(r)) for r in rows])
        s.table_out, room = torch.full_like(s.table, -1), held + own_pages + 3
        s.shares_out, s.free_out, s.n_free_out, s.moved = _zeros(room), _zeros(room), _zeros(1), _zeros(pages)
        s.copies, s.n_copies = _zeros(pages, 2), _zeros(1)
        s.to = torch.zeros((layers, room, 2, hkv, PAGE * hd), dtype=dt, device=DEV)
    else:                       # the children's places are empty; requests and pages in a pool that others use too
        wanted = sum((lens[p] if t < 0 else t) % PAGE > 0 for p, t, _ in children)
        free = int(wanted * case["room"])
        pages = held + free
        perm = list(range(pages))
        rng.shuffle(perm)
        rows = []
        for h in lens:
            rows.append(perm[:_pages(h)] + [-1] * (width - _pages(h)))
            del perm[:_pages(h)]
        rows += [[-1] * width for _ in children]
        s.lens, s.table, s.shares = _i32(lens + [0] * len(children)), _i32(rows), _zeros(pages)
        s.free, s.n_free = _i32(perm + [0] * held), _i32([free])
        s.src, s.tokens = _i32([p for p, _, _ in children]), _i32([t for _, t, _ in children])
        s.dst = _i32([n - 1 - i for i in range(len(children))])
        s.kv_len, s.n_free_after, s.copies, s.n_copies = _zeros(n), _zeros(1), _zeros(len(children), 2), _zeros(1)
        s.keep = _i32([-1] * len(lens) + [k for _, _, k in reversed(children)])
        s.kept, s.n_free_kept, s.more, s.n_more = _zeros(n), _zeros(1), _zeros(n, 2), _zeros(1)
    s.pools = torch.empty((layers, pages, 2, hkv, PAGE * hd), dtype=dt, device=DEV).normal_(0.0, 1.5, generator=gen)


def _prepare_logits(case, s, rng, gen):
    reqs, vocab = _logit_rows(case), case["vocab"]
    n, total, longest = len(reqs), sum(r for _, _, r, _ in reqs), max(1, max(h for _, h, _, _ in reqs))
    s.vocab, s.max_rows = vocab, max(r for _, _, r, _ in reqs)

    def ids(*shape):            # few tokens often, many seldom
        u = torch.rand(shape, generator=gen, device=DEV)
        return (u.pow(4) * vocab).int().clamp(max=vocab - 1)
    s.logits = torch.randn((total, vocab), generator=gen, device=DEV).mul_(4.0).to(torch.bfloat16 if case["dtype"] == "bf16" else torch.float32)
    s.out = torch.empty((total, vocab), dtype=torch.float32, device=DEV)
    off = [0]
    for _, _, r, _ in reqs:
        off.append(off[-1] + r)
    s.row_off, s.tokens = _i32(off), ids(total)
    s.penalties = s.history = s.history_len = s.prompt_len = s.biases = s.mask = s.mask_row = None
    if case["penalties"]:
        # repetition, presence, frequency; every fifth request has none
        r = torch.rand((n, 3), generator=gen, device=DEV)
        p = torch.stack((1.0 + 0.3 * r[:, 0], r[:, 1], 0.5 * r[:, 2]), -1)
        at = torch.arange(n, device=DEV) % 5 == 4
        p[at] = torch.tensor([1.0, 0.0, 0.0], device=DEV)
        s.penalties, s.history = p.contiguous(), ids(n, longest)
        s.prompt_len, s.history_len = _i32([p for p, _, _, _ in reqs]), _i32([h for _, h, _, _ in reqs])
    if case["biases"]:
        some = [torch.randperm(vocab, generator=gen, device=DEV)[:min(m, vocab)] for _, _, _, m in reqs]
        offs = [0]
        for x in some:
            offs.append(offs[-1] + x.numel())
        at = torch.cat(some).int()
        s.biases = (_i32(offs), at, torch.randn(at.numel(), generator=gen, device=DEV).mul_(3.0))
    if case["allowed"] < 1.0:
        words = -(-vocab // 32)
        bits = torch.rand((total, words, 32), generator=gen, device=DEV) < case["allowed"]
        words = (bits.long() << torch.arange(32, device=DEV)).sum(-1)
        s.mask = torch.where(words >= 1 << 31, words - (1 << 32), words).int()
        # every row has a state of its grammar; every seventh is outside of it
        s.mask_row = _i32([-1 if r % 7 == 6 else r for r in range(total)])


def prepare(case, seed):
    rng, gen = random.Random(int(seed)), torch.Generator(device=DEV).manual_seed(int(seed))
    s = SimpleNamespace(op=case["op"])
    {"norm": _prepare_norm, "logits": _prepare_logits}.get(s.op, _prepare_pages)(case, s, rng, gen)
    return s


# ---- the plain forms ---------------------------------------------------------------------------

def _keys_of(pool, hd):
    """K of pages [..., heads, 64 * hd] as [..., heads, tile, eight keys, half, key, depth block, group, element]."""
    k = pool.unflatten(-1, (2, 2, hd // 32, 4, 4, 4, 8))
    d = k.dim() - 7
    return k.permute(*range(d), d, d + 4, d + 1, d + 5, d + 2, d + 3, d + 6)


def _values_of(pool, hd):
    """V of pages [..., heads, 64 * hd] as [..., heads, tile, eight keys, key, depth block, element]."""
    v = pool.unflatten(-1, (2, hd // 16, 4, 16, 8))
    d = v.dim() - 5
    return v.permute(*range(d), d, d + 2, d + 4, d + 1, d + 3)


def _plain_norm_rotate(s, x, gain):
    x, a, r = x.float(), s.angles[s.pos.long()][:, None], s.rotary_dim
    x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + s.eps)
    if gain is not None:
        x = x * gain
    part, rest = x[..., :r], x[..., r:]
    lo, hi = (part[..., :r // 2], part[..., r // 2:]) if s.pairs == "half" else (part[..., 0::2], part[..., 1::2])
    c, n = a[..., 0], a[..., 1]
    turned = (lo * c - hi * n, hi * c + lo * n)
    part = torch.cat(turned, -1) if s.pairs == "half" else torch.stack(turned, -1).flatten(-2)
    return torch.cat((part, rest), -1)


def _plain_norm(s):
    s.q_out.copy_(_plain_norm_rotate(s, s.q, s.q_gain))
    page, key = s.slot.long() // PAGE, s.slot.long() % PAGE
    k, v = _keys_of(s.pool[:, 0], s.hd), _values_of(s.pool[:, 1], s.hd)
    rows = _plain_norm_rotate(s, s.k, s.k_gain).to(s.pool.dtype)
    k.movedim(1, 5)[page, key // 32, key // 8 % 4, key // 4 % 2, key % 4] = rows.unflatten(-1, (s.hd // 32, 4, 8))
    v.movedim(1, 4)[page, key // 32, key // 8 % 4, key % 8] = s.v.unflatten(-1, (s.hd // 16, 16))
    return {"q": s.q_out, "pool": s.pool}


def _plain_copy(pools, copies, n_copies, to):
    pair = copies[torch.arange(copies.shape[0], device=DEV) < n_copies].long()
    to[:, pair[:, 1]] = pools[:, pair[:, 0]]


def _plain_fork(s):
    width, n_free = s.table.shape[1], s.n_free.long()
    src, dst, at = s.src.long(), s.dst.long(), torch.arange(s.table.shape[1], device=DEV)
    held = s.lens.long()[src]
    t = torch.where((s.tokens < 0) | (s.tokens > held), held, s.tokens.long())
    need = (t % PAGE > 0).long()
    upto = need.cumsum(0)
    ok = (need == 0) | (upto <= n_free)
    last = t // PAGE
    fresh = s.free[(n_free - upto).clamp(min=0)]
    rows = s.table[src]
    shared = (at < last[:, None]) & ok[:, None]
    s.shares.index_add_(0, rows.long().clamp(min=0).flatten(), shared.flatten().int())
    mine = (at == last[:, None]) & (ok & (need > 0))[:, None]
    s.table[dst] = torch.where(shared, rows, torch.where(mine, fresh[:, None], s.table[dst]))
    s.kv_len.copy_(s.lens)
    s.kv_len[dst] = torch.where(ok, t, 0).int()
    took = ok & (need > 0)
    pair = torch.stack((rows.gather(1, last.clamp(max=width - 1)[:, None])[:, 0], fresh), -1)
    s.copies[(upto - 1)[took]] = pair[took]
    s.n_copies.copy_(torch.minimum(upto[-1:], n_free))
    s.n_free_after.copy_(n_free - s.n_copies)
    _plain_copy(s.pools, s.copies, s.n_copies, s.pools)
    return {"table": s.table, "shares": s.shares, "kv_len": s.kv_len, "copies": s.copies, "n_copies": s.n_copies,
            "n_free": s.n_free_after, "pools": s.pools}


def _plain_keep(s):
    n, width = s.table.shape
    at, pool = torch.arange(width, device=DEV), s.shares.numel()
    held, never = s.kv_len.long(), n * width
    keep = torch.where((s.keep < 0) | (s.keep > held), held, s.keep.long())
    first, last = (keep + PAGE - 1) // PAGE, (held + PAGE - 1) // PAGE
    gone = (at >= first[:, None]) & (at < last[:, None]) & (s.table >= 0)
    page = torch.where(gone, s.table, 0).long().flatten()
    shares = s.shares.long().index_add(0, page, -gone.flatten().long())
    # a page that its last holder gives back goes on the list, in the order in which the requests first name it
    order = torch.where(gone, torch.arange(never, device=DEV).view(n, width), never).flatten()
    named = torch.full((pool,), never, device=DEV).scatter_reduce(0, page, order, "amin")
    freed = (shares < 0) & (named < never)
    by_name = torch.where(freed, named, never + 1).argsort()
    n_freed, n_free, place = freed.sum(), s.n_free_after.long(), torch.arange(s.free.numel(), device=DEV)
    new = (place >= n_free) & (place < n_free + n_freed)
    free = torch.where(new, by_name[(place - n_free).clamp(0, pool - 1)].int(), s.free)
    n_free, shares = n_free + n_freed, shares.clamp(min=0)
    # a shared page that a request keeps a part of: all but its last holder get a copy
    end = (keep // PAGE).clamp(max=width - 1)
    kept = s.table.gather(1, end[:, None])[:, 0].long()
    cut = (keep < held) & (keep % PAGE > 0) & (kept >= 0)
    kept = kept.clamp(min=0)
    cuts = torch.zeros_like(shares).index_add(0, kept, cut.long())
    b = torch.arange(n, device=DEV)
    latest = torch.full((pool,), -1, device=DEV).scatter_reduce(0, kept, torch.where(cut, b, -1), "amax")
    copied = cut & ~((cuts[kept] > shares[kept]) & (latest[kept] == b))
    shares = shares.index_add(0, kept, -copied.long())
    upto = copied.long().cumsum(0)
    ok = copied & (upto <= n_free)
    fresh = free[(n_free - upto).clamp(min=0)]
    s.more[(upto - 1)[ok]] = torch.stack((kept.int(), fresh), -1)[ok]
    s.n_more.copy_(torch.minimum(upto[-1:], n_free))
    ends = (at == end[:, None]) & copied[:, None]
    s.table.copy_(torch.where(ends, torch.where(ok, fresh, -1)[:, None], torch.where(gone, -1, s.table)))
    s.kept.copy_(torch.where(copied & ~ok, keep // PAGE * PAGE, keep))
    s.n_free_kept.copy_(n_free - s.n_more)
    s.free.copy_(free)
    s.shares.copy_(shares)


def _plain_branch(s):
    out = _plain_fork(s)
    _plain_keep(s)
    _plain_copy(s.pools, s.more, s.n_more, s.pools)
    return {**out, "kept": s.kept, "free": s.free, "more": s.more, "n_more": s.n_more, "n_free_kept": s.n_free_kept}


def _plain_compact(s):
    pages, room, at = s.shares.numel(), s.shares_out.numel(), torch.arange(s.table.shape[1], device=DEV)
    there = (at < ((s.lens.long() + PAGE - 1) // PAGE)[:, None]) & (s.table >= 0)
    held = torch.zeros(pages, device=DEV).index_add(0, s.table.long().clamp(min=0).flatten(), there.flatten().float()) > 0
    rank = held.long().cumsum(0) - 1
    s.moved.copy_(torch.where(held & (rank < room), rank, -1))
    s.table_out.copy_(torch.where(there, s.moved[s.table.long().clamp(min=0)], -1))
    live, place = held.long().sum(), torch.arange(room, device=DEV)
    old = held.nonzero()[:, 0][:room]
    s.copies[:old.numel()] = torch.stack((old, torch.arange(old.numel(), device=DEV)), -1).int()
    s.n_copies.copy_(live.clamp(max=room))
    s.shares_out.zero_()
    s.shares_out[:old.numel()] = s.shares[old]
    s.free_out.copy_(torch.where(place < room - live, place + live, s.free_out))
    s.n_free_out.copy_((room - live).clamp(min=0))
    _plain_copy(s.pools, s.copies, s.n_copies, s.to)
    return {"table": s.table_out, "shares": s.shares_out, "free": s.free_out, "n_free": s.n_free_out, "moved": s.moved,
            "copies": s.copies, "n_copies": s.n_copies, "to": s.to}


def _plain_logits(s):
    total, vocab, off = s.logits.shape[0], s.vocab, s.row_off.long()
    z, row = s.logits.float(), torch.arange(s.logits.shape[0], device=DEV)
    seq = torch.searchsorted(off, row, right=True) - 1
    if s.penalties is not None:
        at, n = torch.arange(s.history.shape[1], device=DEV), off.numel() - 1
        there = at < s.history_len[:, None]
        ids = torch.where(there, s.history, vocab).long()
        out = there & (at >= s.prompt_len[:, None])
        every = torch.zeros((n, vocab + 1), dtype=torch.int32, device=DEV).scatter_add(1, ids, there.int())
        given = torch.zeros_like(every).scatter_add(1, ids, out.int())
        back = row[:, None] - torch.arange(s.max_rows, device=DEV)          # a row comes after the tokens of the rows before it
        mine = back >= off[seq][:, None]
        ids = torch.where(mine, s.tokens[back.clamp(min=0)], vocab).long()
        drafts = torch.zeros((total, vocab + 1), dtype=torch.int32, device=DEV).scatter_add(1, ids, mine.int())
        seen = (every[seq] + drafts)[:, :vocab] > 0
        count = (given[seq] + drafts)[:, :vocab]
        rep, presence, frequency = (p[:, None] for p in s.penalties[seq].unbind(-1))
        z = torch.where(seen, torch.where(z > 0, z / rep, z * rep), z)
        z = torch.where(count > 0, z - (presence + frequency * count), z)
    if s.biases is not None:
        offs, ids, values = s.biases
        whose = torch.searchsorted(offs.long(), torch.arange(ids.numel(), device=DEV), right=True) - 1
        bias = torch.zeros((off.numel() - 1, vocab), device=DEV)
        bias[whose, ids.long()] = values
        z = z + bias[seq]
    if s.mask is not None:
        bit = torch.arange(vocab, device=DEV)
        allowed = (s.mask[s.mask_row.long().clamp(min=0)][:, bit // 32] >> (bit % 32)) & 1
        z = torch.where((allowed > 0) | (s.mask_row < 0)[:, None], z, -math.inf)
    s.out.copy_(z)
    return s.out


# ---- one pass ----------------------------------------------------------------------------------

def run(s):
    if not own:
        return {"norm": _plain_norm, "fork": _plain_fork, "branch": _plain_branch, "compact": _plain_compact,
                "logits": _plain_logits}[s.op](s)
    import paper_2510_15312_amd as vf
    if s.op == "norm":
        vf.vf_norm_rotary_append(s.q, s.k, s.v, s.q_gain, s.k_gain, s.eps, s.angles, s.pos, s.slot, s.q_out, s.pool,
                                 vf.VF_ROTARY_HALF if s.pairs == "half" else vf.VF_ROTARY_INTERLEAVED)
        return {"q": s.q_out, "pool": s.pool}
    if s.op == "logits":
        vf.vf_logits_adjust(s.logits, s.row_off, s.out, s.penalties, s.history, s.history_len, s.prompt_len, s.tokens, s.biases,
                            s.mask, s.mask_row)
        return s.out
    if s.op == "compact":
        vf.vf_pages_compact(s.lens, s.table, s.shares, s.table_out, s.shares_out, s.free_out, s.n_free_out, s.moved, s.copies, s.n_copies)
        vf.vf_pages_copy(s.pools, s.copies, s.n_copies, s.to)
        return {"table": s.table_out, "shares": s.shares_out, "free": s.free_out, "n_free": s.n_free_out, "moved": s.moved,
                "copies": s.copies, "n_copies": s.n_copies, "to": s.to}
    vf.vf_pages_fork(s.src, s.dst, s.tokens, s.lens, s.free, s.n_free, s.table, s.shares, s.kv_len, s.n_free_after, s.copies, s.n_copies)
    vf.vf_pages_copy(s.pools, s.copies, s.n_copies, s.pools)
    out = {"table": s.table, "shares": s.shares, "kv_len": s.kv_len, "copies": s.copies, "n_copies": s.n_copies,
           "n_free": s.n_free_after, "pools": s.pools}
    if s.op == "fork":
        return out
    vf.vf_pages_keep(s.kv_len, s.keep, s.free, s.n_free_after, s.table, s.shares, s.kept, s.n_free_kept, s.more, s.n_more)
    vf.vf_pages_copy(s.pools, s.more, s.n_more, s.pools)
    return {**out, "kept": s.kept, "free": s.free, "more": s.more, "n_more": s.n_more, "n_free_kept": s.n_free_kept}


# ---- the definition in 64 bits -----------------------------------------------------------------

def _k_place(hd):
    """Offset of K[key][d] inside a page's block of one head."""
    key, d = torch.arange(PAGE, device=DEV)[:, None], torch.arange(hd, device=DEV)[None, :]
    low = key % 32
    frag = ((key // 32) * 2 + low % 8 // 4) * (hd // 32) + d // 32
    return (frag * 64 + d % 32 // 8 * 16 + low // 8 * 4 + low % 4) * 8 + d % 8


def _v_place(hd):
    key, d = torch.arange(PAGE, device=DEV)[:, None], torch.arange(hd, device=DEV)[None, :]
    frag = (key // 32) * (hd // 16) + d // 16
    return (frag * 64 + key % 32 // 8 * 16 + d % 16) * 8 + key % 8


def exact(case, seed):
    if case["op"] not in ("norm", "logits"):
        return None                                     # whole numbers and copies
    s = prepare(case, seed)
    if s.op == "norm":
        pool, pos, r = s.pool.double(), s.pos.long(), s.rotary_dim
        i = torch.arange(r // 2, device=DEV)
        a, b = (i, i + r // 2) if s.pairs == "half" else (2 * i, 2 * i + 1)
        c, n = s.angles.double()[pos].unbind(-1)
        c, n = c[:, None], n[:, None]

        def turned(x, gain):
            x = x.double()
            x = x / (x.pow(2).sum(-1, keepdim=True) / s.hd + s.eps).sqrt()
            x = x if gain is None else x * gain.double()
            y = x.clone()
            y[..., a] = x[..., a] * c - x[..., b] * n
            y[..., b] = x[..., b] * c + x[..., a] * n
            return y
        page, key = s.slot.long() // PAGE, s.slot.long() % PAGE
        k = turned(s.k, s.k_gain)
        for h in range(s.hkv):
            pool[page[:, None], 0, h, _k_place(s.hd)[key]] = k[:, h]
            pool[page[:, None], 1, h, _v_place(s.hd)[key]] = s.v[:, h].double()
        return {"q": turned(s.q, s.q_gain), "pool": pool}
    out, off = s.logits.double(), s.row_off.tolist()
    hist_len, prompt_len = (x.tolist() if x is not None else None for x in (s.history_len, s.prompt_len))
    offs, mask_row = (s.biases[0].tolist() if s.biases else None), (s.mask_row.tolist() if s.mask is not None else None)
    shift = torch.arange(32, device=DEV)
    for b in range(len(off) - 1):
        for r in range(off[b], off[b + 1]):
            z = out[r]
            if s.penalties is not None:
                rep, presence, frequency = s.penalties[b].tolist()
                text = torch.cat((s.history[b, :hist_len[b]], s.tokens[off[b]:r + 1])).long()
                given = torch.bincount(text[min(prompt_len[b], hist_len[b]):], minlength=s.vocab).double()
                seen = torch.unique(text)
                z[seen] = torch.where(z[seen] > 0, z[seen] / rep, z[seen] * rep)
                z -= presence * (given > 0) + frequency * given
            if offs is not None:
                z[s.biases[1][offs[b]:offs[b + 1]].long()] += s.biases[2][offs[b]:offs[b + 1]].double()
            if mask_row is not None and mask_row[r] >= 0:
                bits = (s.mask[mask_row[r]].long()[:, None] >> shift & 1).flatten()[:s.vocab]
                z[bits == 0] = -math.inf
    return out


# ---- what a pass cannot do without -------------------------------------------------------------

def work(case):
    if case["op"] == "logits":
        reqs = _logit_rows(case)
        rows = sum(r for _, _, r, _ in reqs)
        per_row = case["vocab"] * ((4 if case["dtype"] == "f32" else 2) + 4 + (0.125 if case["allowed"] < 1.0 else 0.0))
        read = (4.0 * sum(h for _, h, _, _ in reqs) if case["penalties"] else 0.0) + (8.0 * sum(m for _, _, _, m in reqs) if case["biases"] else 0.0)
        return {"bytes": rows * per_row + read, "flops": 3.0 * rows * case["vocab"]}
    hq, hkv, hd, layers, _, dtype = SHAPES[case["shape"]]
    es = 2 if dtype == "bf16" else 4
    if case["op"] == "norm":
        reqs = _new_rows(case)
        total, half = sum(w for _, w in reqs), int(hd * case["part"]) // 2
        angles = min(total, max(h + w for h, w in reqs)) * half * 8
        return {"bytes": 2.0 * es * total * (hq + 2 * hkv) * hd + 8.0 * total + angles,
                "flops": 4.0 * total * (hq + hkv) * hd + 6.0 * total * (hq + hkv) * half}
    lens, children = _family(case)
    page = es * layers * 2 * hkv * PAGE * hd
    if case["op"] == "compact":
        held = sum(_pages(h) for h in lens) + sum(lens[p] % PAGE > 0 for p, _, _ in children)
        entries = sum(_pages(h) for h in lens) + sum(_pages(lens[p]) for p, _, _ in children)
        return {"bytes": 2.0 * page * held + 8.0 * entries + 8.0 * held, "flops": 0.0}
    takes = [lens[p] if t < 0 else t for p, t, _ in children]
    wanted = sum(t % PAGE > 0 for t in takes)
    free = int(wanted * case["room"])
    copied = min(wanted, free)
    entries = sum(_pages(t) for t in takes)
    small = 8.0 * entries + 8.0 * len(lens) + 20.0 * len(children)
    if case["op"] == "fork":
        return {"bytes": 2.0 * page * copied + small, "flops": 0.0}
    # the forks' own pages come back where they are cut off; those that are cut inside a page that they share get another copy
    left, again = free, 0
    for (_, _, k), t in zip(children, takes):
        granted = t % PAGE == 0 or left > 0
        left -= granted and t % PAGE > 0
        again += granted and k % PAGE > 0 and _pages(k) <= t // PAGE
    return {"bytes": 2.0 * page * (copied + again) + 2 * small, "flops": 0.0}
