"""What is timed of the operators that verify trees of drafted tokens with all lengths on the GPU: page tables and slot maps, attention
of a tree over the cache, the path that is accepted with the move of its keys and values, and adjusted logits.

Kinds of case
  pages      update_pages: pages taken for a step's tokens, tables and slot maps; then those behind the kept tokens given back
  attention  TreeBatch.attention: trees behind cached contexts of the paged cache
  commit     TreeBatch.accept and .commit: the path that the targets follow, and its keys and values moved together in every layer
  logits     adjust_logits: penalties for tokens seen before, biases and grammar masks
Head counts and widths are those of the shapes in workloads/shapes.py (4/4 x 64, 32/8 x 128, 64/8 x 128) or generic, lengths those of
its recipes.  Everything else follows from the case and the seed.  `run` computes a case in plain torch operations, or, where `own` is
set, by the package's calls."""
import math
import random
from types import SimpleNamespace

import numpy as np
import torch

own = False

PAGE = 16
MOST_NODES = 256
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}
ERANGE, ENOSPC = -2, -3


# ------------------------------------------------------------------------------------------------ the cases
def _pages(batch, ctx, new, columns, spare=1.0, lengths=1):
    """ctx, new = (low, high) of cached lengths and of a step's tokens; spare: free pages for this share of what is asked for."""
    return {"kind": "pages", "batch": batch, "ctx_lo": ctx[0], "ctx_hi": ctx[1], "new_lo": new[0], "new_hi": new[1], "columns": columns,
            "spare": spare, "lengths": lengths}


def _attention(batch, heads, ctx, nodes, shape="tree", lse=False, lengths=1):
    hq, hkv, hd = heads
    return {"kind": "attention", "batch": batch, "hq": hq, "hkv": hkv, "hd": hd, "ctx_lo": ctx[0], "ctx_hi": ctx[1], "new_lo": nodes[0],
            "new_hi": nodes[1], "shape": shape, "lse": lse, "lengths": lengths}


def _commit(batch, layers, heads, ctx, nodes, match, shape="tree", lengths=1):
    """match: how often a target is the token of one of its node's children."""
    hq, hkv, hd = heads
    return {"kind": "commit", "batch": batch, "layers": layers, "hq": hq, "hkv": hkv, "hd": hd, "ctx_lo": ctx[0], "ctx_hi": ctx[1],
            "new_lo": nodes[0], "new_hi": nodes[1], "match": match, "shape": shape, "lengths": lengths}


def _logits(batch, nodes, vocab, dtype, history, biases=0, allowed=1.0, shape="tree", pitch=0, lengths=1):
    """nodes = (low, high) rows of a request, (0, 0): one row without a tree; history = (low, high) tokens; allowed: share of the
    vocabulary that a mask leaves (1: no mask); pitch: elements from row to row (0: the vocabulary)."""
    return {"kind": "logits", "batch": batch, "new_lo": nodes[0], "new_hi": nodes[1], "vocab": vocab, "dtype": dtype, "ctx_lo": history[0],
            "ctx_hi": history[1], "biases": biases, "allowed": allowed, "shape": shape, "pitch": pitch or vocab, "lengths": lengths}


TINY, WIDE8, WIDE64 = (4, 4, 64), (32, 8, 128), (64, 8, 128)


def listed():
    return [
        # one decoding step of a few requests: all latency
        {"name": "pages_8", **_pages(8, (32, 2048), (1, 9), 160)},
        # a large batch of prompts' pieces, some behind long contexts, from a pool that has pages for most of them
        {"name": "pages_1024_pieces", **_pages(1024, (0, 8192), (1, 512), 544, spare=0.9)},
        # the small decoder: trees of eight nodes
        {"name": "attention_tiny_4", **_attention(4, TINY, (32, 128), (8, 8), lse=True)},
        # one reader of a long document, a tree of some dozen nodes behind it
        {"name": "attention_1_long", **_attention(1, WIDE8, (31000, 31000), (26, 26))},
        # the headline batch's contexts with trees in place of chunks
        {"name": "attention_64_trees", **_attention(64, WIDE8, (128, 4096), (8, 64))},
        # many requests of long-tailed contexts, few nodes each
        {"name": "attention_256_few", **_attention(256, WIDE8, (64, 8192), (1, 8))},
        # the larger decoder, wide trees, its statistics wanted too
        {"name": "attention_32_wide", **_attention(32, WIDE64, (1024, 4096), (48, 160), shape="wide", lse=True)},
        # the small decoder's two layers
        {"name": "commit_tiny_4", **_commit(4, 2, TINY, (32, 128), (8, 8), 0.7)},
        # trees of a whole 8B shape's layers; short contexts, since only the pages with nodes are touched
        {"name": "commit_64x32", **_commit(64, 32, WIDE8, (0, 48), (8, 32), 0.7)},
        # one row each of a few requests in a small vocabulary, as in plain sampling
        {"name": "logits_4", **_logits(4, (0, 0), 4096, "f32", (32, 128))},
        # the verified rows of the headline batch: history and path penalized, some tokens biased
        {"name": "logits_64_trees", **_logits(64, (1, 16), 32000, "f32", (128, 4096), biases=16)},
        # many rows of a large vocabulary under a grammar, rows of an odd pitch
        {"name": "logits_256_masked", **_logits(256, (8, 8), 128256, "bf16", (64, 8192), biases=3, allowed=0.03, shape="chain", pitch=128261)},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _heads(rng):
    if rng.random() < 0.6:
        return rng.choice((TINY, WIDE8, WIDE64))
    hkv = rng.choice((1, 2, 3, 5, 8))
    return (hkv * rng.choice((1, 2, 3, 7, 12, 16)), hkv, rng.choice((64, 128)))


def draw(rng):
    what = rng.random()
    lengths = rng.randrange(2, 1 << 20)
    shape = rng.choice(("tree", "tree", "wide", "chain"))
    if what < 0.25:
        b = _log(rng, 1, 1024)
        ctx, new = _log(rng, 16, 8192), _log(rng, 1, 512)
        return _pages(b, (rng.choice((0, ctx // 4)), ctx), (rng.choice((0, 1, new)), new), (ctx + new) // PAGE + 2 + rng.randrange(64),
                      rng.choice((0.3, 0.9, 1.0, 2.0)), lengths)
    if what < 0.6:
        heads = _heads(rng)
        b = _log(rng, 1, 256)
        # keys and scores that the plain form lays out for the whole batch stay below those of the largest listed cases
        ctx = _log(rng, 16, max(17, min(32000, (400 << 20) // (b * heads[1] * heads[2]))))
        nodes = _log(rng, 1, max(2, min(MOST_NODES, (1 << 30) // (b * heads[0] * (ctx + 64)))))
        nodes = min(nodes, max(1, int(0.25e12 / (4.0 * b * heads[0] * heads[2] * (ctx + nodes)))))
        return _attention(b, heads, (rng.choice((0, ctx // 4, ctx)), ctx), (rng.choice((0, 1, nodes)), nodes), shape, rng.random() < 0.5, lengths)
    if what < 0.75:
        heads = _heads(rng)
        b = _log(rng, 1, 128)
        nodes = _log(rng, 1, 128)
        ctx = _log(rng, 1, 100)
        most = max(1, (256 << 20) // (b * (ctx + nodes + PAGE) * 2 * heads[1] * heads[2] * 2))
        return _commit(b, _log(rng, 1, min(80, most)), heads, (rng.choice((0, ctx)), ctx), (rng.choice((1, nodes)), nodes),
                       rng.choice((0.0, 0.5, 0.8, 1.0)), shape, lengths)
    vocab = _log(rng, 1000, 160000)
    dtype = rng.choice(("f32", "bf16", "f16"))
    rows = _log(rng, 1, max(1, (64 << 20) // vocab))
    nodes = rng.choice((0, 1, 4, 16, 64))
    b = max(1, min(512, rows // max(1, nodes)))
    hist = _log(rng, 1, 16384)
    return _logits(b, (rng.choice((min(1, nodes), nodes)), nodes), vocab, dtype, (rng.choice((0, hist)), hist), rng.choice((0, 1, 20, 300)),
                   rng.choice((1.0, 1.0, 0.5, 0.01)), shape, vocab + rng.choice((0, 0, 1, 7, 64)), lengths)


# ------------------------------------------------------------------------------------------------ inputs
def _lengths(case):
    """Cached tokens and new ones (nodes) of each request."""
    rng = np.random.Generator(np.random.PCG64(case["lengths"]))
    b, lo, hi = case["batch"], case["ctx_lo"], case["ctx_hi"]
    ctx = np.rint(np.exp(rng.uniform(math.log(max(lo, 1)), math.log(max(hi, 1)), size=b))).astype(np.int64)
    ctx = np.clip(np.where((lo == 0) & (rng.random(b) < 0.1), 0, ctx), lo, hi)
    new = rng.integers(case["new_lo"], case["new_hi"] + 1, size=b)
    if not new.any():
        new[0] = case["new_hi"]
    return ctx, new


def _parents(case, new):
    """The parent of each node inside its request, -1 for children of the context; request after request."""
    rng = np.random.Generator(np.random.PCG64(case["lengths"] + 7))
    at = np.arange(int(new.sum())) - np.repeat(np.cumsum(new) - new, new)
    if case["shape"] == "chain":
        return at - 1
    # the first node is the last token that was emitted, so all others hang on it; trees grow at their later nodes
    back = rng.integers(1, 9, size=len(at)) if case["shape"] == "tree" else rng.integers(1, 129, size=len(at))
    return np.where(at == 0, -1, np.maximum(at - back, 0))


def _ancestors(parent, new):
    """[sum new][widest]: whether a node's path from the root, itself included, goes through node k of its request."""
    widest = max(1, int(new.max(initial=0)))
    out = np.zeros((len(parent), widest), bool)
    begin = np.repeat(np.cumsum(new) - new, new)
    at = np.arange(len(parent)) - begin
    for k in range(widest):
        rows = np.nonzero(at == k)[0]
        up = parent[rows]
        out[rows] = np.where((up >= 0)[:, None], out[begin[rows] + np.maximum(up, 0)], False)
        out[rows, k] = True
    return out


def _table(case, ctx, new, columns=0):
    """Page table of as many pages as each request needs, in a shuffled pool, and the number of pages."""
    rng = np.random.Generator(np.random.PCG64(case["lengths"] + 3))
    need = (ctx + new + PAGE - 1) // PAGE
    pool = rng.permutation(int(need.sum()))
    table = np.zeros((len(ctx), max(1, columns or int(need.max()))), np.int64)
    filled = np.arange(table.shape[1])[None] < need[:, None]
    table[filled] = pool
    return table, max(1, len(pool))


def _i32(a):
    return torch.from_numpy(np.ascontiguousarray(a, np.int32)).cuda()


def _normal(shape, dtype, gen, scale=1.0):
    return (torch.randn(shape, generator=gen, device="cuda") * scale).to(dtype)


def _tokens(shape, vocab, gen):
    """Token ids of which a few are much more frequent than the others."""
    return (torch.rand(shape, generator=gen, device="cuda").pow(3.0) * vocab).to(torch.int32).clamp_(max=vocab - 1)


def _inputs(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    s = SimpleNamespace(case=case)
    ctx, new = _lengths(case)
    kind = case["kind"]
    if kind == "pages":
        b, columns = case["batch"], case["columns"]
        held = (ctx + PAGE - 1) // PAGE
        grow = (ctx + new + PAGE - 1) // PAGE - held
        rng = np.random.Generator(np.random.PCG64(int(seed)))
        spare = int(grow.sum() * case["spare"]) + 1
        s.n_pages = int(held.sum()) + spare
        ids = rng.permutation(s.n_pages)
        table = np.zeros((b, columns), np.int64)
        table[np.arange(columns)[None] < held[:, None]] = ids[spare:]
        free = np.zeros(s.n_pages, np.int64)
        free[:spare] = ids[:spare]
        s.table, s.held, s.free, s.n_free = _i32(table), _i32(held), _i32(free), _i32(np.array([spare]))
        s.ctx, s.new, s.rows = _i32(ctx), _i32(new), int(new.sum())
        # what is kept of a step: a part of its tokens
        s.kept, s.none = _i32(ctx + rng.integers(0, new + 1)), torch.zeros(b, dtype=torch.int32, device="cuda")
        return s
    if kind == "logits" and case["new_hi"] == 0:
        new, parent = np.ones(len(ctx), np.int64), None
    else:
        parent = _parents(case, new)
    t = int(new.sum())
    s.n_ctx, s.n_new, s.parent_host = ctx, new, parent
    s.parent, s.ctx, s.new = None if parent is None else _i32(parent), _i32(ctx), _i32(new)
    s.cu = None if parent is None else _i32(np.concatenate([[0], np.cumsum(new)]))
    if kind == "logits":
        v, b = case["vocab"], len(ctx)
        s.logits = _normal((t, case["pitch"]), DTYPES[case["dtype"]], gen, 3.0)[:, :v]
        s.history = _tokens((b, max(1, int(ctx.max()))), v, gen)
        s.n_prompt = (torch.rand(b, generator=gen, device="cuda") * s.ctx).to(torch.int32)
        s.repetition = 1.0 + 0.5 * torch.rand(b, generator=gen, device="cuda")
        s.presence = 0.8 * torch.rand(b, generator=gen, device="cuda")
        s.frequency = 0.4 * torch.rand(b, generator=gen, device="cuda")
        s.bias_id = s.bias = s.mask = None
        if case["biases"]:
            # tokens of their own: neighbours of a request's first one, in steps that do not meet again
            first = torch.randint(0, v, (b, 1), generator=gen, device="cuda")
            step = max(1, v // case["biases"])
            s.bias_id = ((first + torch.arange(case["biases"], device="cuda") * step) % v).to(torch.int32)
            s.bias = _normal((b, case["biases"]), torch.float32, gen, 4.0)
        if case["allowed"] < 1.0:
            words = (v + 31) // 32
            keep = torch.zeros((t, words), dtype=torch.int32, device="cuda")
            for bit in range(32):
                keep |= (torch.rand((t, words), generator=gen, device="cuda") < case["allowed"]).to(torch.int32) << bit
            s.mask = keep
        s.tokens = None if parent is None else _tokens((t,), v, gen)
        return s
    s.table_host, s.n_pages = _table(case, ctx, new)
    s.table = _i32(s.table_host)
    if kind == "attention":
        dims = (s.n_pages, case["hkv"], PAGE, case["hd"])
        s.q = _normal((t, case["hq"], case["hd"]), torch.bfloat16, gen, 1.5)
    else:
        dims = (case["layers"], s.n_pages, case["hkv"], PAGE, case["hd"])
        rng = np.random.Generator(np.random.PCG64(int(seed)))
        tokens = rng.integers(0, 32000, size=t)
        target = rng.integers(0, 32000, size=t)
        begin = np.repeat(np.cumsum(new) - new, new)
        child = np.nonzero((parent >= 0) & (rng.random(t) < case["match"]))[0]
        child = rng.permutation(child)                        # of several children the one that is last here is the target
        target[begin[child] + parent[child]] = tokens[child]
        s.tokens, s.target = _i32(tokens), _i32(target)
        s.given = torch.minimum(s.new, torch.ones_like(s.new))
    s.k_pool = _normal(dims, torch.bfloat16, gen)
    s.v_pool = _normal((*dims[:-2], dims[-1], dims[-2]), torch.bfloat16, gen)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if case["kind"] not in ("attention", "commit") and not (case["kind"] == "logits" and s.parent is not None):
        return s
    # where each node stands and what lies on its path: for the plain form
    new = s.n_new
    t, b, widest = int(new.sum()), len(new), max(1, int(new.max(initial=0)))
    req = np.repeat(np.arange(b), new)
    at = np.arange(t) - np.repeat(np.cumsum(new) - new, new)
    s.on_path = torch.from_numpy(_ancestors(s.parent_host, new)).cuda()
    s.req, s.at = torch.from_numpy(req).cuda(), torch.from_numpy(at).cuda()
    cu = np.cumsum(new) - new
    rows = cu[:, None] + np.minimum(np.arange(widest)[None], np.maximum(new, 1)[:, None] - 1)
    s.rows = torch.from_numpy(np.clip(rows, 0, max(0, t - 1))).cuda()
    s.back = torch.from_numpy(req * widest + at).cuda()
    if case["kind"] != "logits":
        pos = s.n_ctx[req] + at
        s.page, s.slot = torch.from_numpy(s.table_host[req, pos // PAGE]).cuda(), torch.from_numpy(pos % PAGE).cuda()
        s.pages, s.last = torch.from_numpy(s.table_host).cuda(), torch.from_numpy(s.n_ctx).cuda()
        if own:
            import paper_2511_07423_amd as synera
            s.batch = synera.TreeBatch(case["hq"], case["hkv"], case["hd"], b, max(1, t), s.table.shape[1])
            s.batch.plan(s.ctx, s.new, s.parent, s.table, s.n_pages)
    return s


# ------------------------------------------------------------------------------------------------ one pass
def _plain_update(s, ctx, new, rows):
    """Pages taken from the stack or returned to it, in the order of requests and columns; then where each token goes."""
    b, columns = s.table.shape
    ctx, new, held, n = ctx.long(), new.long(), s.held.long(), s.n_free.long()
    need = (ctx + new + PAGE - 1) // PAGE
    sane = (ctx >= 0) & (new >= 0)
    fits = sane & (need <= columns)
    need = torch.where(fits, need, held)
    grow = (need - held).clamp_min(0)
    upto = grow.cumsum(0)
    served = fits & ((grow == 0) | (upto <= n))
    status = torch.where(sane, torch.where(served, 0, ENOSPC), ERANGE)
    back = (held - need).clamp_min(0) * served
    before = back.cumsum(0) - back
    col = torch.arange(columns, device=ctx.device)[None]
    take = (col >= held[:, None]) & (col < need[:, None]) & served[:, None]
    give = (col >= need[:, None]) & (col < held[:, None]) & served[:, None]
    at = (n - 1 - (upto - grow)[:, None] - (col - held[:, None])).clamp_(0, len(s.free) - 1)
    s.table.copy_(torch.where(take, s.free[at], s.table))
    left = n - (grow * served).sum()
    to = left + back.sum() - 1 - before[:, None] - (col - need[:, None])
    s.free[to[give]] = s.table[give]
    s.n_free.copy_(left + back.sum())
    s.held.copy_(torch.where(served, need, held))
    count = torch.where((new >= 0) & (new <= PAGE * columns), new, 0)
    cu = torch.cat([count.new_zeros(1), count.cumsum(0)])
    row = torch.arange(rows, device=ctx.device)
    req = torch.searchsorted(cu[1:], row, right=True)
    pos = ctx[req] + row - cu[req]
    slot = s.table[req, (pos // PAGE).clamp_(0, columns - 1)] * PAGE + pos % PAGE
    good = served[req]
    i32 = lambda x: x.to(torch.int32)  # noqa: E731
    return i32(cu), i32(torch.where(good, pos, -1)), i32(torch.where(good, slot, -1)), i32(status)


def _pages_pass(s, update):
    cu, pos, slot, status = update(s, s.ctx, s.new, s.rows)
    _, _, _, after = update(s, s.kept, s.none, 0)
    return {"cu": cu, "pos": pos, "slot": slot, "status": status, "after": after, "table": s.table, "held": s.held, "free": s.free,
            "n_free": s.n_free}


def _plain_attention(s):
    case = s.case
    b, c = s.rows.shape
    hkv, hd, g = case["hkv"], case["hd"], case["hq"] // case["hkv"]
    n = s.pages.shape[1] * PAGE
    k = s.k_pool[s.pages].permute(0, 2, 4, 1, 3).float().reshape(b, hkv, hd, n)
    v = s.v_pool[s.pages].permute(0, 2, 1, 4, 3).float().reshape(b, hkv, n, hd)
    q = s.q[s.rows].float().view(b, c, hkv, g, hd).permute(0, 2, 1, 3, 4).reshape(b, hkv, c * g, hd)
    x = torch.matmul(q, k) / math.sqrt(hd)
    node = torch.arange(n, device=q.device)[None] - s.last[:, None]
    seen = torch.gather(s.on_path[s.rows], 2, node.clamp(0, c - 1)[:, None].expand(b, c, n))
    hidden = ~((node < 0)[:, None] | (seen & (node < c)[:, None]))
    x = x.view(b, hkv, c, g, n).masked_fill_(hidden[:, None, :, None], -math.inf).view(b, hkv, c * g, n)
    m = x.amax(-1, keepdim=True)
    p = torch.exp(x.sub_(m))
    l = p.sum(-1, keepdim=True)
    o = torch.matmul(p, v) / l
    back = lambda y: y.view(b, hkv, c, g, -1).permute(0, 2, 1, 3, 4).reshape(b * c, hkv * g, -1)[s.back]  # noqa: E731
    out = {"o": back(o).to(torch.bfloat16)}
    if case["lse"]:
        out["lse"] = back(m + torch.log(l)).squeeze(-1)
    return out


def _plain_commit(s):
    """The path: nodes that are given or match their parent's target, first among their siblings, on a path of such nodes."""
    b, c = s.rows.shape
    new, given = s.new.long(), s.given.long()
    live = torch.arange(c, device=new.device)[None] < new[:, None]
    parent, tokens, target = s.parent[s.rows].long(), s.tokens[s.rows], s.target[s.rows]
    col = torch.arange(c, device=new.device)
    wanted = torch.gather(target, 1, parent.clamp_min(0))
    fits = live & (parent >= 0) & (tokens == wanted)
    earlier = (parent[:, :, None] == parent[:, None]) & fits[:, None] & (col[None, :, None] > col[None, None, :])
    good = torch.where(col[None] < given[:, None], live, fits & ~earlier.any(-1))
    up = torch.zeros((b, c, c), dtype=torch.bool, device=new.device)
    up.view(b * c, c)[s.back] = s.on_path
    on = live & (~up | good[:, None]).all(-1)
    n_path = on.sum(1)
    path = torch.where(on, col[None], c).sort(1).values
    last = torch.gather(path, 1, (n_path - 1).clamp_min(0)[:, None]).clamp_max(c - 1)
    token = torch.where(n_path > 0, torch.gather(target, 1, last)[:, 0], -1)
    path = torch.where(col[None] < n_path[:, None], path, -1).reshape(-1)[s.back]
    # every node of a path is read before any is written
    to = (s.at < n_path[s.req]).nonzero()[:, 0]
    src = to - s.at[to] + path[to]
    s.k_pool[:, s.page[to], :, s.slot[to]] = s.k_pool[:, s.page[src], :, s.slot[src]]
    s.v_pool[:, s.page[to], :, :, s.slot[to]] = s.v_pool[:, s.page[src], :, :, s.slot[src]]
    i32 = lambda x: x.to(torch.int32)  # noqa: E731
    return {"accept_len": i32(n_path - given), "token": i32(token), "path": i32(path), "n_path": i32(n_path), "k_pool": s.k_pool, "v_pool": s.v_pool}


def _plain_logits(s):
    v = s.case["vocab"]
    t, b = s.logits.shape[0], s.history.shape[0]
    at = torch.arange(s.history.shape[1], device=s.history.device)[None]
    ids = s.history.long()
    seen = torch.zeros((b, v), dtype=torch.float32, device=ids.device).scatter_add_(1, ids, (at < s.ctx[:, None]).float())
    made = torch.zeros_like(seen).scatter_add_(1, ids, ((at < s.ctx[:, None]) & (at >= s.n_prompt[:, None])).float())
    if s.parent is not None:
        seen, made = seen[s.req], made[s.req]
        path = s.tokens[s.rows].long()[s.req]
        seen.scatter_add_(1, path, s.on_path.float())
        made.scatter_add_(1, path, s.on_path.float())
    of = (lambda x: x[s.req][:, None]) if s.parent is not None else (lambda x: x[:, None])
    x = s.logits.float()
    x = torch.where(seen > 0, torch.where(x > 0, x / of(s.repetition), x * of(s.repetition)), x)
    x = x - (of(s.frequency) * made + of(s.presence) * (made > 0))
    if s.bias is not None:
        add = torch.zeros((b, v), dtype=torch.float32, device=ids.device).scatter_(1, s.bias_id.long(), s.bias)
        x = x + (add[s.req] if s.parent is not None else add)
    if s.mask is not None:
        token = torch.arange(v, device=ids.device)
        x = torch.where((s.mask[:, token // 32] >> (token % 32)) & 1 == 1, x, -math.inf)
    return x.to(s.logits.dtype)


def _own_logits(s):
    import paper_2511_07423_amd as synera
    return synera.adjust_logits(s.logits, cu=s.cu, history=s.history, history_len=s.ctx, n_prompt=s.n_prompt, repetition=s.repetition,
                                presence=s.presence, frequency=s.frequency, bias_id=s.bias_id, bias=s.bias, mask=s.mask, tokens=s.tokens,
                                parent=s.parent)


def _own_update(s, ctx, new, rows):
    import paper_2511_07423_amd as synera
    return synera.update_pages(s.table, s.held, s.free, s.n_free, ctx, new, rows)


def run(s):
    kind = s.case["kind"]
    if kind == "pages":
        return _pages_pass(s, _own_update if own else _plain_update)
    if kind == "logits":
        return {"logits": _own_logits(s) if own else _plain_logits(s)}
    if kind == "attention":
        if not own:
            return _plain_attention(s)
        if s.case["lse"]:
            o, lse = s.batch.attention(s.q, s.k_pool, s.v_pool, want_lse=True)
            return {"o": o, "lse": lse}
        return {"o": s.batch.attention(s.q, s.k_pool, s.v_pool)}
    if not own:
        return _plain_commit(s)
    out = s.batch.accept(s.tokens, s.target, n_given=s.given)
    s.batch.commit(out["path"], out["n_path"], s.k_pool, s.v_pool)
    return {**out, "k_pool": s.k_pool, "v_pool": s.v_pool}


# ------------------------------------------------------------------------------------------------ work
def work(case):
    """Every input once, every output once; the products of attention, or the few operations of an element."""
    ctx, new = _lengths(case)
    t, b = float(new.sum()), case["batch"]
    if case["kind"] == "pages":
        grow = float(((ctx + new + PAGE - 1) // PAGE - (ctx + PAGE - 1) // PAGE).sum())
        return {"bytes": 8.0 * t + 40.0 * b + 16.0 * grow, "flops": 4.0 * t}
    if case["kind"] == "logits":
        if case["new_hi"] == 0:
            t = float(b)
        size, v = BYTES[case["dtype"]], case["vocab"]
        masks = 4.0 * t * ((v + 31) // 32) if case["allowed"] < 1.0 else 0.0
        return {"bytes": t * v * size * (1.0 + case["allowed"]) + masks + 4.0 * float(ctx.sum()) + 8.0 * b * (case["biases"] + 2) + 8.0 * t,
                "flops": 4.0 * t * v}
    hq, hkv, hd = case["hq"], case["hkv"], case["hd"]
    if case["kind"] == "commit":
        # what the path moves goes by the targets: a node for each third level of a tree of as many nodes, as drawn
        moved = t / 4.0 * case["match"]
        return {"bytes": moved * case["layers"] * 8.0 * hkv * hd + 16.0 * t, "flops": 4.0 * t}
    depth = float(_ancestors(_parents(case, new), new).sum())
    pairs = float((ctx * new).sum()) + depth
    return {"bytes": float((ctx + new).sum()) * 4.0 * hkv * hd + 4.0 * t * hq * hd + (4.0 * t * hq if case["lse"] else 0.0),
            "flops": 4.0 * pairs * hq * hd}


# ------------------------------------------------------------------------------------------------ from the definition, in 64 bits
def _exact_attention(s):
    case = s.case
    hq, hkv, hd = case["hq"], case["hkv"], case["hd"]
    g = hq // hkv
    t = int(s.n_new.sum())
    o = torch.empty((t, hq, hd), dtype=torch.float64, device="cuda")
    lse = torch.empty((t, hq), dtype=torch.float64, device="cuda")
    first = 0
    for i, (l, n) in enumerate(zip(s.n_ctx.tolist(), s.n_new.tolist())):
        if n == 0:
            continue
        see = torch.ones((n, l + n), dtype=torch.bool)
        see[:, l:] = False
        for j in range(n):                                    # a node sees what its parent sees, and itself
            up = int(s.parent_host[first + j])
            if up >= 0:
                see[j, l:] = see[up, l:]
            see[j, l + j] = True
        see = see.cuda()
        ids = torch.from_numpy(s.table_host[i, : (l + n + PAGE - 1) // PAGE]).cuda()
        for h in range(hkv):
            keys = s.k_pool[ids, h].reshape(-1, hd)[: l + n].double()
            vals = s.v_pool[ids, h].transpose(1, 2).reshape(-1, hd)[: l + n].double()
            q = s.q[first: first + n, h * g: (h + 1) * g].double().reshape(n * g, hd)
            x = (q @ keys.T.contiguous()).view(n, g, l + n) / math.sqrt(hd)
            x = torch.where(see[:, None], x, torch.full_like(x, -math.inf))
            z = torch.logsumexp(x, -1)
            lse[first: first + n, h * g: (h + 1) * g] = z
            o[first: first + n, h * g: (h + 1) * g] = (torch.exp(x - z[..., None]).view(n * g, -1) @ vals).view(n, g, hd)
        first += n
    return {"o": o, "lse": lse} if case["lse"] else {"o": o}


def _exact_logits(s):
    """Request by request: how often each token was seen, by sorting what was."""
    if s.logits.numel() > 1 << 27 or s.logits.shape[0] > 3000:
        return None                                           # (row by row, that takes minutes)
    x = s.logits.double()
    first = 0
    for i, n in enumerate(s.n_new.tolist()):
        past = s.history[i, : int(s.n_ctx[i])].cpu().numpy()
        prompt = int(s.n_prompt[i])
        rho, pres, freq = (float(p[i]) for p in (s.repetition, s.presence, s.frequency))
        tokens = None if s.parent is None else s.tokens[first: first + n].cpu().numpy()
        for j in range(n):
            more = []
            while tokens is not None and (j if not more else up) >= 0:
                at = j if not more else up
                more.append(tokens[at])
                up = int(s.parent_host[first + at])
            made = np.concatenate([past[prompt:], np.array(more, past.dtype)])
            every = np.unique(np.concatenate([past[:prompt], made]))
            ids, times = np.unique(made, return_counts=True)
            row = x[first + j]
            e = torch.from_numpy(every.astype(np.int64)).cuda()
            row[e] = torch.where(row[e] > 0, row[e] / rho, row[e] * rho)
            e = torch.from_numpy(ids.astype(np.int64)).cuda()
            row[e] -= freq * torch.from_numpy(times.astype(np.float64)).cuda() + pres
            if s.bias is not None:
                row[s.bias_id[i].long()] += s.bias[i].double()
        first += n
    if s.mask is not None:
        bits = torch.arange(32, device="cuda", dtype=torch.int32)
        allowed = ((s.mask[:, :, None] >> bits) & 1).flatten(1)[:, : x.shape[1]]
        x[allowed == 0] = -math.inf
    return {"logits": x}


def _exact_commit(s):
    """Request by request: the children of the node at hand in order, until none has the token that follows it."""
    tokens, target = s.tokens.cpu().numpy(), s.target.cpu().numpy()
    k_pool, v_pool = s.k_pool.double(), s.v_pool.double()
    place = lambda i, p: (int(s.table_host[i, p // PAGE]), p % PAGE)  # noqa: E731
    first = 0
    for i, (l, n) in enumerate(zip(s.n_ctx.tolist(), s.n_new.tolist())):
        path = [0] if n else []
        while path:
            at = path[-1]
            next_ = [j for j in range(at + 1, n) if s.parent_host[first + j] == at and tokens[first + j] == target[first + at]]
            if not next_:
                break
            path.append(next_[0])
        for k, j in enumerate(path):
            (to, a), (page, b) = place(i, l + k), place(i, l + j)
            k_pool[:, to, :, a], v_pool[:, to, :, :, a] = k_pool[:, page, :, b].clone(), v_pool[:, page, :, :, b].clone()
        first += n
    return {"accept_len": None, "token": None, "path": None, "n_path": None, "k_pool": k_pool, "v_pool": v_pool}


def exact(case, seed):
    if case["kind"] == "pages":
        return None                                           # whole numbers
    s = _inputs(case, seed)
    return {"attention": _exact_attention, "commit": _exact_commit, "logits": _exact_logits}[case["kind"]](s)


if __name__ == "__main__":
    for case in listed() + [draw(random.Random(i)) for i in range(6)]:
        print(case, work(case))
