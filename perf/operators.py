"""What is timed of the operators around a paged cache that requests share: rotary positions, norms of queries and keys with
the rotation, appends with the rotation on the way, and attention whose shared prefixes are read once for all.

Kinds of case
  rope       Rope.apply: queries and keys turned by their positions
  norm_rope  Rope.norm_apply: each head normed, then turned
  append     SharedBatch.append_rope: queries turned, keys turned into their pages, values into theirs
  attention  SharedBatch.attention: a ragged batch over the paged cache, some of its pages shared
Head counts and widths are those of the shapes in workloads/shapes.py (4/4 x 64, 32/8 x 128, 64/8 x 128) or generic.
Everything else follows from the case and the seed.  `run` computes a case in plain torch operations, or, where `own` is
set, by the package's calls."""
import math
import random
from types import SimpleNamespace

import numpy as np
import torch

own = False

PAGE = 16
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}
EPS = 1e-5
FACTOR, LOW, HIGH, ORIGINAL = 8.0, 1.0, 4.0, 8192      # how positions are scaled, where they are


# ------------------------------------------------------------------------------------------------ the cases
def _rope(kind, tokens, heads, dtype, layout, rot=0, scaling="none", far=4096, base=10000.0, fused=True):
    """far: positions up to here; rot: rotated values of a head (0: all); fused: heads are slices of one QKV array."""
    hq, hkv, hd = heads
    return {"kind": kind, "tokens": tokens, "hq": hq, "hkv": hkv, "hd": hd, "dtype": dtype, "layout": layout, "rot": rot or hd,
            "scaling": scaling, "far": far, "base": base, "fused": fused}


def _append(batch, heads, ctx, new, dtype, layout, rot=0, norm=False, scaling="none", lengths=1):
    """ctx, new = (low, high) of the cached lengths and of the rows each request appends."""
    hq, hkv, hd = heads
    return {"kind": "append", "batch": batch, "hq": hq, "hkv": hkv, "hd": hd, "ctx_lo": ctx[0], "ctx_hi": ctx[1], "new_lo": new[0],
            "new_hi": new[1], "dtype": dtype, "layout": layout, "rot": rot or hd, "norm": norm, "scaling": scaling,
            "base": 10000.0, "lengths": lengths}


def _attention(batch, heads, groups, prefix, own_len, new, lse=False, lengths=1):
    """`groups` groups of requests, each behind a prefix of its own of up to `prefix` tokens; then own_len = (low, high) cached
    tokens and new = (low, high) new ones of each request."""
    hq, hkv, hd = heads
    return {"kind": "attention", "batch": batch, "hq": hq, "hkv": hkv, "hd": hd, "groups": groups, "prefix": prefix,
            "own_lo": own_len[0], "own_hi": own_len[1], "new_lo": new[0], "new_hi": new[1], "lse": lse, "lengths": lengths}


TINY, WIDE8, WIDE64 = (4, 4, 64), (32, 8, 128), (64, 8, 128)


def listed():
    return [
        # one token of one request, far out in a long context: all latency
        {"name": "rope_1_far", **_rope("rope", 1, WIDE8, "bf16", "interleaved", scaling="bands", far=120000, base=500000.0)},
        # a prompt's queries and keys, half of each head turned
        {"name": "rope_8192_half_part", **_rope("rope", 8192, WIDE8, "bf16", "half", rot=64, scaling="linear", far=32768)},
        # one decoding step of 64 requests
        {"name": "norm_rope_64", **_rope("norm_rope", 64, WIDE64, "bf16", "half", far=8192)},
        # heads of 80 of which 20 values turn, fp16, an odd number of tokens
        {"name": "norm_rope_777_odd", **_rope("norm_rope", 777, (20, 20, 80), "f16", "half", rot=20)},
        # prompts' rows in 32 bits, as the projections of this library leave them
        {"name": "norm_rope_6000_f32", **_rope("norm_rope", 6000, WIDE8, "f32", "interleaved", far=16384)},
        # one decoding step of 64 requests into their pages
        {"name": "append_64x1", **_append(64, WIDE8, (0, 512), (1, 1), "bf16", "half")},
        # ragged draft chunks in 32 bits, heads normed on the way
        {"name": "append_64_chunks", **_append(64, WIDE8, (0, 512), (1, 16), "f32", "interleaved", norm=True)},
        # a prefill engine's rows of one layer
        {"name": "append_24_prompts", **_append(24, WIDE8, (0, 40), (512, 2048), "bf16", "half", scaling="bands")},
        # the small decoder: four chunks behind 64 shared tokens
        {"name": "attention_tiny_4", **_attention(4, TINY, 1, 64, (0, 40), (4, 4), lse=True)},
        # parallel samples of one long prompt, one token each
        {"name": "attention_256x1", **_attention(256, WIDE8, 1, 8192, (64, 1024), (1, 1))},
        # ragged draft chunks of four applications' requests, each behind its application's prompt
        {"name": "attention_64_chunks", **_attention(64, WIDE8, 4, 2048, (128, 2048), (1, 16), lse=True)},
        # questions about one long document, prefilled behind it
        {"name": "attention_8_prompts", **_attention(8, WIDE64, 1, 16384, (0, 0), (128, 256))},
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
    if what < 0.4:
        hq, hkv, hd = _heads(rng)
        if rng.random() < 0.35:
            hd = rng.choice((48, 72, 80, 96, 112, 160, 256))
        rot = rng.choice((hd, hd, hd // 2, hd // 4))
        dtype = rng.choice(("bf16", "bf16", "f16", "f32"))
        most = max(1, (96 << 20) // ((hq + hkv) * hd * BYTES[dtype]))
        return _rope(rng.choice(("rope", "norm_rope")), _log(rng, 1, most), (hq, hkv, hd), dtype,
                     rng.choice(("interleaved", "half")), rot - rot % 2, rng.choice(("none", "linear", "bands")), _log(rng, 512, 200000),
                     rng.choice((10000.0, 500000.0)), rng.random() < 0.5)
    if what < 0.65:
        heads = _heads(rng)
        b = _log(rng, 1, 128)
        most = max(1, (64 << 20) // ((heads[0] + 2 * heads[1]) * heads[2] * 4 * b))
        n = _log(rng, 1, min(4096, most))
        lo = _log(rng, 1, 400)
        return _append(b, heads, (rng.choice((0, lo)), lo), (rng.choice((1, max(1, n // 2))), n), rng.choice(("bf16", "f16", "f32")),
                       rng.choice(("interleaved", "half")), rng.choice((heads[2], heads[2] // 2)), rng.random() < 0.4,
                       rng.choice(("none", "linear", "bands")), lengths)
    heads = _heads(rng)
    b = _log(rng, 1, 256)
    groups = min(b, rng.choice((1, 1, 2, 4, 16)))
    # keys and scores that the plain form lays out for the whole batch stay below those of the largest listed case
    ctx = _log(rng, 64, max(65, min(16384, (1 << 31) // (b * heads[1] * heads[2]))))
    part = rng.choice((0.0, 0.5, 0.9, 0.98))
    prefix = int(ctx * part) // PAGE * PAGE
    rest = max(1, ctx - prefix)
    most = max(1, (1 << 31) // (b * heads[0] * (ctx + 64)))
    new = _log(rng, 1, min(most, 512)) if rng.random() < 0.5 else 1
    new = min(new, max(1, int(1.0e12 / (4.0 * b * heads[0] * heads[2] * (ctx + new)))))
    return _attention(b, heads, groups, prefix, (rng.choice((0, rest // 4)), rest), (rng.choice((1, new)), new), rng.random() < 0.5, lengths)


# ------------------------------------------------------------------------------------------------ inputs
def _frequencies(case):
    """What each pair turns by from one position to the next, in 64 bits."""
    half = case["rot"] // 2
    f = case["base"] ** (-np.arange(half, dtype=np.float64) / half)
    if case["scaling"] == "linear":
        f = f / FACTOR
    elif case["scaling"] == "bands":
        t = np.clip((ORIGINAL * f / (2 * math.pi) - LOW) / (HIGH - LOW), 0.0, 1.0)
        f = (1 - t) * f / FACTOR + t * f
    return f


def _handle(case):
    import paper_2511_07423_amd as synera
    scaling = {"none": None, "linear": ("linear", FACTOR), "bands": ("bands", FACTOR, LOW, HIGH, ORIGINAL)}[case["scaling"]]
    return synera.Rope(case["hd"], case["rot"], layout=case["layout"], base=case["base"], scaling=scaling)


def _plan(case, ctx, new, table, n_pages):
    import paper_2511_07423_amd as synera
    batch = synera.SharedBatch(case["hq"], case["hkv"], case["hd"], len(ctx), int(new.sum()), table.shape[1])
    batch.plan(ctx, new, table, n_pages)
    return batch


def _lengths(case):
    """(shared pages, cached tokens, new tokens) of each request, their page table and the number of pages: shared pages
    first in every row, pages in a shuffled pool."""
    rng = np.random.Generator(np.random.PCG64(case["lengths"]))
    b = case["batch"]
    new = rng.integers(case["new_lo"], case["new_hi"] + 1, size=b)
    if case["kind"] == "append":
        group, shared = np.arange(b), np.zeros(b, np.int64)
        ctx = rng.integers(case["ctx_lo"], case["ctx_hi"] + 1, size=b)
    else:
        groups = case["groups"]
        group = np.concatenate([np.arange(groups), rng.integers(0, groups, size=b - groups)])
        most = case["prefix"] // PAGE
        shared = np.rint(most * (rng.uniform(0.5, 1.0, size=groups) if groups > 1 else np.ones(1))).astype(np.int64)[group]
        lo, hi = case["own_lo"], case["own_hi"]
        rest = np.rint(np.exp(rng.uniform(math.log(max(lo, 1)), math.log(max(hi, 1)), size=b))).astype(np.int64) if hi > 0 else np.zeros(b, np.int64)
        ctx = shared * PAGE + np.clip(rest, lo, hi)
    pages = (ctx + new + PAGE - 1) // PAGE
    first = {}
    at, rows = 0, []
    for i in range(b):
        if group[i] not in first:
            first[group[i]] = at
            at += int(shared[i])
        rows.append(np.concatenate([first[group[i]] + np.arange(shared[i]), at + np.arange(pages[i] - shared[i])]))
        at += int(pages[i] - shared[i])
    pool = rng.permutation(at)
    table = np.zeros((b, int(pages.max())), np.int32)
    for i in range(b):
        table[i, : pages[i]] = pool[rows[i]]
    return ctx.astype(np.int32), new.astype(np.int32), table, at


def _normal(shape, dtype, gen, scale=1.0):
    return (torch.randn(shape, generator=gen, device="cuda") * scale).to(dtype)


def _qkv(case, tokens, gen, with_v):
    """Query, key and value heads [tokens][heads][width], as slices of one array or on their own."""
    counts = [case["hq"], case["hkv"]] + ([case["hkv"]] if with_v else [])
    if case.get("fused", True):
        x = _normal((tokens, sum(counts) if with_v else sum(counts) + case["hkv"], case["hd"]), DTYPES[case["dtype"]], gen, 1.5)
        cuts = np.cumsum([0] + counts)
        return [x[:, cuts[i]: cuts[i + 1]] for i in range(len(counts))]
    return [_normal((tokens, n, case["hd"]), DTYPES[case["dtype"]], gen, 1.5) for n in counts]


def _gains(case, gen):
    return [(1 + 0.1 * torch.randn(case["hd"], generator=gen, device="cuda")).to(torch.bfloat16) for _ in range(2)]


def _inputs(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    s = SimpleNamespace(case=case)
    if case["kind"] in ("rope", "norm_rope"):
        t = case["tokens"]
        s.q, s.k = _qkv(case, t, gen, False)
        s.gains = _gains(case, gen) if case["kind"] == "norm_rope" else None
        # runs of neighbouring positions, as a batch of prompts or chunks has them
        start = torch.randint(0, max(1, case["far"] - 256), (t // 256 + 1,), generator=gen, device="cuda")
        s.pos = (start.repeat_interleave(256)[:t] + torch.arange(t, device="cuda") % 256).to(torch.int32)
        return s
    s.ctx, s.new, s.table, s.n_pages = _lengths(case)
    t = int(s.new.sum())
    dims = (s.n_pages, case["hkv"], PAGE, case["hd"])
    s.k_pool = _normal(dims, torch.bfloat16, gen)
    s.v_pool = _normal((dims[0], dims[1], dims[3], dims[2]), torch.bfloat16, gen)
    if case["kind"] == "append":
        s.q, s.k, s.v = _qkv(case, t, gen, True)
        s.gains = _gains(case, gen) if case["norm"] else None
    else:
        s.q = _normal((t, case["hq"], case["hd"]), torch.bfloat16, gen, 1.5)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if case["kind"] != "attention":
        s.freq = torch.from_numpy(_frequencies(case)).cuda()
    if case["kind"] in ("append", "attention"):
        # where each new token stands: its request, its position, its page and slot; for the plain form
        req = np.repeat(np.arange(len(s.new)), s.new)
        at = np.arange(len(req)) - np.repeat(np.cumsum(s.new) - s.new, s.new)
        pos = s.ctx[req] + at
        s.pos = torch.from_numpy(pos.astype(np.int32)).cuda()
        s.page = torch.from_numpy(s.table[req, pos // PAGE].astype(np.int64)).cuda()
        s.slot = torch.from_numpy((pos % PAGE).astype(np.int64)).cuda()
    if case["kind"] == "attention":
        widest = int(s.new.max())
        cu = np.cumsum(s.new) - s.new
        rows = cu[:, None] + np.minimum(np.arange(widest)[None], s.new[:, None] - 1)
        s.rows = torch.from_numpy(rows.astype(np.int64)).cuda()
        s.back = torch.from_numpy((req * widest + at).astype(np.int64)).cuda()
        s.last = torch.from_numpy((s.ctx[:, None] + np.arange(widest)[None]).astype(np.int64)).cuda()
        s.pages = torch.from_numpy(s.table.astype(np.int64)).cuda()
    if own:
        if case["kind"] != "attention":
            s.rope = _handle(case)
        if case["kind"] in ("append", "attention"):
            s.batch = _plan(case, s.ctx, s.new, s.table, s.n_pages)
    return s


# ------------------------------------------------------------------------------------------------ one pass
def _normed(x, gain):
    x = x.float()
    if gain is None:
        return x
    return x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * gain.float()


def _turned(x, pos, freq, layout):
    """x f32 [tokens][heads][width]"""
    ang = pos.double()[:, None] * freq
    c, s = torch.cos(ang).float()[:, None], torch.sin(ang).float()[:, None]
    rot = 2 * freq.numel()
    out = x.clone()
    if layout == "interleaved":
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        out[..., 0:rot:2], out[..., 1:rot:2] = a * c - b * s, b * c + a * s
    else:
        a, b = x[..., : rot // 2], x[..., rot // 2: rot]
        out[..., : rot // 2], out[..., rot // 2: rot] = a * c - b * s, b * c + a * s
    return out


def _plain_attention(s):
    case = s.case
    b, c = s.rows.shape
    hkv, hd, g = case["hkv"], case["hd"], case["hq"] // case["hkv"]
    n = s.pages.shape[1] * PAGE
    k = s.k_pool[s.pages].permute(0, 2, 4, 1, 3).float().reshape(b, hkv, hd, n)
    v = s.v_pool[s.pages].permute(0, 2, 1, 4, 3).float().reshape(b, hkv, n, hd)
    q = s.q[s.rows].float().view(b, c, hkv, g, hd).permute(0, 2, 1, 3, 4).reshape(b, hkv, c * g, hd)
    x = torch.matmul(q, k) / math.sqrt(hd)
    hidden = torch.arange(n, device=q.device) > s.last[:, None, :, None, None]
    x = x.view(b, hkv, c, g, n).masked_fill_(hidden, -math.inf).view(b, hkv, c * g, n)
    m = x.amax(-1, keepdim=True)
    p = torch.exp(x.sub_(m))
    l = p.sum(-1, keepdim=True)
    o = torch.matmul(p, v) / l
    back = lambda y: y.view(b, hkv, c, g, -1).permute(0, 2, 1, 3, 4).reshape(b * c, hkv * g, -1)[s.back]  # noqa: E731
    out = {"o": back(o).to(torch.bfloat16)}
    if case["lse"]:
        out["lse"] = back(m + torch.log(l)).squeeze(-1)
    return out


def run(s):
    case = s.case
    kind = case["kind"]
    if own:
        if kind == "rope":
            q, k = s.rope.apply(s.pos, s.q, s.k)
            return {"q": q, "k": k}
        if kind == "norm_rope":
            q, k = s.rope.norm_apply(s.pos, s.q, s.k, s.gains[0], s.gains[1], EPS)
            return {"q": q, "k": k}
        if kind == "append":
            gains = s.gains or (None, None)
            q = s.batch.append_rope(s.rope, s.q, s.k, s.v, s.k_pool, s.v_pool, q_gain=gains[0], k_gain=gains[1], eps=EPS)
            return {"q": q, "k_pool": s.k_pool, "v_pool": s.v_pool}
        if case["lse"]:
            o, lse = s.batch.attention(s.q, s.k_pool, s.v_pool, want_lse=True)
            return {"o": o, "lse": lse}
        return {"o": s.batch.attention(s.q, s.k_pool, s.v_pool)}
    if kind == "attention":
        return _plain_attention(s)
    gains = s.gains or (None, None)
    q = _turned(_normed(s.q, gains[0]), s.pos, s.freq, case["layout"])
    k = _turned(_normed(s.k, gains[1]), s.pos, s.freq, case["layout"])
    if kind != "append":
        return {"q": q.to(s.q.dtype), "k": k.to(s.k.dtype)}
    s.k_pool[s.page, :, s.slot] = k.to(torch.bfloat16)
    s.v_pool[s.page, :, :, s.slot] = s.v.to(torch.bfloat16)
    return {"q": q.to(torch.bfloat16), "k_pool": s.k_pool, "v_pool": s.v_pool}


# ------------------------------------------------------------------------------------------------ work
def work(case):
    """Every input once, every output once; the products of attention, or the few operations of an element."""
    hq, hkv, hd = case["hq"], case["hkv"], case["hd"]
    if case["kind"] in ("rope", "norm_rope"):
        n = case["tokens"] * (hq + hkv) * hd
        ops = 3.0 * n * case["rot"] / hd + (4.0 * n if case["kind"] == "norm_rope" else 0.0)
        return {"bytes": 2.0 * n * BYTES[case["dtype"]] + 4.0 * case["tokens"], "flops": ops}
    ctx, new, table, _ = _lengths(case)
    t = float(new.sum())
    if case["kind"] == "append":
        n = t * (hq + 2 * hkv) * hd
        turned = t * (hq + hkv) * hd
        return {"bytes": n * (BYTES[case["dtype"]] + 2), "flops": 3.0 * turned * case["rot"] / hd + (4.0 * turned if case["norm"] else 0.0)}
    pages = (ctx.astype(np.int64) + new + PAGE - 1) // PAGE
    seen = np.unique(np.concatenate([table[i, : pages[i]] for i in range(len(ctx))]))
    pairs = float((new.astype(np.float64) * ctx + new * (new + 1.0) / 2).sum())
    return {"bytes": len(seen) * 4.0 * PAGE * hkv * hd + 4.0 * t * hq * hd + (4.0 * t * hq if case["lse"] else 0.0),
            "flops": 4.0 * pairs * hq * hd}


# ------------------------------------------------------------------------------------------------ from the definition, in 64 bits
def _spun(case, x, gain, pos):
    """A head's pairs as complex numbers times e^(i angle)."""
    x = x.double()
    if gain is not None:
        x = gain.double() * x / torch.sqrt(x.square().sum(-1, keepdim=True) / x.shape[-1] + EPS)
    half = case["rot"] // 2
    f = [case["base"] ** (-2.0 * i / case["rot"]) for i in range(half)]
    if case["scaling"] == "linear":
        f = [v / FACTOR for v in f]
    if case["scaling"] == "bands":
        turns = [ORIGINAL * v / (2 * math.pi) for v in f]
        mix = [0.0 if r <= LOW else 1.0 if r >= HIGH else (r - LOW) / (HIGH - LOW) for r in turns]
        f = [w * v + (1 - w) * v / FACTOR for v, w in zip(f, mix)]
    ang = torch.outer(pos.double(), torch.tensor(f, dtype=torch.float64, device=x.device))
    turn = torch.polar(torch.ones_like(ang), ang)[:, None]
    head, tail = x[..., : case["rot"]], x[..., case["rot"]:]
    if case["layout"] == "interleaved":
        z = torch.view_as_complex(head.reshape(*head.shape[:-1], half, 2).contiguous()) * turn
        head = torch.view_as_real(z).flatten(-2)
    else:
        z = torch.complex(head[..., :half].contiguous(), head[..., half:].contiguous()) * turn
        head = torch.cat([z.real, z.imag], -1)
    return torch.cat([head, tail], -1)


def exact(case, seed):
    s = _inputs(case, seed)
    if case["kind"] in ("rope", "norm_rope"):
        gains = s.gains or (None, None)
        return {"q": _spun(case, s.q, gains[0], s.pos), "k": _spun(case, s.k, gains[1], s.pos)}
    k_pool, v_pool = s.k_pool.double(), s.v_pool.double()
    begins = np.concatenate([[0], np.cumsum(s.new)])
    if case["kind"] == "append":
        pos = torch.cat([torch.arange(int(l), int(l) + int(n), device="cuda") for l, n in zip(s.ctx, s.new)])
        gains = s.gains or (None, None)
        q, k = _spun(case, s.q, gains[0], pos), _spun(case, s.k, gains[1], pos)
        for i, (l, n) in enumerate(zip(s.ctx, s.new)):
            at = np.arange(l, l + n)
            page = torch.from_numpy(s.table[i, at // PAGE].astype(np.int64)).cuda()
            slot = torch.from_numpy((at % PAGE).astype(np.int64)).cuda()
            k_pool[page, :, slot] = k[begins[i]: begins[i + 1]]
            v_pool[page, :, :, slot] = s.v[begins[i]: begins[i + 1]].double()
        return {"q": q, "k_pool": k_pool, "v_pool": v_pool}
    hq, hkv, hd = case["hq"], case["hkv"], case["hd"]
    g = hq // hkv
    o = torch.empty((int(begins[-1]), hq, hd), dtype=torch.float64, device="cuda")
    lse = torch.empty((int(begins[-1]), hq), dtype=torch.float64, device="cuda")
    for i, (l, n) in enumerate(zip(s.ctx.tolist(), s.new.tolist())):
        ids = torch.from_numpy(s.table[i, : (l + n + PAGE - 1) // PAGE].astype(np.int64)).cuda()
        see = torch.arange(l + n, device="cuda")[None] <= (l + torch.arange(n, device="cuda"))[:, None]
        for h in range(hkv):
            keys = k_pool[ids, h].reshape(-1, hd)[: l + n]
            vals = v_pool[ids, h].transpose(1, 2).reshape(-1, hd)[: l + n]
            q = s.q[begins[i]: begins[i + 1], h * g: (h + 1) * g].double().reshape(n * g, hd)
            x = (q @ keys.T.contiguous()).view(n, g, l + n) / math.sqrt(hd)
            x = torch.where(see[:, None], x, torch.full_like(x, -math.inf))
            z = torch.logsumexp(x, -1)
            lse[begins[i]: begins[i + 1], h * g: (h + 1) * g] = z
            o[begins[i]: begins[i + 1], h * g: (h + 1) * g] = (torch.exp(x - z[..., None]).view(n * g, -1) @ vals).view(n, g, hd)
    return {"o": o, "lse": lse} if case["lse"] else {"o": o}


if __name__ == "__main__":
    for case in listed() + [draw(random.Random(i)) for i in range(6)]:
        print(case, work(case))
