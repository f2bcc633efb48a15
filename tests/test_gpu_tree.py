"""GPU parity of the operators that verify trees of drafted tokens with plain Python and float64: page tables, attention, accepted paths and
their move, adjusted logits; at the sizes, masks and lengths where they can go wrong."""
import gc
import random

import numpy as np
import pytest
import torch

import shared_reference as ref
import tree_reference as tree

pytestmark = pytest.mark.gpu
DEV, P = "cuda:0", 16
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


@pytest.fixture(autouse=True)
def nothing_left_behind():
    """What a test's refusals leave in cycles (graphs among it) goes with the test, not inside a later test's capture."""
    yield
    gc.collect()


def synera():
    import paper_2511_07423_amd as s
    return s


def i32(a):
    return torch.from_numpy(np.ascontiguousarray(a, np.int32)).to(DEV)


def draw(shape, seed, dtype=torch.bfloat16, scale=1.0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return (torch.randn(shape, generator=g, device=DEV) * scale).to(dtype)


def bits(shape, value):
    return torch.full(shape, value, dtype=torch.int16, device=DEV).view(torch.bfloat16)


# ------------------------------------------------------------------------------------------------ pages
def pages_state(rng, B, columns, spare):
    held = np.array([rng.randrange(0, columns + 1) for _ in range(B)], np.int32)
    n_pages = int(held.sum()) + spare
    ids = np.array(rng.sample(range(n_pages), n_pages), np.int32)
    table = np.full((B, columns), -5, np.int32)
    at = 0
    for i in range(B):
        table[i, : held[i]] = ids[at: at + held[i]]
        at += held[i]
    free = np.concatenate([ids[at:], np.full(n_pages - spare, -9, np.int32)]).astype(np.int32)
    return table, held, free, spare


def check_pages(table, held, free, n_free, ctx, new, n_rows, shared=None):
    dev = [i32(x) for x in (table, held, free, [n_free])]
    got = synera().update_pages(*dev, i32(ctx), i32(new), n_rows, None if shared is None else i32(shared))
    cu, pos, slot, status, left = tree.update_pages(table, held, free, n_free, ctx, new, n_rows, shared)
    named = zip(("cu", "status"), (got[0], got[3]), (cu, status))
    for name, g, w in [*named, ("table", dev[0], table), ("held", dev[1], held), ("free", dev[2], free), ("n_free", dev[3], [left])]:
        assert np.array_equal(g.cpu().numpy(), w), name
    t = min(int(cu[-1]), n_rows)
    assert np.array_equal(got[1].cpu().numpy()[:t], pos[:t]) and np.array_equal(got[2].cpu().numpy()[:t], slot[:t])
    return left


@pytest.mark.parametrize("seed", range(24))
def test_pages(seed):
    rng = random.Random(seed)
    B = rng.choice((1, 2, 7, 64, 300, 1024, 1025, 2500))
    columns = rng.choice((1, 3, 40))
    state = list(pages_state(rng, B, columns, rng.choice((1, B, 10 * B))))
    for step in range(3):
        ctx = np.array([rng.choice((0, 1, 15, 16, 17, rng.randrange(columns * P + 1))) for _ in range(B)])
        new = np.array([rng.choice((0, 0, 1, 2, 16, rng.randrange(max(1, columns * P // 4)))) for _ in range(B)])
        if step == 1 and B > 2:                                # what only the device sees
            ctx[rng.randrange(B)], new[rng.randrange(B)], ctx[rng.randrange(B)] = -3, -1, 2 ** 31 - 1
            new[rng.randrange(B)] = P * columns + 1
        shared = None if step == 0 else np.array([rng.choice((0, 0, 1, 2, columns, -4)) for _ in range(B)])
        rows = int(np.clip(new, 0, P * columns).sum()) + rng.choice((-3, 0, 5))
        state[3] = check_pages(*state, ctx, new, max(0, rows), shared)


@pytest.mark.parametrize("rows", [0, 1, 100000])
def test_pages_of_long_rows(rows):
    """A prompt of many pages, and rows given back whole."""
    rng = random.Random(rows)
    state = list(pages_state(rng, 5, 9000, 20000))
    ctx, new = np.array([0, 5, 140000, 16 * 9000, 70]), np.array([rows // 5, rows // 5, 1, 0, rows // 5])
    state[3] = check_pages(*state, ctx, new, rows)
    check_pages(*state, np.zeros(5, np.int64), np.zeros(5, np.int64), 0)


def test_pages_taken_back():
    """A step that is taken back leaves the stack as it was, and every page is held once or free once."""
    rng = random.Random(5)
    table, held, free, n = pages_state(rng, 50, 30, 900)
    need = np.maximum(held, 1)
    ctx = need * P - 3
    state = [i32(x) for x in (table, held, free, [n])]
    s = synera()
    s.update_pages(*state, i32(ctx), i32(np.zeros(50)), 0)
    before = [x.clone() for x in state]
    new = np.array([rng.randrange(0, min(90, 30 * P - int(c) + 1)) for c in ctx])
    _, _, slot, status = s.update_pages(*state, i32(ctx), i32(new), int(new.sum()))
    assert (status == 0).all() and (slot >= 0).all() and slot.unique().numel() == int(new.sum())
    h, t, f = state[1].cpu().numpy(), state[0].cpu().numpy(), state[2].cpu().numpy()[: state[3].item()]
    every = np.concatenate([t[i, : h[i]] for i in range(50)] + [f])
    assert np.array_equal(np.sort(every), np.arange(len(free)))
    s.update_pages(*state, i32(ctx), i32(np.zeros(50)), 0)
    n = before[3].item()
    assert torch.equal(state[1], before[1]) and state[3].item() == n and torch.equal(state[2][:n], before[2][:n])


def test_pages_of_states_that_cannot_be():
    """Counts outside their ranges are read as the nearest that can be, rows that hold what they cannot are refused."""
    s = synera()
    table, held = i32(np.arange(12).reshape(3, 4)), i32([4, 5, -1])
    free, n_free = i32(np.arange(20)), i32([99])
    cu, pos, slot, status = s.update_pages(table, held, free, n_free, i32([64, 1, 1]), i32([0, 3, 4]), 7)
    assert status.tolist() == [0, s.EINVAL, s.EINVAL] and held.tolist() == [4, 5, -1] and n_free.item() == 20
    assert cu.tolist() == [0, 0, 3, 7] and (pos == -1).all() and (slot == -1).all()
    n_free.fill_(-5)
    _, _, _, status = s.update_pages(table, i32([0, 4, 0]), free, n_free, i32([1, 2, 0]), i32([0, 0, 0]), 0)
    assert status.tolist() == [s.ENOSPC, 0, 0] and n_free.item() == 3


# ------------------------------------------------------------------------------------------------ trees
def grow(rng, n, shape):
    if shape == "chain":
        return list(range(-1, n - 1))
    if shape == "roots":
        return [-1] * n
    if shape == "forest":
        return [rng.randrange(-1, j) if j else -1 for j in range(n)]
    return [-1 if j == 0 else max(0, j - rng.randrange(1, 6)) for j in range(n)]


def make(rng, B, ctx_hi, n_hi, shapes=("chain", "roots", "forest", "tree"), zero=0.2):
    trees = [grow(rng, 0 if rng.random() < zero and B > 1 else rng.randrange(1, n_hi + 1), rng.choice(shapes)) for _ in range(B)]
    if not any(trees):
        trees[0] = [-1]
    ctx = np.array([rng.choice((0, rng.randrange(ctx_hi + 1), ctx_hi)) for _ in range(B)])
    need = [-(-(int(c) + len(t)) // P) for c, t in zip(ctx, trees)]
    columns, n_pages = max(1, max(need)) + rng.randrange(3), sum(need) + 2
    ids = rng.sample(range(n_pages), n_pages)
    table = np.full((B, columns), -1, np.int32)
    for i, k in enumerate(need):
        table[i, :k] = [ids.pop() for _ in range(k)]
    return ctx, trees, table, n_pages


def filled(ctx, trees, table, n_pages, hkv, hd, seed, junk=0x7FC0):
    """Pools in which every position that a request holds has values and everything else is junk (NaN)."""
    k, v = bits((n_pages, hkv, P, hd), junk), bits((n_pages, hkv, hd, P), junk)
    live = torch.zeros((n_pages, P), dtype=torch.bool)
    for c, t, row in zip(ctx, trees, table):
        at = np.arange(int(c) + len(t))
        live[row[at // P], at % P] = True
    live = live.to(DEV)
    return (torch.where(live[:, None, :, None], draw(k.shape, seed), k).contiguous(),
            torch.where(live[:, None, None, :], draw(v.shape, seed + 1), v).contiguous())


def planned(hq, hkv, hd, ctx, trees, table, n_pages, more=0):
    T = sum(map(len, trees))
    b = synera().TreeBatch(hq, hkv, hd, len(trees) + more, T + more, table.shape[1] + more)
    status = b.plan(i32(ctx), i32([len(t) for t in trees]), i32(sum(trees, [])), i32(table), n_pages)
    assert (status == 0).all()
    return b


def check_attention(hq, hkv, hd, ctx, trees, table, n_pages, seed, scale=None, std=1.5):
    b = planned(hq, hkv, hd, ctx, trees, table, n_pages, more=seed % 3)
    k, v = filled(ctx, trees, table, n_pages, hkv, hd, seed)
    T = sum(map(len, trees))
    q = draw((T + 3, hq, hd), seed + 2, scale=std)
    out = bits((T + 3, hq, hd), 0x1234)
    got, lse = b.attention(q, k, v, scale=scale, out=out, want_lse=True)
    want, want_lse, eo, el = tree.attention(ref.to64(q)[:T], ref.to64(k), ref.to64(v), ctx, trees, table, hd ** -0.5 if scale is None else scale)
    ref.close(ref.to64(got)[:T], want, eo, "o")
    ref.close(ref.to64(lse)[:T], want_lse, el, "lse")
    assert torch.equal(got[T:].view(torch.int16), bits((3, hq, hd), 0x1234).view(torch.int16))     # rows behind the batch stay
    return b, q, k, v


@pytest.mark.parametrize("seed", range(20))
def test_attention(seed):
    rng = random.Random(seed)
    hkv = rng.choice((1, 2, 3))
    hq, hd = hkv * rng.choice((1, 3, 4, 7, 16)), rng.choice((64, 128))
    args = make(rng, rng.choice((1, 2, 5, 20)), rng.choice((0, 40, 700)), rng.choice((1, 5, 33)))
    check_attention(hq, hkv, hd, *args, seed * 10)


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("ctx,n", [(0, 1), (0, 2), (15, 1), (16, 1), (31, 1), (31, 2), (32, 1), (100, 60), (127, 1), (128, 128), (255, 3), (0, 256), (77, 256),
                                   (1000, 40), (5000, 1), (5003, 33)])
def test_attention_one_request(ctx, n, hd):
    """Lengths around pages, tiles and cuts, the fewest and the most nodes; every class of rows."""
    rng = random.Random(ctx + n)
    need = -(-(ctx + n) // P)
    table = np.array([rng.sample(range(need), need)], np.int32)
    for hq, hkv, shape in ((1, 1, "forest"), (8, 2, "tree"), (16, 1, "roots")):
        check_attention(hq, hkv, hd, np.array([ctx]), [grow(rng, n, shape)], table, need, ctx + n)


@pytest.mark.parametrize("hq,hkv", [(128, 8), (80, 5), (33, 11), (10, 10), (48, 3)])
def test_attention_of_many_rows(hq, hkv):
    """Requests of many tiles and of one, whose units begin in different lists, some of no nodes in between, keys cut and whole."""
    rng = random.Random(hq)
    trees = [grow(rng, n, rng.choice(("tree", "wide", "chain"))) for n in (200, 3, 0, 77, 256, 1, 130)]
    for ctx in ((0, 700, 5, 90, 31, 1500, 128), (20, 0, 0, 3, 0, 17, 0)):
        need = [-(-(c + len(t)) // P) for c, t in zip(ctx, trees)]
        ids, table, at = rng.sample(range(sum(need)), sum(need)), np.full((len(need), max(need)), -1, np.int32), 0
        for i, k in enumerate(need):
            table[i, :k] = ids[at:at + k]
            at += k
        check_attention(hq, hkv, 64, np.array(ctx), trees, table, sum(need), 4)


def test_attention_of_a_long_context():
    """More steps than any length of ranges but the last few covers with what room there is for partial results."""
    rng, need = random.Random(12), -(-(150000 + 21) // P)
    table = np.array([rng.sample(range(need), need)], np.int32)
    check_attention(3, 1, 64, np.array([150000]), [grow(rng, 21, "tree")], table, need, 5)


def outputs_of(b, T, q, k, v, rope, B):
    """All calls behind a plan, on T rows, with what they leave."""
    out = bits((T, b.n_q_heads, b.head_dim), 0x1234)
    if T:
        b.append_rope(rope, None, q[:T, :b.n_kv_heads], q[:T, :b.n_kv_heads], k, v)
    else:
        b.append_rope(rope, q[:0], q[:0, :b.n_kv_heads], q[:0, :b.n_kv_heads], k, v)
    _, lse = b.attention(q[:T], k, v, out=out, want_lse=True)
    tokens = i32(np.zeros(T))
    got = b.accept(tokens, tokens, anchor=i32(np.zeros(B)))
    b.commit(got["path"], got["n_path"], k, v)
    return out, lse, got


def test_steps_without_nodes_and_plans_that_have_not_run():
    """No request has a node; and calls behind a plan that is captured and not replayed, eager ones and captured ones on no rows: nothing is written."""
    s, (hq, hkv, hd), B, n_pages = synera(), (4, 2, 64), 3, 8
    q = draw((10, hq, hd), 1)
    k, v = draw((n_pages, hkv, P, hd), 2), draw((n_pages, hkv, hd, P), 3)
    before = k.clone(), v.clone()
    rope = s.Rope(hd, layout="half")
    b = s.TreeBatch(hq, hkv, hd, B, 10, 2)
    table = i32(np.arange(6).reshape(3, 2))
    status = b.plan(i32([5, 0, 20]), i32([0, 0, 0]), i32([]), table, n_pages)
    out, lse, got = outputs_of(b, 0, q, k, v, rope, B)
    assert status.tolist() == [0, 0, 0] and lse.shape == (0, hq)
    assert got["accept_len"].tolist() == got["n_path"].tolist() == [0, 0, 0] and got["token"].tolist() == [-1] * 3 and got["path"].numel() == 0

    b = s.TreeBatch(hq, hkv, hd, B, 10, 2)
    ctx, new, parent = i32([5, 0, 20]), i32([2, 1, 3]), i32([-1, 0, -1, -1, 0, 0])
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        status = b.plan(ctx, new, parent, table, n_pages)
    out, _, _ = outputs_of(b, 6, q, k, v, rope, B)
    assert torch.equal(out.view(torch.int16), bits(out.shape, 0x1234).view(torch.int16))
    assert torch.equal(k.view(torch.int16), before[0].view(torch.int16)) and torch.equal(v.view(torch.int16), before[1].view(torch.int16))
    graph.replay()
    out, _, got = outputs_of(b, 6, q, k, v, rope, B)
    assert status.tolist() == [0, 0, 0] and not torch.equal(k.view(torch.int16), before[0].view(torch.int16))
    assert torch.isfinite(out).all()

    b.plan(i32([5, 0, 20]), i32([0, 0, 0]), i32([]), table, n_pages)
    none, at = torch.cuda.CUDAGraph(), (k.clone(), v.clone(), q.clone())
    torch.cuda.synchronize()
    with torch.cuda.graph(none):
        b.append_rope(rope, q[:0], q[:0, :hkv], q[:0, :hkv], k, v)
        b.attention(q[:0], k, v, out=q[:0])
    b.plan(ctx, new, parent, table, n_pages)
    none.replay()
    torch.cuda.synchronize()
    for x, y in zip((k, v, q), at):
        assert torch.equal(x.view(torch.int16), y.view(torch.int16))


def test_attention_many_requests():
    """More requests than a block has threads; most of them short, one long, some without nodes."""
    args = make(random.Random(9), 700, 40, 3)
    check_attention(2, 1, 64, *args, 3)
    rng = random.Random(10)
    trees = [grow(rng, rng.randrange(0, 3), "forest") for _ in range(300)] + [grow(rng, 200, "tree")]
    ctx = np.array([rng.randrange(30) for _ in range(300)] + [9000])
    need = [-(-(int(c) + len(t)) // P) for c, t in zip(ctx, trees)]
    table = np.zeros((301, max(need)), np.int32)
    at = 0
    for i, k in enumerate(need):
        table[i, :k] = at + np.arange(k)
        at += k
    check_attention(4, 2, 64, ctx, trees, table, at, 4)


def test_pages_beyond_two_to_the_32_bytes():
    """The last pages of pools of over 2^32 bytes, and layers that far apart: appends, attention and moves are what they are in a small pool, bit for bit."""
    hq, hkv, hd, page = 8, 8, 128, 8 * P * 128
    n_pages = (1 << 32) // (2 * page) + 40
    ctx, trees, table, n = make(random.Random(11), 4, 120, 20, zero=0.0)
    s, T = synera(), sum(map(len, trees))
    far = table.copy()
    far[table >= 0] = n_pages - 1 - table[table >= 0]
    x = draw((T, hq + 2 * hkv, hd), 1)
    rope = s.Rope(hd)
    outs = []
    for t, pages in ((table, n), (far, n_pages)):
        k, v = (torch.zeros((2, pages, hkv, P, hd), dtype=torch.bfloat16, device=DEV), torch.zeros((2, pages, hkv, hd, P), dtype=torch.bfloat16, device=DEV))
        ids = torch.from_numpy(t[t >= 0].astype(np.int64)).to(DEV)
        k[:, ids], v[:, ids] = draw((2, len(ids), hkv, P, hd), 2), draw((2, len(ids), hkv, hd, P), 3)
        b = s.TreeBatch(hq, hkv, hd, 4, T, t.shape[1])
        assert (b.plan(i32(ctx), i32([len(c) for c in trees]), i32(sum(trees, [])), i32(t), pages) == 0).all()
        q = b.append_rope(rope, x[:, :hq], x[:, hq: hq + hkv], x[:, hq + hkv:], k[1], v[1])
        o = b.attention(q, k[1], v[1])
        acc = b.accept(i32(np.zeros(T)), i32(np.zeros(T)), n_given=i32(np.ones(4)))        # first children all the way down
        b.commit(acc["path"], acc["n_path"], k, v)
        outs.append((q, o, acc["path"], k[:, ids].clone(), v[:, ids].clone()))
        del k, v
        torch.cuda.empty_cache()
    assert all(torch.equal(p, q) for p, q in zip(*outs))


def test_replayed_plans_of_other_sizes():
    """Behind a replayed plan that has more rows than a call's tensors, what lies in them is worked on and nothing behind them is touched; one that has
    more requests than the last plan that was called is served whole."""
    s, hq, hkv, hd = synera(), 4, 2, 64
    ctx, trees, table, n = make(random.Random(12), 6, 700, 9, shapes=("tree",), zero=0.0)
    new, T = [len(t) for t in trees], sum(map(len, trees))
    k, v = filled(ctx, trees, table, n, hkv, hd, 5)
    q = draw((T, hq, hd), 6)
    b = planned(hq, hkv, hd, ctx, trees, table, n)
    want = b.attention(q, k, v)
    args = i32(ctx), i32(new), i32(sum(trees, [])), i32(table), n
    first = [x[:2].contiguous() for x in args[:2]]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            b.plan(*args)
        few = new[0] + new[1]
        for _ in range(3):
            b.plan(*first, args[2][:few].contiguous(), args[3][:2].contiguous(), n)
            assert torch.equal(b.attention(q[:few], k, v)[:few], want[:few])
            graph.replay()
            out = bits((T, hq, hd), 0x1234)
            b.attention(q, k, v, out=out)                      # (the last plan that was called has two requests)
            assert torch.equal(out, want)
            cut = new[0] + new[1] + 1
            out = bits((T, hq, hd), 0x1234)
            b.attention(q[:cut], k, v, out=out[:cut])
            rope, x = s.Rope(hd), draw((cut, hq + 2 * hkv, hd), 8)
            out_q = bits((T, hq, hd), 0x1234)
            kp, vp = k.clone(), v.clone()
            b.append_rope(rope, x[:, :hq], x[:, hq: hq + hkv], x[:, hq + hkv:], kp, vp, out_q=out_q[:cut])
            acc = b.accept(i32(np.zeros(cut)), i32(np.zeros(cut)), n_given=i32(np.ones(2)))
            side.synchronize()
            assert torch.equal(out[:few], want[:few]) and (out[few:].view(torch.int16) == 0x1234).all()
            assert (out_q[cut:].view(torch.int16) == 0x1234).all() and (out_q[:cut].view(torch.int16) != 0x1234).any()
            assert (acc["n_path"] >= 1).all()


def test_attention_of_chains_is_that_of_chunks():
    """Trees whose parents are the nodes before them against the attention over chunks: both within their error of float64."""
    rng = random.Random(3)
    ctx, trees, table, n = make(rng, 9, 600, 30, shapes=("chain",), zero=0.0)
    b, q, k, v = check_attention(8, 2, 128, ctx, trees, table, n, 0)
    new = np.array([len(t) for t in trees], np.int32)
    s = synera().SharedBatch(8, 2, 128, 9, int(new.sum()), table.shape[1])
    s.plan(ctx, new, table, n)
    T = int(new.sum())
    _, _, eo, _ = tree.attention(ref.to64(q)[:T], ref.to64(k), ref.to64(v), ctx, trees, table, 128 ** -0.5)
    ref.close(ref.to64(b.attention(q, k, v))[:T], ref.to64(s.attention(q, k, v))[:T], 2 * eo, "chunks")


def test_attention_repeats_bit_for_bit_and_shares_pages():
    rng = random.Random(4)
    ctx, trees, table, n = make(rng, 12, 900, 20, zero=0.0)
    ctx[:] = np.maximum(ctx, 200)
    shared = rng.sample(range(n, n + 12), 12)                  # twelve pages that all requests begin with
    need = [-(-(int(c) + len(t)) // P) for c, t in zip(ctx, trees)]
    at = n + 12
    table = np.full((12, max(need)), -1, np.int32)
    for i, k in enumerate(need):
        table[i, :12], table[i, 12:k] = shared, np.arange(at, at + k - 12)
        at += k - 12
    b, q, k, v = check_attention(8, 2, 128, ctx, trees, table, at, 1)
    T = sum(map(len, trees))
    first = b.attention(q, k, v)[:T]
    for _ in range(3):
        assert torch.equal(b.attention(q, k, v)[:T], first)


def test_attention_scales_and_large_scores():
    args = make(random.Random(6), 5, 300, 12)
    for scale, std in ((1e-4, 1.0), (1.0, 1.5), (7.0, 3.0)):
        check_attention(4, 2, 64, *args, 3, scale=scale, std=std)


def test_attention_strides():
    hq, hkv, hd = 6, 2, 64
    ctx, trees, table, n = make(random.Random(7), 6, 100, 9)
    b = planned(hq, hkv, hd, ctx, trees, table, n)
    k, v = filled(ctx, trees, table, n, hkv, hd, 5)
    T = sum(map(len, trees))
    q = draw((T, hq + 2 * hkv, hd), 6)[:, :hq]
    plain = b.attention(q.contiguous(), k, v)
    assert torch.equal(b.attention(q, k, v), plain)
    out = torch.zeros((hq, T, hd), dtype=torch.bfloat16, device=DEV).transpose(0, 1)
    assert b.attention(q, k, v, out=out) is out and torch.equal(out, plain)


def test_attention_hidden_values():
    """Infinities and NaN: of a key or value, they reach the nodes that see it and no other; of a query, its own row."""
    hq, hkv, hd = 4, 2, 128
    trees = [[-1], [-1, 0, 0, 1, 1, 2, 2, 5], [-1] * 5 + [0, 1, 2, 3, 4] * 6]
    ctx = np.array([40, 21, 133])
    need = [-(-(int(c) + len(t)) // P) for c, t in zip(ctx, trees)]
    table = np.full((3, max(need)), -1, np.int32)
    for i, k in enumerate(need):
        table[i, :k] = sum(need[:i]) + np.arange(k)
    for bad in (float("inf"), float("-inf"), float("nan")):
        k, v = filled(ctx, trees, table, sum(need), hkv, hd, 5)
        at = 21 + 2                                            # seen by nodes 2, 5, 6, 7 of request 1 alone
        v[table[1, at // P], 1, 5, at % P] = bad
        at = 133 + 3                                           # by node 3 of request 2 and its children
        k[table[2, at // P], 0, at % P, 9] = float("nan")
        b = planned(hq, hkv, hd, ctx, trees, table, sum(need))
        q = draw((sum(map(len, trees)), hq, hd), 6)
        q[0, 3, 0] = float("nan")
        got, lse = b.attention(q, k, v, want_lse=True)
        want, wl, eo, el = tree.attention(ref.to64(q), ref.to64(k), ref.to64(v), ctx, trees, table, hd ** -0.5)
        ref.close(ref.to64(got), want, eo, f"o with {bad}")
        ref.close(ref.to64(lse), wl, el, f"lse with {bad}")


def test_plan_refuses_single_requests():
    """What only the device sees refuses its request: it has a status, no outputs and appends nothing; the others are as they would be without it."""
    s, hq, hkv, hd = synera(), 4, 2, 64
    trees = [[-1, 0, 0], [-1, 1], [-1, 0], [-1, -2], [-1, 0, 1], [-1], [-1, 0], [], [-1, 0, 1, 1]]
    ctx = np.array([20, 5, -1, 9, 30, 3 * P, 40, 7, 12])
    table = np.arange(9 * 3, dtype=np.int32).reshape(9, 3)
    table[4, 1] = 27                                           # outside the pool
    table[6, 0] = -1
    want_status = [0, s.EINVAL, s.ERANGE, s.EINVAL, s.ERANGE, s.ENOSPC, s.ERANGE, 0, 0]
    T = sum(map(len, trees))
    b = s.TreeBatch(hq, hkv, hd, 9, T, 3)
    status = b.plan(i32(ctx), i32([len(t) for t in trees]), i32(sum(trees, [])), i32(table), 27)
    assert status.tolist() == want_status
    k, v = draw((27, hkv, P, hd), 1), draw((27, hkv, hd, P), 2)
    x = draw((T, hq + 2 * hkv, hd), 3)
    out_q, out = bits((T, hq, hd), 0x1234), bits((T, hq, hd), 0x1234)
    k0, v0 = k.clone(), v.clone()
    rope = s.Rope(hd)
    b.append_rope(rope, x[:, :hq], x[:, hq: hq + hkv], x[:, hq + hkv:], k, v, out_q=out_q)
    b.attention(out_q, k, v, out=out)
    tokens, target = i32(np.arange(T)), i32(np.arange(T) + 1)
    acc = b.accept(tokens, target, n_given=i32(np.ones(9)))
    cu = np.concatenate([[0], np.cumsum([len(t) for t in trees])])
    for i, st in enumerate(want_status):
        rows = slice(cu[i], cu[i + 1])
        if st:
            assert (out[rows].view(torch.int16) == 0x1234).all() and (out_q[rows].view(torch.int16) == 0x1234).all()
            assert acc["n_path"][i] == 0 and acc["token"][i] == -1 and acc["accept_len"][i] == 0 and (acc["path"][rows] == -1).all()
    live = [i for i, st in enumerate(want_status) if st == 0]
    b2 = s.TreeBatch(hq, hkv, hd, 9, T, 3)
    sub = [trees[i] for i in live]
    b2.plan(i32(ctx[live]), i32([len(t) for t in sub]), i32(sum(sub, [])), i32(table[live]), 27)
    rows = torch.cat([torch.arange(cu[i], cu[i + 1]) for i in live]).to(DEV)
    y = x[rows]
    q2 = b2.append_rope(rope, y[:, :hq], y[:, hq: hq + hkv], y[:, hq + hkv:], k0, v0)
    assert torch.equal(k, k0) and torch.equal(v, v0) and torch.equal(out_q[rows], q2)
    assert torch.equal(out[rows], b2.attention(q2, k0, v0))
    # sizes: nodes beyond the most, and rows beyond those there are
    n = i32([2, 257, -1, 3, 2])
    b = s.TreeBatch(hq, hkv, hd, 5, 8, 3)
    status = b.plan(i32([0] * 5), n, i32([-1, 0, -1, 0, 1, -1]), i32(table[[0, 1, 2, 3, 5]]), 27)
    assert status.tolist() == [0, s.EINVAL, s.EINVAL, 0, s.ENOSPC]
    acc = b.accept(i32(np.zeros(6)), i32(np.zeros(6)), anchor=i32([0] * 5))
    assert acc["n_path"].tolist() == [2, 0, 0, 3, 0] and acc["path"].tolist() == [0, 1, 0, 1, 2, -1]


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("hd,rot,hq,hkv,layout", [(128, 128, 8, 2, "half"), (64, 20, 3, 3, "interleaved"), (128, 64, 2, 1, "half")])
def test_append(hd, rot, hq, hkv, layout, dtype):
    """Each node is turned by its place in the text and lies at its place in the cache; nothing else is written."""
    s = synera()
    for seed, (B, ctx_hi, n_hi) in enumerate(((1, 0, 1), (7, 40, 3), (6, 20, 40), (2, 90, 200))):
        ctx, trees, table, n = make(random.Random(seed + hd), B, ctx_hi, n_hi)
        b = planned(hq, hkv, hd, ctx, trees, table, n)
        rope = s.Rope(hd, rot, layout=layout)
        T = sum(map(len, trees))
        x = draw((T + 2, hq + 2 * hkv, hd), seed, TYPES[dtype], 2.0)
        q, k, v = x[:, :hq], x[:, hq: hq + hkv], x[:, hq + hkv:]
        norm = seed % 2 == 0
        gq, gk = (draw((hd,), 5) + 1, draw((hd,), 6) + 1) if norm else (None, None)
        kp, vp = bits((n + 1, hkv, P, hd), 0x1234), bits((n + 1, hkv, hd, P), 0x4321)
        out_q = bits((T + 2, hq, hd), 0x2345)
        b.append_rope(rope, q, k, v, kp, vp, q_gain=gq, k_gain=gk, out_q=out_q)
        depth = np.concatenate([[len(p) - 1 for p in tree.paths(t)] for t in trees]).astype(np.int64)
        req = np.repeat(np.arange(B), [len(t) for t in trees])
        at = np.concatenate([np.arange(len(t)) for t in trees]) + ctx[req]
        freq = ref.frequencies(rot)
        for got, x_, gain, name in ((out_q[:T], q, gq, "q"), (None, k, gk, "k")):
            want, err = ref.turn(ref.to64(x_)[:T], ctx[req] + depth, freq, layout, 1.0, None if gain is None else ref.to64(gain), 1e-5)
            if got is None:
                page, slot = torch.from_numpy(table[req, at // P].astype(np.int64)).to(DEV), torch.from_numpy(at % P).to(DEV)
                got = kp[page, :, slot]
            ref.close(ref.to64(got), want, np.abs(want) * 2.0 ** -8 + err * (1 + 2.0 ** -8) + 1e-38, name)
        assert torch.equal(vp[page, :, :, slot], v[:T].to(torch.bfloat16)) and (out_q[T:].view(torch.int16) == 0x2345).all()
        kp[page, :, slot], vp[page, :, :, slot] = bits((), 0x1234), bits((), 0x4321)
        assert (kp.view(torch.int16) == 0x1234).all() and (vp.view(torch.int16) == 0x4321).all()


# ------------------------------------------------------------------------------------------------ accepted paths
def targets(rng, trees, match, vocab=50):
    """Tokens (few, so that siblings share some) and targets that follow some child with probability `match`."""
    tokens, target = [], []
    for t in trees:
        tok = [rng.randrange(vocab) for _ in t]
        tgt = [rng.randrange(vocab) for _ in t]
        for j in rng.sample(range(len(t)), len(t)):
            if t[j] >= 0 and rng.random() < match:
                tgt[t[j]] = tok[j]
        tokens += tok
        target += tgt
    return np.array(tokens), np.array(target)


def commit_by_hand(k, v, ctx, trees, table, path, n_path):
    t = 0
    for i, tr in enumerate(trees):
        for j in range(int(n_path[i])):
            a, b = int(ctx[i]) + j, int(ctx[i]) + int(path[t + j])
            k[:, table[i, a // P], :, a % P] = k[:, table[i, b // P], :, b % P].clone()
            v[:, table[i, a // P], :, :, a % P] = v[:, table[i, b // P], :, :, b % P].clone()
        t += len(tr)


@pytest.mark.parametrize("seed", range(12))
def test_accept_and_commit(seed):
    rng = random.Random(seed)
    B, layers, hkv, hd = rng.choice((1, 3, 40)), rng.choice((1, 2, 5)), rng.choice((1, 3, 8)), rng.choice((64, 128))
    ctx, trees, table, n = make(rng, B, rng.choice((0, 30)), rng.choice((1, 12, 64, 256)))
    b = planned(hkv, hkv, hd, ctx, trees, table, n)
    tokens, target = targets(rng, trees, rng.choice((0.0, 0.7, 1.0)), rng.choice((3, 1000)))
    anchor = np.array([tokens[c] if len(t) and rng.random() < 0.7 else -2 for c, t in zip(np.cumsum([0] + [len(t) for t in trees]), trees)])
    given = None if seed % 3 == 0 else np.array([rng.choice((0, 0, 1, 1, -2, 300)) for _ in range(B)])
    use_anchor = given is None or seed % 3 == 1
    got = b.accept(i32(tokens), i32(target), i32(anchor) if use_anchor else None, None if given is None else i32(given))
    want = tree.accept(trees, tokens, target, anchor if use_anchor else None, given)
    for name, w in zip(("accept_len", "token", "path", "n_path"), want):
        assert np.array_equal(got[name].cpu().numpy(), w), name
    pools = draw((layers, n, hkv, P, hd), 1), draw((layers, n, hkv, hd, P), 2)
    by_hand = [x.clone() for x in pools]
    commit_by_hand(*by_hand, ctx, trees, table, want[2], want[3])
    b.commit(got["path"], got["n_path"], *pools)
    assert torch.equal(pools[0], by_hand[0]) and torch.equal(pools[1], by_hand[1])
    # one layer, as pools of four dimensions; and layers of a larger array
    wide = [torch.cat([x, x], 1)[:, :n] for x in (draw((layers, n, hkv, P, hd), 1), draw((layers, n, hkv, hd, P), 2))]
    b.commit(got["path"], got["n_path"], *wide)
    assert torch.equal(wide[0], by_hand[0]) and torch.equal(wide[1], by_hand[1])
    one = draw((layers, n, hkv, P, hd), 1)[0].clone(), draw((layers, n, hkv, hd, P), 2)[0].clone()
    b.commit(got["path"], got["n_path"], *one)
    assert torch.equal(one[0], by_hand[0][0]) and torch.equal(one[1], by_hand[1][0])


def test_commit_of_paths_that_cannot_be():
    """Nodes outside k .. n - 1 stay where they are."""
    trees, ctx, table = [[-1, 0, 1, 2, 3, 4]], np.array([30]), np.arange(3, dtype=np.int32)[None]
    b = planned(2, 2, 64, ctx, trees, table, 3)
    pools = draw((1, 3, 2, P, 64), 1), draw((1, 3, 2, 64, P), 2)
    by_hand = [x.clone() for x in pools]
    b.commit(i32([2, 0, 6, -7, 5, 2 ** 31 - 1]), i32([9]), *pools)
    commit_by_hand(*by_hand, ctx, trees, table, np.array([2, 1, 2, 3, 5, 5]), [6])
    assert torch.equal(pools[0], by_hand[0]) and torch.equal(pools[1], by_hand[1])
    b.commit(i32([5] * 6), i32([-3]), *pools)
    assert torch.equal(pools[0], by_hand[0])


# ------------------------------------------------------------------------------------------------ logits
def check_logits(rng, trees, B, vocab, dtype, seed, parts, pitch=0, in_place=False):
    """parts: the names of what is given."""
    T = B if trees is None else sum(map(len, trees))
    pitch = pitch or vocab
    wide = draw((T, pitch), seed, TYPES[dtype], 3.0)
    logits = wide[:, :vocab]
    req = np.arange(B) if trees is None else np.repeat(np.arange(B), [len(t) for t in trees])
    rs = np.random.RandomState(seed)
    if T and vocab > 3:
        logits[0, 1], logits[0, 2], logits[T - 1, 3] = float("nan"), float("-inf"), float("inf")
    a = dict.fromkeys(("history", "history_len", "n_prompt", "repetition", "presence", "frequency", "bias_id", "bias", "mask", "tokens", "parent"))
    if "history" in parts:
        columns = rs.randint(0, 300)
        a["history"] = rs.randint(-2, min(vocab, 40) + 2, size=(B, columns))
        a["history_len"] = rs.randint(-1, columns + 3, size=B)
        if "n_prompt" in parts:
            a["n_prompt"] = rs.randint(-1, columns + 2, size=B)
    for name in ("repetition", "presence", "frequency"):
        if name in parts:
            a[name] = (rs.rand(B) * (1.5 if name == "repetition" else 1.0) + (0.4 if name == "repetition" else -0.3)).astype(np.float32)
    if "bias" in parts:
        n = rs.randint(0, 40)
        a["bias_id"] = rs.randint(-1, vocab + 1, size=(B, n))
        a["bias"] = (rs.randn(B, n) * 5).astype(np.float32)
        a["bias"][rs.rand(B, n) < 0.1] = -np.inf
    allowed = None
    if "mask" in parts:
        words = rs.randint(-2 ** 31, 2 ** 31, size=(T, (vocab + 31) // 32), dtype=np.int64).astype(np.int32)
        if T > 1:
            words[1] = 0                                       # a row that its mask leaves empty
        a["mask"] = words
        allowed = np.unpackbits(words.view(np.uint8), axis=1, bitorder="little")[:, :vocab].astype(bool)
    path = [[] for _ in range(T)]
    if "tree" in parts and trees is not None:
        a["tokens"], a["parent"] = rs.randint(-1, min(vocab, 30) + 1, size=T), np.array(sum(trees, []))
        path, t = [], 0
        for tr in trees:
            path += [[a["tokens"][t + j] for j in p] for p in tree.paths(tr)]
            t += len(tr)
    x = ref.to64(logits)
    want, err = tree.adjust(x, req, a["history"], a["history_len"], a["n_prompt"], a["repetition"], a["presence"], a["frequency"], a["bias_id"],
                            a["bias"], allowed, path)
    f32 = ("repetition", "presence", "frequency", "bias")
    dev = {n: None if w is None else torch.from_numpy(np.ascontiguousarray(w)).to(DEV) if n in f32 else i32(w) for n, w in a.items()}
    cu = None if trees is None else i32(np.concatenate([[0], np.cumsum([len(t) for t in trees])]))
    before = wide.clone()
    got = synera().adjust_logits(logits, cu=cu, out=logits if in_place else None, **dev)
    tiny = {"f32": 2.0 ** -149, "bf16": 2.0 ** -133, "f16": 2.0 ** -24}[dtype]               # a step of the smallest values
    with np.errstate(all="ignore"):
        allow = ref.half_step(TYPES[dtype]) * (np.abs(want) + err) + err + tiny
    if dtype == "f16":                                         # beyond the type's range: infinity
        want = np.where(np.abs(want) >= 65520, np.sign(want) * np.inf, want)
    ref.close(ref.to64(got), want, np.where(np.isfinite(allow), allow, 0), "logits")
    if in_place:
        assert got is logits
        assert torch.equal(wide[:, vocab:].view(torch.uint8), before[:, vocab:].view(torch.uint8))
    else:
        assert torch.equal(wide.view(torch.uint8), before.view(torch.uint8))


EVERY = ("history", "n_prompt", "repetition", "presence", "frequency", "bias", "mask", "tree")


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("vocab", [1, 7, 31, 33, 1000, 8192, 8193, 20011, 32000])
def test_logits(vocab, dtype):
    rng = random.Random(vocab)
    for seed, (B, n_hi, parts, pitch) in enumerate(((1, 0, EVERY, 0), (5, 0, EVERY, vocab + 1), (4, 9, EVERY, vocab + 3), (3, 5, (), 0), (3, 40, ("tree", "presence"), 0),
                                                    (4, 6, ("history", "frequency"), 0), (4, 6, ("mask",), vocab + 8), (4, 6, ("bias", "repetition"), 0))):
        trees = None if n_hi == 0 else [grow(rng, rng.randrange(0, n_hi + 1) if i else n_hi, "forest") for i in range(B)]
        check_logits(rng, trees, B, vocab, dtype, seed + vocab, parts, pitch, in_place=seed % 2 == 1)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("B,vocab", ((60, 37), (50, 1096), (3, 17000)))
def test_logits_of_trees_that_share_blocks(B, vocab, dtype):
    """More rows than blocks take one by one, most tokens on several nodes: each row counts its own path's."""
    rng = random.Random(B)
    for seed, (parts, pitch) in enumerate(((EVERY, 0), (("tree", "frequency", "repetition"), vocab + 1), (("tree", "presence", "mask"), vocab + 8))):
        trees = [grow(rng, rng.choice((64, 63, 256, 0)), rng.choice(("tree", "chain", "wide"))) for i in range(B)]
        for in_place in (False, True):
            check_logits(rng, trees, B, vocab, dtype, seed, parts, pitch, in_place=in_place)


def test_logits_of_one_row_and_none():
    s = synera()
    check_logits(random.Random(1), [[], [-1], []], 3, 129, "f32", 1, EVERY)
    assert s.adjust_logits(torch.empty((0, 50), device=DEV), cu=i32([0, 0])).shape == (0, 50)
    x = draw((3, 50), 1, torch.float32)
    assert torch.equal(s.adjust_logits(x), x)


def test_logits_long_paths_and_histories():
    """A chain of more rows than a tree of the cache may have, histories beyond a block's own width, one token all over."""
    rng = random.Random(2)
    check_logits(rng, [grow(rng, 700, "chain"), grow(rng, 3, "tree"), grow(rng, 300, "tree")], 3, 500, "f32", 3, ("tree", "frequency", "presence", "repetition"))
    s = synera()
    history = torch.full((2, 200000), 5, dtype=torch.int32, device=DEV)
    history[0, ::2] = 7
    x = torch.zeros((2, 9000), device=DEV)
    out = s.adjust_logits(x, history=history, history_len=i32([200000, 100001]), n_prompt=i32([0, 1]), frequency=torch.full((2,), 0.5, device=DEV))
    assert out[0, 5] == -50000 and out[0, 7] == -50000 and out[1, 5] == -50000 and (out != 0).sum() == 3


def test_logits_of_a_long_tree_and_its_splits():
    """Rows of one request whose paths are long and part ways: each is what it is by itself."""
    s, rng, n, vocab = synera(), random.Random(4), 600, 3000
    parent = [-1] + [j - 1 if rng.random() < 0.9 else rng.randrange(-1, j) for j in range(1, n)]
    tokens = [rng.randrange(100) for _ in range(n)]
    x = draw((n, vocab), 7, torch.float32)
    freq = torch.full((1,), 0.25, device=DEV)
    out = s.adjust_logits(x, cu=i32([0, n]), tokens=i32(tokens), parent=i32(parent), frequency=freq)
    want = x.double().cpu()
    for j, path in enumerate(tree.paths(parent)):
        for t in path:
            want[j, tokens[t]] -= 0.25
    assert (out.cpu().double() - want).abs().max() < 4 * 2.0 ** -24 * (want.abs().max() + 100)


def test_logits_rows_and_parents_that_cannot_be():
    """Row ranges outside the rows are cut, parents that are not before their nodes end a path."""
    s = synera()
    x = torch.zeros((4, 40), device=DEV)
    pres = torch.ones(3, device=DEV)
    out = torch.full_like(x, 3.0)
    s.adjust_logits(x, cu=i32([-5, 2, 1, 99]), tokens=i32([1, 2, 3, 4]), parent=i32([0, 5, -3, 0]), presence=pres, out=out)
    want = torch.zeros((4, 40))
    want[0, 1] = want[1, 2] = -1                               # (the second request has no rows, the third begins at row 1)
    got = out.cpu()
    assert torch.equal(got[0], want[0])
    assert got[2, 3] == -1 and got[3, 4] == -1


# ------------------------------------------------------------------------------------------------ a step of a server
class Server:
    """The state of a serving loop whose lengths stay on the GPU, and its step: pages, plan, for each layer append and attention, logits,
    argmax, accepted path, commit.  Drafts, weights and logits are draws."""

    def __init__(self, B, cols, room, layers=2, hq=8, hkv=2, hd=64, vocab=640, spare=400, seed=0):
        s, self.s = synera(), synera()
        self.B, self.room, self.layers, self.vocab, self.heads = B, room, layers, vocab, (hq, hkv, hd)
        rng = np.random.RandomState(seed)
        self.table, self.held = i32(np.zeros((B, cols))), i32(np.zeros(B))
        self.free, self.n_free = i32(rng.permutation(spare)), i32([spare])
        self.ctx = i32(np.zeros(B))
        self.batch = s.TreeBatch(hq, hkv, hd, B, room, cols)
        self.rope = s.Rope(hd, layout="half")
        self.k, self.v = bits((layers, spare, hkv, P, hd), 0x7FC0), bits((layers, spare, hkv, hd, P), 0x7FC0)
        self.n, self.parent, self.tokens = i32(np.zeros(B)), i32(np.zeros(room)), i32(np.zeros(room))
        self.x = [draw((room, hq + 2 * hkv, hd), 1) for _ in range(layers)]
        self.logits = draw((room, vocab), 2, torch.float32, 2.0)
        self.given = i32(np.ones(B))
        self.history, self.pres = i32(np.zeros((B, cols * P))), torch.full((B,), 0.3, device=DEV)
        self.none = i32(np.zeros(B))

    def load(self, trees, seed):
        rng = random.Random(seed)
        flat = sum(trees, [])
        self.n.copy_(i32([len(t) for t in trees]))
        self.parent[: len(flat)] = i32(flat)
        tokens = [rng.randrange(self.vocab) for _ in flat]
        self.tokens[: len(flat)] = i32(tokens)
        for x in self.x:
            x.copy_(draw(x.shape, rng.randrange(1 << 20)))
        self.logits.copy_(draw(self.logits.shape, rng.randrange(1 << 20), torch.float32, 2.0))
        at = 0
        for t in trees:                                        # most nodes' argmax is some child's token
            for j in range(1, len(t)):
                if t[j] >= 0 and rng.random() < 0.8:
                    self.logits[at + t[j], tokens[at + j]] = 30.0
            at += len(t)

    def step(self):
        hq, hkv, _ = self.heads
        cu, pos, slot, status = self.s.update_pages(self.table, self.held, self.free, self.n_free, self.ctx, self.n, self.room)
        planned = self.batch.plan(self.ctx, self.n, self.parent, self.table, self.k.shape[1])
        outs = []
        for layer in range(self.layers):
            x = self.x[layer]
            q = self.batch.append_rope(self.rope, x[:, :hq], x[:, hq: hq + hkv], x[:, hq + hkv:], self.k[layer], self.v[layer])
            outs.append(self.batch.attention(q, self.k[layer], self.v[layer]))
        y = self.s.adjust_logits(self.logits, cu=cu, history=self.history, history_len=self.none, presence=self.pres, tokens=self.tokens,
                                 parent=self.parent)
        target, _, _ = self.s.confidence(y, want_prob=False, want_entropy=False)
        acc = self.batch.accept(self.tokens, target, n_given=self.given)
        self.batch.commit(acc["path"], acc["n_path"], self.k, self.v)
        self.ctx += acc["n_path"]
        _, _, _, after = self.s.update_pages(self.table, self.held, self.free, self.n_free, self.ctx, self.none, 0)
        return {"cu": cu, "slot": slot, "pos": pos, "status": status, "planned": planned, "o": outs, "y": y, "target": target, **acc, "after": after}

    def state(self):
        return [self.table, self.held, self.free, self.n_free, self.ctx, self.k, self.v]


def same(a, b, rows):
    """Outputs of two steps, over the rows that there are."""
    for name, x in a.items():
        y = b[name]
        if name == "o":
            assert all(torch.equal(p[:rows], q[:rows]) for p, q in zip(x, y)), name
        elif name in ("slot", "pos", "y", "target", "path"):
            assert torch.equal(x[:rows], y[:rows]), name
        else:
            assert torch.equal(x, y), name


def test_steps_of_a_server():
    """A run of all operators over steps of growing contexts, each against float64 over what the cache holds, the cache against a record of the text."""
    v = Server(6, 12, 80, seed=3)
    hq, hkv, hd = v.heads
    text = [[] for _ in range(6)]                              # what each request's cache should hold: (layer 0's key rows, values)
    for step in range(5):
        rng = random.Random(step)
        trees = [grow(rng, rng.randrange(0, 14) if i else 9, "tree") for i in range(6)]
        v.load(trees, step)
        ctx = v.ctx.cpu().numpy()
        k_then = None
        out = v.step()
        T = sum(map(len, trees))
        assert (out["status"] == 0).all() and (out["planned"] == 0).all()
        tokens, target = v.tokens.cpu().numpy()[:T], out["target"].cpu().numpy()[:T]
        want = tree.accept(trees, tokens, target, None, np.ones(6))
        for name, w in zip(("accept_len", "token", "n_path"), (want[0], want[1], want[3])):
            assert np.array_equal(out[name].cpu().numpy(), w), name
        assert np.array_equal(out["path"].cpu().numpy()[:T], want[2])
        assert np.array_equal(v.ctx.cpu().numpy(), ctx + want[3])
        # the cache holds the text: rows of the accepted nodes behind those of the steps before
        t = 0
        table = v.table.cpu().numpy()
        vals = v.x[1][:, hq + hkv:].clone()
        for i, tr in enumerate(trees):
            text[i] += [vals[t + int(j)] for j in want[2][t: t + int(want[3][i])]]
            t += len(tr)
            if text[i]:
                at = np.arange(len(text[i]))
                page, slot = torch.from_numpy(table[i, at // P].astype(np.int64)).to(DEV), torch.from_numpy(at % P).to(DEV)
                assert torch.equal(v.v[1][page, :, :, slot], torch.stack(text[i])), (step, i)
        # the attention of the last layer, over the cache as it was before the paths were moved: put together again from the text
        pool_k, pool_v = v.k[1].clone(), v.v[1].clone()
        t = 0
        b = v.s.TreeBatch(hq, hkv, hd, 6, 80, 12)
        state = [x.clone() for x in (v.table, v.held, v.free, v.n_free)]
        v.s.update_pages(*state, i32(ctx), v.n, 0)
        b.plan(i32(ctx), v.n, v.parent, state[0], v.k.shape[1])
        x = v.x[1]
        q = b.append_rope(v.rope, x[:, :hq], x[:, hq: hq + hkv], x[:, hq + hkv:], pool_k, pool_v)
        wo, _, eo, _ = tree.attention(ref.to64(q[:T]), ref.to64(pool_k), ref.to64(pool_v), ctx, trees, state[0].cpu().numpy(), hd ** -0.5)
        ref.close(ref.to64(out["o"][1][:T]), wo, eo, f"o of step {step}")
        assert k_then is None and (out["after"] == 0).all()
        assert np.array_equal(v.held.cpu().numpy(), -(-(ctx + want[3]) // P))


def test_captured_steps():
    """The whole step as a graph, replayed over growing contexts and other trees, against eager steps, with eager work between the replays."""
    a, b = Server(5, 10, 64, seed=4), Server(5, 10, 64, seed=4)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for v in (a, b):
            v.load([[-1], [-1, 0], [], [-1, 0, 0], [-1]], 99)
            v.step()
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            got = b.step()
        for step in range(6):
            rng = random.Random(step + 50)
            trees = [grow(rng, rng.randrange(0, 13), rng.choice(("tree", "chain", "forest"))) for _ in range(5)]
            if step == 3:
                trees = [[] for _ in range(5)]
            for v in (a, b):
                v.load(trees, step)
            graph.replay()
            want = a.step()
            side.synchronize()
            rows = sum(map(len, trees))
            same(got, want, rows)
            for x, y in zip(a.state(), b.state()):
                assert torch.equal(x.view(torch.uint8), y.view(torch.uint8)), step
            torch.cuda.synchronize()


def test_two_handles_on_two_streams():
    runs = []
    for i in range(2):
        ctx, trees, table, n = make(random.Random(i), 20, 500, 9)
        b, q, k, v = check_attention(8, 2, 64, ctx, trees, table, n, i)
        T = sum(map(len, trees))
        runs.append((b, q, k, v, b.attention(q, k, v)[:T].clone(), torch.cuda.Stream(), T))
    torch.cuda.synchronize()
    outs = [[], []]
    for _ in range(5):
        for i, (b, q, k, v, _, st, T) in enumerate(runs):
            with torch.cuda.stream(st):
                outs[i].append(b.attention(q, k, v)[:T])
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(o, runs[i][4]) for o in outs[i])


def test_refusals():
    """What the host can see is refused, and nothing is launched."""
    s = synera()
    ctx, trees, table, n = make(random.Random(1), 3, 40, 5, zero=0.0)
    b = planned(4, 2, 64, ctx, trees, table, n)
    T = sum(map(len, trees))
    k, v, q = draw((n, 2, P, 64), 1), draw((n, 2, 64, P), 2), draw((T, 4, 64), 3)
    with pytest.raises(ValueError):
        b.attention(q[:-1], k, v)                              # fewer rows than the plan's
    with pytest.raises(ValueError):
        b.attention(q, k[:-1], v)
    with pytest.raises(s.SyneraError):
        b.attention(q, k, v, out=q)
    for scale in (0.0, -1.0, float("nan")):
        with pytest.raises(ValueError):
            b.attention(q, k, v, scale=scale)
    for args in ((i32(ctx)[:2], i32([1, 1, 1]), i32([-1] * 3), i32(table), n), (i32(ctx).long(), i32([1, 1, 1]), i32([-1] * 3), i32(table), n),
                 (i32(ctx), i32([1, 1, 1]), i32([-1] * 3).cpu(), i32(table), n), (i32(ctx), i32([1, 1, 1]), i32([-1] * 3), i32(table)[:, :0], n)):
        with pytest.raises((ValueError, s.SyneraError)):
            b.plan(*args)
    for args, status in (((i32([0] * 4), i32([1] * 4), i32([-1] * 4), i32(np.zeros((4, 1))), 4), s.ENOSPC),
                         ((i32([0]), i32([1]), i32([-1] * (T + 1)), i32([[0]]), 4), s.ENOSPC),
                         ((i32([0]), i32([1]), i32([-1]), i32(np.zeros((1, table.shape[1] + 1))), 4), s.ENOSPC),
                         ((i32([0]), i32([1]), i32([-1]), i32([[0]]), 0), s.EINVAL), ((i32([0]), i32([1]), i32([-1]), i32([[0]]), 1 << 27), s.EUNSUP)):
        with pytest.raises(s.SyneraError) as e:
            b.plan(*args)
        assert e.value.status == status
    tok = i32(np.zeros(T))
    with pytest.raises(s.SyneraError):
        b.accept(tok, tok)                                     # neither anchor nor given nodes
    with pytest.raises(s.SyneraError):
        b.accept(tok[:-1], tok[:-1], anchor=i32([0] * 3))
    with pytest.raises(ValueError):
        b.accept(tok, tok[:-1], anchor=i32([0] * 3))
    good = b.accept(tok, tok, anchor=i32([0] * 3))
    for pools in ((k, k[:, :, :, :32]), (k[:-1], v[:-1]), (k.float(), v.float()), (k.view(n, 2, 64, P), v)):
        with pytest.raises((ValueError, s.SyneraError)):
            b.commit(good["path"], good["n_path"], *pools)
    with pytest.raises(s.SyneraError):
        b.commit(good["path"], good["n_path"], k, k.view(n, 2, 64, P))        # one on the other
    x = draw((4, 64), 1, torch.float32)
    for bad in (dict(history=i32(np.zeros((4, 3)))), dict(bias_id=i32(np.zeros((4, 3)))), dict(tokens=i32([0] * 4), parent=i32([0] * 4)), dict(cu=i32([0, 4]), tokens=i32([0] * 4)),
                dict(out=x[1:].new_empty((4, 64)).double()), dict(mask=i32(np.zeros((4, 3)))), dict(repetition=torch.ones(3, device=DEV)),
                dict(history=i32(np.zeros((4, 3))), history_len=i32([0] * 3))):
        with pytest.raises((ValueError, s.SyneraError)):
            s.adjust_logits(x, **bad)
    wide = draw((5, 64), 1, torch.float32)
    with pytest.raises(s.SyneraError):
        s.adjust_logits(wide[:4], out=wide[1:])
    for bad in (x.cpu(), x.double(), x.t()):
        with pytest.raises(ValueError):
            s.adjust_logits(bad)
