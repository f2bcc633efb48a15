"""Whole steps over trees of drafted tokens where something gives out on the way: pools that run dry, counts out of range, replayed plans of other
sizes; and the shapes of trees and paths that the tests of the single operators leave out."""
import gc
import random

import numpy as np
import pytest
import torch

import shared_reference as ref
import tree_reference as tree
from test_gpu_tree import DEV, EVERY, P, TYPES, Server, check_attention, check_logits, grow, i32, make, same, synera

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def nothing_left_behind():
    yield
    gc.collect()


# ------------------------------------------------------------------------------------------------ pools that run dry
class HeldServer(Server):
    """The server whose plans know how many pages each request holds."""

    def __init__(self, *args, **more):
        super().__init__(*args, **more)
        plan = self.batch.plan
        self.batch.plan = lambda *what: plan(*what, held=self.held)


def test_steps_whose_pool_runs_out():
    """Requests that the pool has no pages for are refused by all calls of the step: nothing of the cache changes but the places of the others' nodes, bit
    for bit, and what each request's cache holds is the record of its text.  Refused ones go on when others have left."""
    B, layers = 5, 2
    v = HeldServer(B, 12, 80, layers=layers, spare=9, seed=5)
    hq, hkv, hd = v.heads
    text = [[] for _ in range(B)]                              # of each request's cache: the rows of x that its positions come from, both layers
    freq, refused, again = ref.frequencies(hd), 0, 0
    was = np.zeros(B, np.int64)
    for step in range(14):
        rng = random.Random(step)
        trees = [grow(rng, rng.randrange(1, 14), "tree") for i in range(B)]
        if step in (7, 10):                                    # a request leaves, another one comes in its place
            text[step % B] = []
            v.ctx[step % B] = 0
        v.load(trees, step)
        before = [x.clone() for x in v.state()]
        ctx = v.ctx.cpu().numpy().astype(np.int64)
        out = v.step()
        T = sum(map(len, trees))
        status, table = out["status"].cpu().numpy(), v.table.cpu().numpy()
        assert np.array_equal(out["planned"].cpu().numpy(), status) and set(status) <= {0, v.s.ENOSPC}
        tokens, target = v.tokens.cpu().numpy()[:T], out["target"].cpu().numpy()[:T]
        want = tree.accept(trees, tokens, target, None, np.ones(B))
        cu = np.concatenate([[0], np.cumsum([len(t) for t in trees])])
        free = torch.ones(v.k.shape[1], P, dtype=torch.bool)   # places that no node of a request that is served has
        for i in range(B):
            path = out["path"].cpu().numpy()[cu[i]:cu[i + 1]]
            if status[i]:
                assert out["n_path"][i] == out["accept_len"][i] == 0 and out["token"][i] == -1 and (path == -1).all()
                continue
            at = ctx[i] + np.arange(len(trees[i]))
            free[table[i, at // P], at % P] = False
            assert out["n_path"][i] == want[3][i] and np.array_equal(path, want[2][cu[i]:cu[i + 1]])
            text[i] += [torch.stack([x[cu[i] + int(j), hq:] for x in v.x]) for j in path[:want[3][i]]]
        assert np.array_equal(v.ctx.cpu().numpy(), ctx + np.where(status == 0, want[3], 0))
        free = free.to(DEV)
        for x, y, dims in ((v.k, before[5], (None, slice(None), None, slice(None), None)), (v.v, before[6], (None, slice(None), None, None))):
            other = x.view(torch.int16) != y.view(torch.int16)
            assert not (other & free[dims]).any(), step
        for i in range(B):
            assert len(text[i]) == v.ctx[i]
            if not text[i]:
                continue
            at = np.arange(len(text[i]))
            page, slot = torch.from_numpy(table[i, at // P].astype(np.int64)).to(DEV), torch.from_numpy(at % P).to(DEV)
            rows = torch.stack(text[i])                        # [position, layer, keys and values, hd]
            for layer in range(layers):
                assert torch.equal(v.v[layer][page, :, :, slot], rows[:, layer, hkv:]), (step, i)
                keys, err = ref.turn(ref.to64(rows[:, layer, :hkv]), at, freq, "half")
                ref.close(ref.to64(v.k[layer][page, :, slot]), keys, np.abs(keys) * 2.0 ** -8 + err * (1 + 2.0 ** -8) + 1e-38, f"keys of {i} in step {step}")
        refused += 0 < (status != 0).sum() < B
        again += int(((was != 0) & (status == 0)).sum())
        was = status
    assert refused >= 3 and again >= 1                         # (some were refused while others went on, and some were served later)


def test_captured_steps_whose_pool_runs_out():
    a, b = (HeldServer(4, 10, 64, spare=6, seed=4) for _ in range(2))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    refused = 0
    with torch.cuda.stream(side):
        for v in (a, b):
            v.load([[-1], [-1, 0], [], [-1, 0, 0]], 99)
            v.step()
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            got = b.step()
        for step in range(9):
            rng = random.Random(step + 50)
            trees = [grow(rng, rng.randrange(0, 14), rng.choice(("tree", "chain", "forest"))) for _ in range(4)]
            for v in (a, b):
                if step == 6:
                    v.ctx[:2] = 0
                v.load(trees, step)
            graph.replay()
            want = a.step()
            side.synchronize()
            cu, bad = np.concatenate([[0], np.cumsum([len(t) for t in trees])]), want["planned"].cpu().numpy() != 0
            assert not bad[[len(t) > 0 and s == 0 for t, s in zip(trees, want["status"].tolist())]].any()
            refused += 0 < bad.sum() < 4
            rows = torch.cat([torch.arange(cu[i], cu[i + 1]) for i in range(4) if not bad[i]]).to(DEV)       # (a refused request has no outputs)
            some = [{n: [o[rows] for o in x] if n == "o" else x[rows] if n in ("y", "target") else x for n, x in w.items()} for w in (got, want)]
            for w in some:
                for name in ("slot", "pos", "path"):
                    w[name] = w[name][:cu[-1]]
            same(*some, int(cu[-1]))
            for x, y in zip(a.state(), b.state()):
                assert torch.equal(x.view(torch.uint8), y.view(torch.uint8)), step
            torch.cuda.synchronize()
    assert refused >= 2


def test_plans_by_held_pages():
    """A request is planned if it holds what its tokens and nodes need; where it holds what cannot be it is refused; and what the host can see."""
    s = synera()
    b = s.TreeBatch(2, 1, 64, 8, 20, 3)
    ctx, n, held = [20, 20, 20, 20, 0, 20, 20, 29], [3, 3, 3, 3, 2, 0, 0, 3], [2, 1, -1, 4, 1, 2, 0, 3]
    parent, table = i32([-1, 0, 0] * 4 + [-1, 0] + [-1, 0, 0]), i32(np.arange(24).reshape(8, 3))
    args = i32(ctx), i32(n), parent, table, 24
    assert b.plan(*args, held=i32(held)).tolist() == [0, s.ENOSPC, s.EINVAL, s.EINVAL, 0, 0, s.ENOSPC, 0]
    acc = b.accept(i32(np.zeros(17)), i32(np.zeros(17)), n_given=i32([1] * 8))
    assert acc["n_path"].tolist() == [2, 0, 0, 0, 2, 0, 0, 2]
    assert acc["path"].tolist() == [0, 1, -1] + [-1] * 9 + [0, 1] + [0, 1, -1]
    assert (b.plan(*args) == 0).all()
    for bad in (i32(held)[:7], i32(held).long(), i32(held).cpu()):
        with pytest.raises(ValueError):
            b.plan(*args, held=bad)
    from paper_2511_07423_amd import binding
    at = [x.data_ptr() for x in args[:4]]
    room = torch.zeros(16, dtype=torch.int32, device=DEV)
    for held_at, status_at in ((room.data_ptr() + 2, room.data_ptr() + 32), (room.data_ptr(), room.data_ptr() + 28)):
        assert binding._lib.synera_tree_plan_held(b._h, 8, at[0], at[1], at[2], 17, at[3], 3, held_at, 24, status_at,
                                                  torch.cuda.current_stream().cuda_stream) == s.EINVAL


# ------------------------------------------------------------------------------------------------ counts out of range
@pytest.mark.parametrize("n,columns,counted,status", [(300, 40, 300, "EINVAL"), (200, 8, 0, "ENOSPC"), (256, 16, 256, "ENOSPC"), (257, 16, 0, "EINVAL"), (257, 17, 257, "EINVAL"),
                                                      (640, 40, 640, "EINVAL"), (641, 40, 0, "EINVAL"), (-1, 8, 0, "EINVAL"), (2 ** 31 - 1, 8, 0, "EINVAL")])
def test_rows_of_a_step_with_a_count_out_of_range(n, columns, counted, status):
    """Page tables, plans, logits and accepted paths number rows alike, whatever one request's count is: the others are what they are without it."""
    s, (hq, hkv, hd), vocab = synera(), (4, 2, 64), 64
    trees, at = [[-1, 0, 0], [-1, 0, 1, 0], [-1, 0]], [0, 2, 4]
    ctx, new = i32([20, 9, 7, 5, 33]), i32([3, n, 4, -1, 2])
    T = 9 + counted
    first = [0, 3 + counted, 7 + counted]                      # rows of the three that can be
    rows = torch.cat([torch.arange(r, r + len(t)) for r, t in zip(first, trees)]).to(DEV)
    n_pages = 64
    table, held, free, n_free = i32(np.zeros((5, columns))), i32(np.zeros(5)), i32(np.random.RandomState(1).permutation(n_pages)), i32([n_pages])
    cu, pos, slot, refused = s.update_pages(table, held, free, n_free, ctx, new, T)
    assert cu.tolist() == [0, 3, 3 + counted, 7 + counted, 7 + counted, T]
    parent, tokens = torch.full((T,), -1, dtype=torch.int32, device=DEV), torch.full((T,), 1, dtype=torch.int32, device=DEV)
    parent[rows] = i32(sum(trees, []))
    tokens[rows] = i32(np.arange(9) + 2)
    logits = torch.zeros((T, vocab), device=DEV)
    follows = {0: 1, 1: 40, 2: 41, 3: 4, 4: 5, 5: 42, 6: 43, 7: 8, 8: 44}       # the target of each of the nine nodes, as a node's place among them or a token
    for node, then in follows.items():
        logits[rows[node], then + 2 if then < 9 else then] = 9.0
    b = s.TreeBatch(hq, hkv, hd, 5, 700, 41)
    for pages in (held, None):
        got = b.plan(ctx, new, parent, table, n_pages, held=pages)
        assert got.tolist() == [0, getattr(s, status), 0, s.EINVAL, 0]
    x = torch.randn((T, hq + 2 * hkv, hd), generator=torch.Generator(device=DEV).manual_seed(1), device=DEV).to(torch.bfloat16)
    k, v = torch.zeros((n_pages, hkv, P, hd), dtype=torch.bfloat16, device=DEV), torch.zeros((n_pages, hkv, hd, P), dtype=torch.bfloat16, device=DEV)
    k1, v1 = k.clone(), v.clone()
    rope = s.Rope(hd)
    mark = torch.full((T, hq, hd), 0x1234, dtype=torch.int16, device=DEV).view(torch.bfloat16)
    out_q, out = mark.clone(), mark.clone()
    b.append_rope(rope, x[:, :hq], x[:, hq: hq + hkv], x[:, hq + hkv:], k, v, out_q=out_q)
    b.attention(out_q, k, v, out=out)
    y = s.adjust_logits(logits, cu=cu, tokens=tokens, parent=parent, presence=torch.full((5,), 0.5, device=DEV))
    target, _, _ = s.confidence(y, want_prob=False, want_entropy=False)
    acc = b.accept(tokens, target, n_given=i32([1] * 5))
    # the same without the two that cannot be
    small = s.TreeBatch(hq, hkv, hd, 3, 9, 41)
    live = torch.tensor(at, device=DEV)
    assert (small.plan(ctx[live].contiguous(), new[live].contiguous(), i32(sum(trees, [])), table[live].contiguous(), n_pages) == 0).all()
    x1 = x[rows]
    q1 = small.append_rope(rope, x1[:, :hq], x1[:, hq: hq + hkv], x1[:, hq + hkv:], k1, v1)
    o1 = small.attention(q1, k1, v1)
    y1 = s.adjust_logits(logits[rows], cu=i32([0, 3, 7, 9]), tokens=tokens[rows], parent=i32(sum(trees, [])), presence=torch.full((3,), 0.5, device=DEV))
    acc1 = small.accept(tokens[rows], target[rows], n_given=i32([1] * 3))
    assert torch.equal(k, k1) and torch.equal(v, v1) and torch.equal(out_q[rows], q1) and torch.equal(out[rows], o1) and torch.equal(y[rows], y1)
    assert torch.equal(acc["path"][rows], acc1["path"]) and all(torch.equal(acc[name][live], acc1[name]) for name in ("accept_len", "n_path", "token"))
    assert acc1["accept_len"].tolist() == [1, 2, 1]
    other = torch.ones(T, dtype=torch.bool, device=DEV)
    other[rows] = False
    assert (acc["path"][other] == -1).all() and (out[other].view(torch.int16) == 0x1234).all() and (out_q[other].view(torch.int16) == 0x1234).all()
    assert (slot[rows] >= 0).all() and (refused == 0).tolist() == [True, n in (256, 257, 300, 640) and columns * P >= n + 9, True, False, True]


def test_rows_that_a_step_has_no_room_for():
    """Of a request that is refused for its count the rows that there are, then the requests behind are refused."""
    s = synera()
    b = s.TreeBatch(2, 1, 64, 4, 500, 40)
    table = i32(np.arange(160).reshape(4, 40))
    status = b.plan(i32([5, 0, 3, 0]), i32([2, 600, 3, 640]), i32([-1] * 400), table, 160)
    assert status.tolist() == [0, s.EINVAL, s.ENOSPC, s.EINVAL]
    acc = b.accept(i32(np.zeros(400)), i32(np.zeros(400)), n_given=i32([1] * 4))
    assert acc["n_path"].tolist() == [1, 0, 0, 0] and acc["path"].tolist() == [0] + [-1] * 399
    # sums beyond 32 bits
    many = s.TreeBatch(2, 1, 64, 2000, 500, 40000)
    table = i32(np.zeros((2000, 40000)))
    status = many.plan(i32([0] * 2000), torch.full((2000,), 640000, dtype=torch.int32, device=DEV), i32([-1] * 400), table, 1)
    assert (status == s.EINVAL).all()
    acc = many.accept(i32(np.zeros(400)), i32(np.zeros(400)), n_given=i32([1] * 2000))
    assert (acc["n_path"] == 0).all() and (acc["path"] == -1).all()


@pytest.mark.parametrize("B,n_rows", [(1, 1), (3, 7), (3, 50), (3, 4096), (3, 4097), (3, 70001), (1500, 2500), (1500, 1)])
def test_places_behind_the_last_token(B, n_rows):
    """A step whose rows have room for more tokens than there are: the others' places are none, whatever the memory held."""
    s, rng = synera(), np.random.RandomState(B)
    new = rng.randint(0, 3, size=B) if n_rows > 1 else np.zeros(B, np.int64)
    ctx, columns = rng.randint(0, 40, size=B), 3
    free = rng.permutation(3 * B)
    for step in range(3):
        junk = [torch.full((2 * B + 1 + 2 * n_rows,), 5, dtype=torch.int32, device=DEV) for _ in range(2)]
        del junk                                               # what the next outputs may lie in
        cu, pos, slot, status = s.update_pages(i32(np.zeros((B, columns))), i32(np.zeros(B)), i32(free), i32([3 * B]), i32(ctx), i32(new), n_rows)
        T = min(int(new.sum()), n_rows)
        assert (status == 0).all() and cu[-1] == new.sum()
        assert (pos[:T] >= 0).all() and (slot[:T] >= 0).all() and (pos[T:] == -1).all() and (slot[T:] == -1).all()


def test_pages_of_more_requests_than_a_launch_has_blocks_for():
    """2^24 requests and some: with 256 threads each the places' launch would have more than 2^32."""
    s, B = synera(), (1 << 24) + 3
    zeros = torch.zeros(B, dtype=torch.int32, device=DEV)
    new, table, held = zeros.clone(), torch.full((B, 1), -5, dtype=torch.int32, device=DEV), zeros.clone()
    some = torch.tensor([0, 1 << 20, (1 << 20) + 1, 1 << 23, (1 << 24) - 1, 1 << 24, B - 1], device=DEV)
    new[some] = 3
    cu, pos, slot, status = s.update_pages(table, held, i32([9, 8, 7, 6, 5, 4, 3]), i32([7]), zeros, new, 30)
    assert (status == 0).all() and cu[-1] == 21 and int(held.sum()) == 7
    assert pos.tolist() == [0, 1, 2] * 7 + [-1] * 9 and table[some, 0].tolist() == [3, 4, 5, 6, 7, 8, 9]
    assert slot.tolist() == [16 * page + j for page in (3, 4, 5, 6, 7, 8, 9) for j in range(3)] + [-1] * 9


def test_as_many_requests_as_a_handle_may_have():
    args = make(random.Random(1), 1 << 14, 40, 2, zero=0.1)
    check_attention(2, 1, 64, *args, 3)


# ------------------------------------------------------------------------------------------------ replayed plans
def step_of(b, s, rope, x, k, v, tokens, target, given):
    """All calls behind a plan, with what they leave; x [rows, heads, hd], pools of both layers."""
    hq, hkv = b.n_q_heads, b.n_kv_heads
    q = b.append_rope(rope, x[:, :hq], x[:, hq: hq + hkv], x[:, hq + hkv:], k[1], v[1])
    o, lse = b.attention(q, k[1], v[1], want_lse=True)
    acc = b.accept(tokens, target, n_given=given)
    b.commit(acc["path"], acc["n_path"], k, v)
    return [q, o, lse, acc["path"], acc["n_path"], acc["accept_len"], acc["token"]]


@pytest.mark.parametrize("called", ["no rows", "no rows, fewer requests of no tables", "one row"])
def test_eager_calls_behind_a_replayed_plan(called):
    """The last plan that was called had no rows, or few; the one on the device, which a graph has replayed since, is what eager calls work on."""
    s, (hq, hkv, hd), B = synera(), (4, 2, 64), 4
    ctx, trees, table, n = make(random.Random(21), B, 600, 30, shapes=("tree",), zero=0.0)
    T = sum(map(len, trees))
    args = i32(ctx), i32([len(t) for t in trees]), i32(sum(trees, [])), i32(table), n
    rope = s.Rope(hd)
    gen = torch.Generator(device=DEV).manual_seed(3)
    x = torch.randn((T, hq + 2 * hkv, hd), generator=gen, device=DEV).to(torch.bfloat16)
    pools = [torch.randn(d, generator=gen, device=DEV).to(torch.bfloat16) for d in ((2, n, hkv, P, hd), (2, n, hkv, hd, P))]
    tokens, given = i32(np.zeros(T)), i32(np.ones(B))          # (every target is the first child's token)
    plain = s.TreeBatch(hq, hkv, hd, B, T, table.shape[1])
    assert (plain.plan(*args) == 0).all()
    k, v = (p.clone() for p in pools)
    want = [*step_of(plain, s, rope, x, k, v, tokens, tokens, given), k, v]
    assert (want[4] > 1).any()

    b = s.TreeBatch(hq, hkv, hd, B, T, table.shape[1])
    b.plan(*args)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            b.plan(*args)
        for _ in range(3):
            if called == "one row":
                b.plan(args[0], i32([0, 1, 0, 0]), i32([-1]), args[3], n)
            else:
                b.plan(args[0], i32(np.zeros(B)), i32([]), args[3] if called == "no rows" else i32(np.zeros((B, 1))), n)
            graph.replay()
            k, v = (p.clone() for p in pools)
            got = [*step_of(b, s, rope, x, k, v, tokens, tokens, given), k, v]
            side.synchronize()
            for w, g in zip(want, got):
                assert torch.equal(w, g)


def test_eager_calls_on_no_rows_behind_a_replayed_plan():
    """Plans of no rows in a handle whose plans were captured: calls on empty tensors do nothing."""
    s, (hq, hkv, hd) = synera(), (2, 1, 64)
    b = s.TreeBatch(hq, hkv, hd, 2, 4, 2)
    rope, table = s.Rope(hd), i32([[0, 1], [2, 3]])
    some, none = (i32([3, 5]), i32([2, 1]), i32([-1, 0, -1]), table, 4), (i32([3, 5]), i32([0, 0]), i32([]), table, 4)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        b.plan(*some)
    graph.replay()
    b.plan(*none)
    k, v = torch.zeros((2, 4, hkv, P, hd), dtype=torch.bfloat16, device=DEV), torch.zeros((2, 4, hkv, hd, P), dtype=torch.bfloat16, device=DEV)
    x = torch.ones((0, hq + 2 * hkv, hd), dtype=torch.bfloat16, device=DEV)
    got = step_of(b, s, rope, x, k, v, i32([]), i32([]), i32([1, 1]))
    assert got[4].tolist() == [0, 0] and (k == 0).all() and (v == 0).all()
    # as C sees them: no rows, no addresses
    from paper_2511_07423_amd import binding
    heads = [binding._pack_heads_rows(0, 0, 0, h, 0, h * hd, hd, h * hd, hd) for h in (hq, hkv)]
    stream = torch.cuda.current_stream().cuda_stream
    assert binding._lib.synera_tree_append_rope(b._h, rope._h, 1, heads[0], heads[1], heads[1], 0.0, k[0].data_ptr(), v[0].data_ptr(), stream) == s.OK
    assert binding._lib.synera_tree_attention(b._h, heads[0], k[0].data_ptr(), v[0].data_ptr(), 1.0, None, stream) == s.OK
    # one row whose steps from token to token, which one token does not need, are none: checked for the one that the last called plan has
    b.plan(i32([3, 5]), i32([0, 1]), i32([-1]), table, 4)
    x = torch.ones((1, hq + 2 * hkv, hd), dtype=torch.bfloat16, device=DEV)
    out = torch.zeros((1, hq, hd), dtype=torch.bfloat16, device=DEV)
    at = [binding._pack_heads_rows(x[:, i].data_ptr(), o, 0, h, 0, 0, hd, 0, hd) for i, h, o in ((0, hq, out.data_ptr()), (hq, hkv, 0), (hq + hkv, hkv, 0))]
    assert binding._lib.synera_tree_append_rope(b._h, rope._h, 1, *at, 0.0, k[0].data_ptr(), v[0].data_ptr(), stream) == s.OK
    assert (out != 0).any() and (k[0] != 0).any()
    k.zero_(), v.zero_()
    assert binding._lib.synera_tree_attention(b._h, binding._pack_heads_rows(x.data_ptr(), out.data_ptr(), 0, hq, 0, 0, hd, 0, hd), k[0].data_ptr(), v[0].data_ptr(), 1.0,
                                              None, stream) == s.OK
    torch.cuda.synchronize()
    assert (k == 0).all() and (v == 0).all()


def test_accept_and_commit_are_checked_for_the_rows_that_they_say():
    """A plan that is replayed later may have as many rows as the call's arrays: addresses and overlaps are checked for all of them."""
    s = synera()
    from paper_2511_07423_amd import binding
    lib, (hq, hkv, hd) = binding._lib, (2, 1, 64)
    b = s.TreeBatch(hq, hkv, hd, 2, 16, 2)
    table = i32([[0, 1], [2, 3]])
    k, v = torch.zeros((4, hkv, P, hd), dtype=torch.bfloat16, device=DEV), torch.zeros((4, hkv, hd, P), dtype=torch.bfloat16, device=DEV)
    rows, out = torch.zeros((2, 16), dtype=torch.int32, device=DEV), torch.zeros((3, 2), dtype=torch.int32, device=DEV)
    room = torch.zeros(64, dtype=torch.int32, device=DEV)
    tok, tgt, path, stream = rows[0].data_ptr(), rows[1].data_ptr(), room.data_ptr(), torch.cuda.current_stream().cuda_stream
    given = i32([1, 1]).data_ptr()

    def accept(n, tokens, target, path, n_path=out[2].data_ptr()):
        return lib.synera_tree_accept(b._h, n, tokens, target, None, given, out[0].data_ptr(), out[1].data_ptr(), path, n_path, stream)
    for n_nodes, parent in ((i32([0, 0]), i32([])), (i32([1, 1]), i32([-1, -1]))):
        assert (b.plan(i32([3, 5]), n_nodes, parent, table, 4) == 0).all()
        for bad in ((16, None, tgt, path), (16, tok, None, path), (16, tok, tgt, None), (16, tok, tgt, tok + 60), (16, tok, tgt, tgt - 8),
                    (16, tok, tgt, path, path + 60), (16, tok, tgt, path, tgt + 60)):
            assert accept(*bad) == s.EINVAL, bad
        assert lib.synera_tree_commit(b._h, 16, None, out[2].data_ptr(), 1, 0, k.data_ptr(), v.data_ptr(), stream) == s.EINVAL
        assert accept(16, tok, tgt, path) == s.OK and accept(16, tok, tgt, path, path + 64) == s.OK
        assert accept(1 << 62, tok, tgt, path, path + 60) == s.EINVAL and accept(1 << 62, tok, tgt, path, path + 64) == s.OK
        assert lib.synera_tree_commit(b._h, 16, path, out[2].data_ptr(), 1, 0, k.data_ptr(), v.data_ptr(), stream) == s.OK
    torch.cuda.synchronize()


@pytest.mark.parametrize("hd,dtype", [(64, torch.bfloat16), (128, torch.float32)])
def test_replayed_plans_with_more_rows_than_the_tensors(hd, dtype):
    """Wherever the tensors end, between two requests or inside one: the requests that lie in them whole are appended as ever, and of the
    others no key, value or query is written."""
    s, hq, hkv, B = synera(), 4, 2, 6
    ctx, trees, table, n = make(random.Random(22), B, 100, 40, shapes=("tree",), zero=0.0)
    trees[3], new = [], [len(t) for t in trees]
    new[3] = 0
    T, cu = sum(new), np.concatenate([[0], np.cumsum(new)])
    args = i32(ctx), i32(new), i32(sum(trees, [])), i32(table), n
    rope = s.Rope(hd)
    gen = torch.Generator(device=DEV).manual_seed(4)
    x = torch.randn((T, hq + 2 * hkv, hd), generator=gen, device=DEV).to(dtype)
    mark = lambda *shape: torch.full(shape, 0x1234, dtype=torch.int16, device=DEV).view(torch.bfloat16)       # noqa: E731
    b = s.TreeBatch(hq, hkv, hd, B, T, table.shape[1])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        b.plan(*args)
        with torch.cuda.graph(graph, stream=side):
            b.plan(*args)
        graph.replay()
        k, v, q = mark(n, hkv, P, hd), mark(n, hkv, hd, P), mark(T, hq, hd)
        b.append_rope(rope, x[:, :hq], x[:, hq: hq + hkv], x[:, hq + hkv:], k, v, out_q=q)
        for cut in sorted({1, T, *cu[1:].tolist(), *(cu[1:-1] + 1).tolist(), *(cu[2:] - 1).tolist()}):
            if not 0 < cut <= T:
                continue
            whole = int((cu <= cut).sum()) - 1                 # requests that end by then
            few = int(cu[whole])
            b.plan(*(i32([0]), i32([0]), i32([])), i32([[0]]), n)
            graph.replay()
            kp, vp, out_q = mark(n, hkv, P, hd), mark(n, hkv, hd, P), mark(T, hq, hd)
            y = x[:cut]
            b.append_rope(rope, y[:, :hq], y[:, hq: hq + hkv], y[:, hq + hkv:], kp, vp, out_q=out_q[:cut])
            side.synchronize()
            assert torch.equal(out_q[:few], q[:few]) and (out_q[few:].view(torch.int16) == 0x1234).all(), cut
            there = torch.zeros((n, P), dtype=torch.bool)
            for i in range(whole):
                at = int(ctx[i]) + np.arange(new[i])
                there[table[i, at // P], at % P] = True
            there = there.to(DEV)
            assert torch.equal(kp, torch.where(there[:, None, :, None], k, mark(1))), cut
            assert torch.equal(vp, torch.where(there[:, None, None, :], v, mark(1))), cut


# ------------------------------------------------------------------------------------------------ wide trees, long paths that part ways
def wide(rng, n):
    """Parents up to 200 nodes back: in other words of the masks and, with several heads, in other tiles."""
    return [-1] + [max(0, j - rng.randrange(1, 201)) for j in range(1, n)]


@pytest.mark.parametrize("hq,hkv,hd", [(16, 2, 64), (12, 1, 128), (3, 3, 64)])
def test_attention_of_wide_trees(hq, hkv, hd):
    rng = random.Random(hq)
    for ctx in ((0, 700, 33, 127), (129, 0, 5, 1000)):
        trees = [wide(rng, n) for n in (256, 200, 64, 129)]
        need = [-(-(c + len(t)) // P) for c, t in zip(ctx, trees)]
        ids, table, at = rng.sample(range(sum(need)), sum(need)), np.full((len(need), max(need)), -1, np.int32), 0
        for i, k in enumerate(need):
            table[i, :k] = ids[at:at + k]
            at += k
        check_attention(hq, hkv, hd, np.array(ctx), trees, table, sum(need), 7)


def test_attention_of_many_rows_behind_a_long_context():
    """2048 rows over 315 steps of 128 keys: ranges of two steps would have 323 584 partial rows, more than there is room for on any card of up to 1264 compute
    units (256 rows for each)."""
    rng, need = random.Random(12), -(-(40000 + 256) // P)
    table = np.array([rng.sample(range(need), need)], np.int32)
    check_attention(8, 1, 64, np.array([40000]), [wide(rng, 256)], table, need, 5)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("B,vocab,shape", [(24, 1000, "forest"), (24, 1000, "tree"), (8, 9001, "wide")])
def test_logits_of_long_trees_that_part_ways(B, vocab, shape, dtype):
    """Trees of more than 256 nodes of which a block takes several rows, some 64 or 96 apart (1536 blocks share them): from one to the next a path is extended,
    or taken away and another one added.  All penalties, biases and masks, new tensors and in place."""
    rng = random.Random(B + vocab)
    for seed, (parts, in_place) in enumerate(((EVERY, False), (EVERY, True), (("tree", "frequency", "presence", "repetition"), True))):
        trees = [(wide(rng, n) if shape == "wide" else grow(rng, n, shape)) for n in (rng.randrange(257, 300) for _ in range(B - 1))] + [grow(rng, 40, "tree")]
        check_logits(rng, trees, B, vocab, dtype, seed, parts, in_place=in_place)


@pytest.mark.parametrize("dtype", TYPES)
def test_logits_of_wide_trees(dtype):
    rng = random.Random(3)
    for in_place in (False, True):
        check_logits(rng, [wide(rng, n) for n in (256, 100, 3, 255)] * 10, 40, 1096, dtype, 5, EVERY, pitch=1097, in_place=in_place)
