"""GPU parity of appends with the rotation and of attention over shared prefixes with float64: element by element, over random trees of
shared pages whose unwritten slots hold NaN."""
import ctypes as C
import gc
import random

import numpy as np
import pytest
import torch

import shared_reference as ref
from test_shared_plan_cpu import make_batch

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


def draw(shape, seed, dtype=torch.bfloat16, scale=1.0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return (torch.randn(shape, generator=g, device=DEV) * scale).to(dtype)


def bits(shape, value):
    return torch.full(shape, value, dtype=torch.int16, device=DEV).view(torch.bfloat16)


def filled_pools(ctx, new, table, n_pages, hkv, hd, seed, junk=0x7FC0, spare=2):
    """Pools in which every position that a request holds or appends has values and everything else is junk (NaN)."""
    k, v = bits((n_pages + spare, hkv, P, hd), junk), bits((n_pages + spare, hkv, hd, P), junk)
    live = torch.zeros((n_pages + spare, P), dtype=torch.bool)
    for c, n, row in zip(ctx, new, table):
        at = np.arange(c + n)
        live[row[at // P], at % P] = True
    live = live.to(DEV)
    k = torch.where(live[:, None, :, None], draw(k.shape, seed), k)
    v = torch.where(live[:, None, None, :], draw(v.shape, seed + 1), v)
    return k.contiguous(), v.contiguous()


def planned(hq, hkv, hd, ctx, new, table, n_pages, more=0):
    b = synera().SharedBatch(hq, hkv, hd, len(ctx) + more, max(1, int(new.sum())) + more, table.shape[1] + more)
    b.plan(ctx, new, table, n_pages)
    return b


def check_attention(hq, hkv, hd, ctx, new, table, n_pages, seed, scale=None, std=1.5):
    b = planned(hq, hkv, hd, ctx, new, table, n_pages)
    k, v = filled_pools(ctx, new, table, n_pages, hkv, hd, seed)
    T = int(new.sum())
    q = draw((T + 3, hq, hd), seed + 2, scale=std)
    out = bits((T + 3, hq, hd), 0x1234)
    got, lse = b.attention(q, k, v, scale=scale, out=out, want_lse=True)
    want, want_lse, eo, el = ref.attention(ref.to64(q)[:T], ref.to64(k), ref.to64(v), ctx, new, table, hd ** -0.5 if scale is None else scale)
    ref.close(ref.to64(got)[:T], want, eo, "o")
    ref.close(ref.to64(lse)[:T], want_lse, el, "lse")
    assert torch.equal(got[T:].view(torch.int16), bits((3, hq, hd), 0x1234).view(torch.int16))     # rows behind the batch stay
    return b, q, k, v


@pytest.mark.parametrize("seed", range(16))
def test_attention_trees(seed):
    rng = random.Random(seed)
    B = rng.choice((1, 2, 5, 20))
    hkv = rng.choice((1, 2, 3))
    hq, hd = hkv * rng.choice((1, 3, 4, 7, 16)), rng.choice((64, 128))
    ctx, new, table, n_pages = make_batch(rng, B, max_new=rng.choice((1, 4, 33)), max_own=rng.choice((0, 30, 500)))
    check_attention(hq, hkv, hd, ctx, new, table, n_pages, seed * 10)


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("ctx,new", [(0, 1), (0, 2), (15, 1), (16, 1), (31, 1), (32, 1), (127, 1), (128, 2), (255, 3), (256, 1), (257, 9), (1000, 40),
                                     (5000, 1), (0, 300), (77, 150)])
def test_attention_one_request(ctx, new, hd):
    """Lengths around pages, tiles and cuts; one token and long chunks; every class of rows."""
    n = -(-(ctx + new) // P)
    table = np.random.RandomState(ctx).permutation(n).astype(np.int32)[None]
    for hq, hkv in ((1, 1), (8, 2)):
        check_attention(hq, hkv, hd, np.array([ctx], np.int32), np.array([new], np.int32), table, n, ctx + new)


def shared_batch(B, shared, own, new, seed=0):
    """B requests behind `shared` common pages, with own[i] more cached tokens and new[i] new ones."""
    own, new = np.broadcast_to(own, B), np.broadcast_to(new, B).astype(np.int32)
    ctx = (shared * P + own).astype(np.int32)
    need = -(-(ctx + new) // P)
    table = np.full((B, int(need.max())), -1, np.int32)
    at = shared
    perm = np.random.RandomState(seed).permutation(shared + int((need - shared).sum())).astype(np.int32)
    for i in range(B):
        table[i, : need[i]] = perm[np.concatenate([np.arange(shared), at + np.arange(need[i] - shared)])]
        at += need[i] - shared
    return ctx, new, table, len(perm)


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("B,shared,own,new", [(2, 8, 0, 1), (40, 33, 5, 1), (70, 9, 40, 2), (9, 40, 0, 20), (3, 65, 17, 64)])
def test_attention_shared(B, shared, own, new, hd):
    rs = np.random.RandomState(B)
    ctx, new, table, n = shared_batch(B, shared, rs.randint(0, own + 1, B), rs.randint(1, new + 1, B), B)
    check_attention(8, 2, hd, ctx, new, table, n, B)


def test_attention_repeats_bit_for_bit():
    ctx, new, table, n = shared_batch(30, 20, 7, 3)
    b, q, k, v = check_attention(8, 2, 128, ctx, new, table, n, 1)
    T = int(new.sum())                                         # (a new output's rows behind the batch are whatever they were)
    first = b.attention(q, k, v)[:T]
    for _ in range(3):
        assert torch.equal(b.attention(q, k, v)[:T], first)


def test_attention_scales_and_large_scores():
    ctx, new, table, n = shared_batch(5, 10, 3, 2)
    for scale, std in ((1e-4, 1.0), (1.0, 1.5), (7.0, 3.0)):
        check_attention(4, 2, 64, ctx, new, table, n, 3, scale=scale, std=std)


def test_attention_strides():
    """Queries inside a fused array, outputs with tokens inside heads."""
    s, hq, hkv, hd = synera(), 6, 2, 64
    ctx, new, table, n = shared_batch(6, 9, 4, 5)
    b = planned(hq, hkv, hd, ctx, new, table, n, more=3)
    k, v = filled_pools(ctx, new, table, n, hkv, hd, 5)
    T = int(new.sum())
    q = draw((T, hq + 2 * hkv, hd), 6)[:, :hq]
    plain = b.attention(q.contiguous(), k, v)
    assert torch.equal(b.attention(q, k, v), plain)
    out = torch.zeros((hq, T, hd), dtype=torch.bfloat16, device=DEV).transpose(0, 1)
    assert b.attention(q, k, v, out=out) is out and torch.equal(out, plain)


def test_attention_hidden_values():
    """Infinities and NaN: of a key or value, they reach the rows that see it and no other; of a query, its own row."""
    hq, hkv, hd = 4, 2, 128
    for bad in (float("inf"), float("-inf"), float("nan")):
        ctx, new, table, n = shared_batch(3, 8, np.array([0, 21, 40]), np.array([1, 12, 40]))
        b = planned(hq, hkv, hd, ctx, new, table, n)
        k, v = filled_pools(ctx, new, table, n, hkv, hd, 5)
        pos = ctx[1] + 7                                       # seen by rows 7 .. 11 of request 1 alone
        v[table[1, pos // P], 1, 5, pos % P] = bad
        pos = ctx[2] + 33
        k[table[2, pos // P], 0, pos % P, 9] = float("nan")    # rows 33 .. 39 of request 2
        q = draw((int(new.sum()), hq, hd), 6)
        q[0, 3, 0] = float("nan")
        got, lse = b.attention(q, k, v, want_lse=True)
        want, wl, eo, el = ref.attention(ref.to64(q), ref.to64(k), ref.to64(v), ctx, new, table, hd ** -0.5)
        ref.close(ref.to64(got), want, eo, f"o with {bad}")
        ref.close(ref.to64(lse), wl, el, f"lse with {bad}")


def check_append(hq, hkv, hd, rot, layout, dtype, ctx, new, table, n_pages, seed, norm=False, shift=0, with_q=True, scaling=None):
    s = synera()
    rope = s.Rope(hd, rot, layout=layout, scaling=scaling)
    b = planned(hq, hkv, hd, ctx, new, table, n_pages)
    T = int(new.sum())
    width = (hq + 2 * hkv) * hd
    flat = draw((T * width + 16,), seed, TYPES[dtype], 2.0)
    x = flat[shift: shift + T * width].view(T, hq + 2 * hkv, hd)
    q, k, v = x[:, :hq], x[:, hq: hq + hkv], x[:, hq + hkv:]
    gq, gk = (draw((hd,), 5) + 1, draw((hd,), 6) + 1) if norm else (None, None)
    kp, vp = bits((n_pages + 1, hkv, P, hd), 0x1234), bits((n_pages + 1, hkv, hd, P), 0x4321)
    oq = b.append_rope(rope, q if with_q else None, k, v, kp, vp, q_gain=gq, k_gain=gk, eps=1e-5)
    pos = np.concatenate([c + np.arange(m) for c, m in zip(ctx, new)]).astype(np.int64)
    req = np.repeat(np.arange(len(ctx)), new)
    freq = ref.frequencies(rot, scaling=scaling)
    step = 2.0 ** -8
    if with_q:
        want, err = ref.turn(ref.to64(q), pos, freq, layout, 1.0, None if gq is None else ref.to64(gq), 1e-5)
        ref.close(ref.to64(oq), want, np.abs(want) * step + err * (1 + step) + 1e-38, "q")
    else:
        assert oq is None
    want, err = ref.turn(ref.to64(k), pos, freq, layout, 1.0, None if gk is None else ref.to64(gk), 1e-5)
    page, slot = torch.from_numpy(table[req, pos // P].astype(np.int64)).to(DEV), torch.from_numpy(pos % P).to(DEV)
    ref.close(ref.to64(kp[page, :, slot]), want, np.abs(want) * step + err * (1 + step) + 1e-38, "k")
    assert torch.equal(vp[page, :, :, slot], v.to(torch.bfloat16))
    kp[page, :, slot] = bits((), 0x1234)                       # everything else is as it was
    vp[page, :, :, slot] = bits((), 0x4321)
    assert (kp.view(torch.int16) == 0x1234).all() and (vp.view(torch.int16) == 0x4321).all()


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("layout", ["interleaved", "half"])
@pytest.mark.parametrize("hd,rot,hq,hkv", [(128, 128, 8, 2), (64, 64, 3, 3), (64, 20, 4, 1), (128, 64, 2, 1), (128, 6, 5, 5)])
def test_append(hd, rot, hq, hkv, layout, dtype):
    for seed, (B, new, own) in enumerate(((1, 1, 0), (7, 1, 40), (6, 20, 40), (2, 90, 7))):
        ctx, n, table, pages = make_batch(random.Random(seed + hd), B, max_new=new, max_own=own, zero=0.2 if B > 2 else 0.0)
        if n.sum() == 0:
            n[0] = 1
            continue
        check_append(hq, hkv, hd, rot, layout, dtype, ctx, n, table, pages, seed, norm=seed % 2 == 0, shift=(0, 8, 1, 2)[seed], with_q=seed != 1,
                     scaling=(None, ("linear", 4.0), ("bands", 8.0, 1.0, 4.0, 64.0), None)[seed])


def test_append_writes_what_rope_and_kv_append_write():
    """The keys an append turns are those that Rope.apply turns, and its pages those of Verifier.kv_append, bit for bit."""
    import workloads as wl
    from helpers import drawn_model, small_shape
    s = synera()
    shape = small_shape(d_model=256, n_q_heads=4, n_kv_heads=4, head_dim=64, d_ffn=128, vocab=128, n_layers=1)
    head, layers = drawn_model(shape, 1, DEV)
    ver = s.Verifier(shape, head, layers, 4, 200, 8)
    ctx, new = np.array([0, 9, 40], np.int32), np.array([50, 3, 1], np.int32)
    table = np.arange(24, dtype=np.int32).reshape(3, 8)
    x = draw((54, 12, 64), 3)
    rope = s.Rope(64, layout="half")
    pos = torch.from_numpy(np.concatenate([c + np.arange(n) for c, n in zip(ctx, new)]).astype(np.int32)).to(DEV)
    q1, k1 = rope.apply(pos, x[:, :4], x[:, 4:8])
    pools = [bits((24, 4, 16, 64), 0), bits((24, 4, 64, 16), 0), bits((1, 24, 4, 16, 64), 0), bits((1, 24, 4, 64, 16), 0)]
    ver.kv_append(0, ctx, new, k1, x[:, 8:].contiguous(), table, 24, pools[2], pools[3])
    b = planned(4, 4, 64, ctx, new, table, 24)
    assert torch.equal(b.append_rope(rope, x[:, :4], x[:, 4:8], x[:, 8:], pools[0], pools[1]), q1)
    assert torch.equal(pools[0], pools[2][0]) and torch.equal(pools[1], pools[3][0])
    ver.close()


def test_steps_of_a_decoder_layer():
    """As a server runs them: norms, rotation, append and attention over three steps of a batch that shares a prompt; one token each, then
    drafts, then a request that joins and one that waits.  Every step against float64 over what the cache then holds."""
    s, hq, hkv, hd = synera(), 8, 2, 128
    rope = s.Rope(hd, 64, layout="half", base=500000.0, scaling=("bands", 8.0, 1.0, 4.0, 8192.0))
    freq = ref.frequencies(64, 500000.0, ("bands", 8.0, 1.0, 4.0, 8192.0))
    gains = draw((hd,), 1) + 1, draw((hd,), 2) + 1
    B, shared, cols = 6, 12, 16
    table = np.concatenate([np.tile(np.arange(shared), (B, 1)), shared + np.arange(B * (cols - shared)).reshape(B, -1)], 1).astype(np.int32)
    n_pages = int(table.max()) + 1
    b = s.SharedBatch(hq, hkv, hd, B, 64, cols)
    kp, vp = bits((n_pages, hkv, P, hd), 0x7FC0), bits((n_pages, hkv, hd, P), 0x7FC0)
    kp[:shared], vp[:shared] = draw((shared, hkv, P, hd), 3), draw((shared, hkv, hd, P), 4)
    ctx = np.full(B, shared * P, np.int32)
    for step, new in enumerate(([1] * B, [4, 1, 9, 2, 1, 0], [1, 0, 30, 3, 5, 2])):
        new = np.array(new, np.int32)
        b.plan(ctx, new, table, n_pages)
        T = int(new.sum())
        x = draw((T, hq + 2 * hkv, hd), 50 + step, torch.float32)
        q, k, v = x[:, :hq], x[:, hq: hq + hkv], x[:, hq + hkv:]
        turned = b.append_rope(rope, q, k, v, kp, vp, q_gain=gains[0], k_gain=gains[1], eps=1e-6)
        o = b.attention(turned, kp, vp)
        pos = np.concatenate([c + np.arange(n) for c, n in zip(ctx, new)]).astype(np.int64)
        req = np.repeat(np.arange(B), new)
        want_q, err = ref.turn(ref.to64(q), pos, freq, "half", 1.0, ref.to64(gains[0]), 1e-6)
        ref.close(ref.to64(turned), want_q, np.abs(want_q) * 2.0 ** -8 + 2 * err, "q")
        want_k, err = ref.turn(ref.to64(k), pos, freq, "half", 1.0, ref.to64(gains[1]), 1e-6)
        got_k = ref.to64(kp)[table[req, pos // P], :, pos % P]
        ref.close(got_k, want_k, np.abs(want_k) * 2.0 ** -8 + 2 * err, "k")
        want, _, eo, _ = ref.attention(ref.to64(turned), ref.to64(kp), ref.to64(vp), ctx, new, table, hd ** -0.5)
        ref.close(ref.to64(o), want, eo, f"o of step {step}")
        ctx = ctx + new


def test_captured_calls_serve_later_plans():
    """A graph of append and attention, captured for one small plan, replayed for others: smaller, larger, cut and uncut, empty."""
    s, hq, hkv, hd = synera(), 8, 2, 64
    rope = s.Rope(hd, layout="half")
    B, cols, room = 12, 140, 96
    b = s.SharedBatch(hq, hkv, hd, B, room, cols)
    n_pages = 1100
    kp, vp = draw((n_pages, hkv, P, hd), 1), draw((n_pages, hkv, hd, P), 2)
    x = draw((room, hq + 2 * hkv, hd), 3)
    q, k, v = x[:, :hq], x[:, hq: hq + hkv], x[:, hq + hkv:]
    out_q, out = torch.zeros((room, hq, hd), dtype=torch.bfloat16, device=DEV), torch.zeros((room, hq, hd), dtype=torch.bfloat16, device=DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        b.plan(np.array([3], np.int32), np.array([1], np.int32), np.zeros((1, 1), np.int32), n_pages)
        with torch.cuda.graph(graph, stream=side):
            b.append_rope(rope, q, k, v, kp, vp, out_q=out_q)
            b.attention(out_q, kp, vp, out=out)
            with pytest.raises(s.SyneraError):                 # a plan cannot be captured
                b.plan(np.array([3], np.int32), np.array([1], np.int32), np.zeros((1, 1), np.int32), n_pages)
        plans = [shared_batch(12, 60, np.arange(12) * 5, 1 + np.arange(12) % 8), shared_batch(1, 0, 0, 96), shared_batch(12, 130, 3, 1),
                 (np.array([5], np.int32), np.zeros(1, np.int32), np.zeros((1, 1), np.int32), 1), shared_batch(2, 1, 1, 1)]
        for round_, (ctx, new, table, _) in enumerate(plans + plans[::-1]):
            x.copy_(draw(x.shape, 100 + round_))
            kp.copy_(draw(kp.shape, 200 + round_))
            vp.copy_(draw(vp.shape, 300 + round_))
            out.fill_(7.0)
            b.plan(ctx, new, table, n_pages)
            graph.replay()
            T = int(new.sum())
            got, got_q = out.clone(), out_q.clone()
            kp2, vp2 = kp.clone(), vp.clone()
            want_q = b.append_rope(rope, q, k, v, kp2, vp2)
            want = b.attention(want_q, kp2, vp2)
            side.synchronize()
            assert torch.equal(kp, kp2) and torch.equal(vp, vp2)
            assert torch.equal(got_q[:T], want_q[:T]) and torch.equal(got[:T], want[:T]), round_
            assert (got[T:] == 7).all()


def test_two_batches_on_two_streams():
    s = synera()
    runs = []
    for i in range(2):
        ctx, new, table, n = shared_batch(20 + i, 30 + i, 9, 2, i)
        k, v = filled_pools(ctx, new, table, n, 2, 64, i)
        q = draw((int(new.sum()), 8, 64), 10 + i)
        b = planned(8, 2, 64, ctx, new, table, n)
        runs.append((b, q, k, v, b.attention(q, k, v), torch.cuda.Stream()))
    torch.cuda.synchronize()
    outs = [[], []]
    for _ in range(5):
        for i, (b, q, k, v, _, st) in enumerate(runs):
            with torch.cuda.stream(st):
                outs[i].append(b.attention(q, k, v))
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(o, runs[i][4]) for o in outs[i])


def test_plans_ahead_of_their_uploads():
    """More plans in a row than there are staging slots: the last one counts, each call sees its own."""
    s = synera()
    b = s.SharedBatch(4, 4, 64, 8, 64, 40)
    k, v, q = draw((400, 4, P, 64), 1), draw((400, 4, 64, P), 2), draw((64, 4, 64), 3)
    plans = [shared_batch(1 + i % 8, 3 + i, 2 * i, 1 + i % 7, i) for i in range(11)]
    got = []
    for ctx, new, table, _ in plans:
        b.plan(ctx, new, table, 400)
        got.append(b.attention(q, k, v)[: int(new.sum())].clone())
    for (ctx, new, table, _), o in zip(plans, got):
        want, _, eo, _ = ref.attention(ref.to64(q)[: int(new.sum())], ref.to64(k), ref.to64(v), ctx, new, table, 0.125)
        ref.close(ref.to64(o), want, eo, "o")


def test_refusals():
    s, hq, hkv, hd = synera(), 4, 2, 64
    ctx, new, table, n = shared_batch(3, 2, 4, 2)
    T = int(new.sum())
    kp, vp = draw((n, hkv, P, hd), 1), draw((n, hkv, hd, P), 2)
    x = draw((T, hq + 2 * hkv, hd), 3)
    q, k, v = x[:, :hq], x[:, hq: hq + hkv], x[:, hq + hkv:]
    rope = s.Rope(hd)
    b = s.SharedBatch(hq, hkv, hd, 3, T, table.shape[1])

    def status(call):
        with pytest.raises(s.SyneraError) as e:
            call()
        return e.value.status
    assert status(lambda: b.attention(q, kp, vp)) == s.EINVAL                       # no plan yet
    assert status(lambda: b.append_rope(rope, q, k, v, kp, vp)) == s.EINVAL
    b.plan(ctx, new, table, n)
    good = b.append_rope(rope, q, k, v, kp, vp)
    o = b.attention(good, kp, vp)
    wide = np.concatenate([table, table[:, :1] * 0 - 1], 1)
    assert status(lambda: b.plan(ctx, new, wide, n)) == s.ENOSPC                    # more columns than the batch has room for
    assert status(lambda: b.plan(ctx, new + 1, table, n)) == s.ENOSPC
    assert status(lambda: b.plan(ctx, new, table, 3)) == s.ERANGE
    assert torch.equal(b.attention(good, kp, vp), o)                                # a refused plan leaves the one before
    for bad in (dict(q=q[:, :2]), dict(k=k[: T - 1]), dict(k=k.float()), dict(q=q.double(), k=k.double(), v=v.double()), dict(k_pool=kp[:-1]),
                dict(k_pool=vp), dict(v_pool=vp.float()), dict(k_pool=kp.transpose(0, 1)), dict(v=v.cpu()), dict(out_q=q.float()),
                dict(k_gain=torch.ones(32, dtype=torch.bfloat16, device=DEV))):
        with pytest.raises(ValueError):
            b.append_rope(**{**dict(rope=rope, q=q, k=k, v=v, k_pool=kp, v_pool=vp), **bad})
    for bad in (dict(q=q.float()), dict(q=q[:1]), dict(scale=0.0), dict(scale=-1.0), dict(out=q.float()), dict(k_pool=kp[:, :1])):
        with pytest.raises(ValueError):
            b.attention(**{**dict(q=good, k_pool=kp, v_pool=vp), **bad})
    assert status(lambda: b.append_rope(s.Rope(128), q, k, v, kp, vp)) == s.EINVAL  # another head width
    assert status(lambda: b.append_rope(rope, q, k, v, kp, vp, eps=-1.0)) == s.EINVAL
    assert status(lambda: b.append_rope(rope, q, k, v, kp, vp, out_q=x[:, 2:6])) == s.EINVAL      # out on the keys
    assert status(lambda: b.append_rope(rope, q, kp.view(-1, 2, 64)[:T], v, kp, vp)) == s.EINVAL  # keys inside the pool
    both = draw((2 * n, hkv, P * hd), 1)
    assert status(lambda: b.append_rope(rope, q, k, v, both[:n].view(n, hkv, P, hd), both[1: n + 1].view(n, hkv, hd, P))) == s.EINVAL
    assert status(lambda: b.attention(good, kp, vp, out=good)) == s.EINVAL          # not in place
    assert status(lambda: b.attention(good, kp, vp, scale=float("inf"))) == s.EINVAL
    odd = torch.empty(T * hq * hd + 8, dtype=torch.bfloat16, device=DEV)
    assert status(lambda: b.attention(odd[1: 1 + T * hq * hd].view(T, hq, hd), kp, vp)) == s.EINVAL
    assert status(lambda: b.attention(good, kp, vp, out=odd[2: 2 + T * hq * hd].view(T, hq, hd))) == s.EINVAL
    pool_as_out = kp.view(-1)[: T * hq * hd].view(T, hq, hd)
    assert status(lambda: b.attention(good, kp, vp, out=pool_as_out)) == s.EINVAL   # out on the keys
    assert status(lambda: b.append_rope(rope, q, k, v, kp, vp, out_q=pool_as_out)) == s.EINVAL
    pool_as_out = kp.view(-1)[: T * hq * hd].view(T, hq, hd)
    assert status(lambda: b.attention(good, kp, vp, out=pool_as_out)) == s.EINVAL   # out on the keys
    assert status(lambda: b.append_rope(rope, q, k, v, kp, vp, out_q=pool_as_out)) == s.EINVAL
    assert torch.equal(b.attention(good, kp, vp), o)


def test_a_scale_that_32_bits_round_to_zero_is_refused():
    s = synera()
    b = s.SharedBatch(2, 1, 64, 1, 1, 1)
    b.plan([4], [1], [[0]], 1)
    kp, vp, q = draw((1, 1, P, 64), 1), draw((1, 1, 64, P), 2), draw((1, 2, 64), 3)
    with pytest.raises(ValueError):
        b.attention(q, kp, vp, scale=1e-60)                                          # (0 would mean 1 / sqrt(head_dim))
    # the smallest scale weighs all keys alike
    o = b.attention(q, kp, vp, scale=2.0 ** -126)
    want = vp[0, 0, :, :5].double().mean(1)
    assert torch.allclose(o[0].double(), want.expand(2, 64), rtol=2.0 ** -7, atol=2.0 ** -7)


@pytest.mark.parametrize("hq,hkv,hd,ctx,new", [(1024, 1, 64, 200, 3), (300, 2, 128, 90, 5), (2, 2, 128, 131077, 1), (1, 1, 64, 70001, 3)])
def test_attention_wide_groups_and_long_contexts(hq, hkv, hd, ctx, new):
    """Tokens whose heads fill several tiles of rows or straddle two; single contexts that all units share."""
    n = -(-(ctx + new) // P)
    table = np.random.RandomState(ctx).permutation(n).astype(np.int32)[None]
    check_attention(hq, hkv, hd, np.array([ctx], np.int32), np.array([new], np.int32), table, n, ctx + new)


def test_pages_whose_offsets_pass_32_bits():
    """The last pages of pools of over 2^32 bytes: what is appended and attended there is what it is in a small pool, bit for bit."""
    s, hq, hkv, hd = synera(), 16, 8, 128
    ctx, new, table, n = shared_batch(5, 20, np.array([0, 3, 16, 90, 200]), np.array([1, 2, 17, 40, 1]))
    many = (1 << 32) // (hkv * P * hd * 2) + n
    T = int(new.sum())
    x = draw((T, hq + 2 * hkv, hd), 1)
    q, k, v = x[:, :hq], x[:, hq: hq + hkv], x[:, hq + hkv:]
    rope = s.Rope(hd)
    small = [draw((n, hkv, P, hd), 2), draw((n, hkv, hd, P), 3)]
    large = [torch.empty((many, *p.shape[1:]), dtype=p.dtype, device=DEV) for p in small]
    for p, whole in zip(small, large):
        whole[many - n:] = p
    got = []
    for pools, at, pages in ((small, 0, n), (large, many - n, many)):
        b = s.SharedBatch(hq, hkv, hd, len(ctx), T, table.shape[1])
        b.plan(ctx, new, np.where(table >= 0, table + at, -1), pages)
        turned = b.append_rope(rope, q, k, v, *pools)
        got.append((turned, b.attention(turned, *pools), pools[0][at:], pools[1][at:]))
    for a, c in zip(*got):
        assert torch.equal(a, c)


@pytest.mark.parametrize("T", [8001, 29003])
def test_appends_that_no_cache_holds(T):
    """Large appends, whose inputs or outputs pass the caches by: the bits of Rope.apply in small calls, and the values as they are."""
    s, hq, hkv, hd = synera(), 32, 8, 128
    ctx, new = np.array([5, 0, 64], np.int32), np.array([T // 2, 1, T - T // 2 - 1], np.int32)
    need = -(-(ctx + new) // P)
    n = int(need.sum())
    perm = np.random.RandomState(T).permutation(n).astype(np.int32)
    table = np.full((3, int(need.max())), -1, np.int32)
    for i in range(3):
        table[i, : need[i]] = perm[need[:i].sum(): need[: i + 1].sum()]
    x = draw((T, hq + 2 * hkv, hd), 1)
    q, k, v = x[:, :hq], x[:, hq: hq + hkv], x[:, hq + hkv:]
    rope = s.Rope(hd, layout="half")
    kp, vp = bits((n, hkv, P, hd), 0x1234), bits((n, hkv, hd, P), 0x4321)
    turned = planned(hq, hkv, hd, ctx, new, table, n).append_rope(rope, q, k, v, kp, vp)
    at = np.concatenate([c + np.arange(m) for c, m in zip(ctx, new)])
    req = np.repeat(np.arange(3), new)
    page, slot = torch.from_numpy(table[req, at // P].astype(np.int64)).to(DEV), torch.from_numpy(at % P).to(DEV)
    pos = torch.from_numpy(at.astype(np.int32)).to(DEV)
    for t in range(0, T, 1500):
        e = min(T, t + 1500)
        wq, wk = rope.apply(pos[t: e], q[t: e], k[t: e])
        assert torch.equal(turned[t: e], wq) and torch.equal(kp[page[t: e], :, slot[t: e]], wk), t
        assert torch.equal(vp[page[t: e], :, :, slot[t: e]], v[t: e]), t
    kp[page, :, slot] = bits((), 0x1234)
    vp[page, :, :, slot] = bits((), 0x4321)
    assert (kp.view(torch.int16) == 0x1234).all() and (vp.view(torch.int16) == 0x4321).all()


def captured(call):
    """A graph of the call, captured on a stream of its own; it never runs."""
    graph, side = torch.cuda.CUDAGraph(keep_graph=True), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    gc.collect()                                               # graphs that other tests left behind wait for the device when they go,
    gc.disable()                                               # which ends a capture
    try:
        with torch.cuda.graph(graph, stream=side):
            call()
    finally:
        gc.enable()
    return graph


def test_captured_calls_are_checked_for_later_plans():
    """Behind a plan of one token, tensors whose later rows lie on one another: an eager call touches none of those, a captured one would for
    a later plan, and is refused."""
    s, hq, hkv, hd, rows = synera(), 4, 2, 64, 32
    rope = s.Rope(hd)
    b = s.SharedBatch(hq, hkv, hd, 4, rows, 4)
    b.plan([3], [1], [[0]], 16)
    kp, vp = draw((16, hkv, P, hd), 1), draw((16, hkv, hd, P), 2)
    width = hq * hd
    flat = draw((2 * (rows + 2) * width,), 3)
    q, k, v = flat[: rows * width].view(rows, hq, hd), draw((rows, hkv, hd), 4), draw((rows, hkv, hd), 5)
    stretched = flat.as_strided((rows, hq, hd), (2 * width, hd, 1))                  # q's first row, other later ones
    behind = flat[8 * width: (rows + 8) * width].view(rows, hq, hd)                  # q's rows 8 ..
    same = draw((1, hq, hd), 6).expand(rows, hq, hd)                                 # one row for all
    inside = flat[rows * width:].as_strided((rows, hq, hd), (hd, 8 * hd, 1))         # heads apart for eight tokens
    free = flat[rows * width: 2 * rows * width].view(rows, hq, hd)

    def refused(call):
        with pytest.raises(s.SyneraError) as e:
            call()
        assert e.value.status == s.EINVAL

    def all_captured():
        for out in (stretched, behind, same, inside):
            refused(lambda: b.append_rope(rope, q, k, v, kp, vp, out_q=out))
        for out in (behind, same, inside):
            refused(lambda: b.attention(q, kp, vp, out=out))
        refused(lambda: b.append_rope(rope, q, behind[:, :2], v, kp, vp, out_q=q))   # queries in place, keys in their later rows
        b.append_rope(rope, q, k, v, kp, vp, out_q=free)
        b.append_rope(rope, q, k, v, kp, vp, out_q=q)                                # in place
        b.append_rope(rope, q[:8], k[:8], v[:8], kp, vp, out_q=behind[:8])           # room for eight tokens
        by_head = free.view(hq, rows, hd).transpose(0, 1)
        b.append_rope(rope, q, k, v, kp, vp, out_q=by_head)
        b.attention(q, kp, vp, out=by_head)
        one = free.view(-1)[: hq * hd].view(hq, 1, hd).transpose(0, 1)               # one row, heads outermost
        b.append_rope(rope, q[:1], k[:1], v[:1], kp, vp, out_q=one)
        b.attention(q[:1], kp, vp, out=one)
    captured(all_captured)
    for out in (stretched, behind, same, inside):                                    # the first rows are apart
        b.append_rope(rope, q, k, v, kp, vp, out_q=out)
    b.attention(q, kp, vp, out=behind)
    # without row counts, captured calls are checked for two tokens at least
    from paper_2511_07423_amd import binding as raw
    heads = [raw._pack_heads(t.data_ptr(), o.data_ptr(), 0, t.shape[1], t.stride(0), t.stride(1), o.stride(0), o.stride(1))
             for t, o in ((q, stretched), (k, k), (v, v), (q, free))]

    def append(at):
        stream = torch.cuda.current_stream().cuda_stream
        return raw._lib.synera_append_rope(b._h, rope._h, 1, heads[at], heads[1], heads[2], 0.0, kp.data_ptr(), vp.data_ptr(), stream)
    got = []
    captured(lambda: got.extend((append(0), append(3))))
    assert got == [s.EINVAL, s.OK] and append(0) == s.OK
    short = raw._pack_heads_rows(k.data_ptr(), 0, 0, hkv, 1, hkv * hd, hd, 0, 0)
    b.plan([3], [2], [[0]], 16)
    assert raw._lib.synera_append_rope(b._h, rope._h, 1, None, short, heads[2], 0.0, kp.data_ptr(), vp.data_ptr(), None) == s.EINVAL
    torch.cuda.synchronize()


def blocks_of_kernels(graph):
    """Grids of the kernels in a captured graph, from the runtime itself."""
    class Params(C.Structure):                                 # hipKernelNodeParams
        _fields_ = [("block", C.c_uint * 3), ("extra", C.c_void_p), ("func", C.c_void_p), ("grid", C.c_uint * 3), ("args", C.c_void_p), ("lds", C.c_uint)]
    path = next(line.split()[-1] for line in open("/proc/self/maps") if "libamdhip64" in line)
    hip = C.CDLL(path)
    at, n = C.c_void_p(graph.raw_cuda_graph()), C.c_size_t(0)
    assert hip.hipGraphGetNodes(at, None, C.byref(n)) == 0
    nodes = (C.c_void_p * n.value)()
    assert hip.hipGraphGetNodes(at, nodes, C.byref(n)) == 0
    grids = []
    for node in nodes:
        kind = C.c_int(-1)
        assert hip.hipGraphNodeGetType(C.c_void_p(node), C.byref(kind)) == 0
        if kind.value == 0:                                    # hipGraphNodeTypeKernel
            params = Params()
            assert hip.hipGraphKernelNodeGetParams(C.c_void_p(node), C.byref(params)) == 0
            grids.append(tuple(params.grid))
    return grids


@pytest.mark.parametrize("dtype,hd", [("bf16", 128), ("f32", 64)])
def test_captured_appends_are_launched_for_the_room_they_have(dtype, hd):
    """Behind a plan of one token: a captured append fills the chip if its tensors have the rows for it, and no more blocks than their rows can
    use if not."""
    s, hq, hkv, rows = synera(), 32, 8, 4096
    rope = s.Rope(hd)
    b = s.SharedBatch(hq, hkv, hd, 64, rows, 300)
    b.plan([3], [1], [[0]], 16)
    kp, vp = draw((16, hkv, P, hd), 1), draw((16, hkv, hd, P), 2)
    x = draw((rows, hq + 2 * hkv, hd), 3, TYPES[dtype])
    out = torch.empty((rows, hq, hd), dtype=torch.bfloat16, device=DEV)
    places = 2 * torch.cuda.get_device_properties(0).multi_processor_count

    def grid(n):
        part = x[:n]
        (blocks, _, _), = blocks_of_kernels(captured(lambda: b.append_rope(rope, part[:, :hq], part[:, hq: hq + hkv], part[:, hq + hkv:], kp, vp,
                                                                           out_q=out[:n])))
        return blocks
    slabs = hkv * hd // 128                                    # pieces of a token's values, one a wavefront
    assert grid(rows) >= 2 * places
    assert grid(1) <= slabs + hq + hkv
    assert grid(8) <= 8 * (slabs + hq + hkv)


def test_a_captured_append_serves_batches_of_any_size():
    """Captured behind one token, replayed for steps, drafts and prompts in every element type: the eager call's bits."""
    s, hq, hkv, hd, rows = synera(), 32, 8, 128, 6000
    rope = s.Rope(hd, 64, layout="half")
    b = s.SharedBatch(hq, hkv, hd, 64, rows, 400)
    n_pages = 1000
    pools = draw((n_pages, hkv, P, hd), 1), draw((n_pages, hkv, hd, P), 2)
    gains = draw((hd,), 3) + 1, draw((hd,), 4) + 1
    plans = [(np.zeros(64, np.int32), np.ones(64, np.int32)), (np.arange(64) * 3, 1 + np.arange(64) % 16), (np.array([5]), np.array([6000])),
             (np.array([0, 7, 31]), np.array([900, 1, 2000])), (np.array([3]), np.array([1]))]
    for dtype in TYPES:
        x = draw((rows, hq + 2 * hkv, hd), 5, TYPES[dtype])
        q, k, v = x[:, :hq], x[:, hq: hq + hkv], x[:, hq + hkv:]
        out = torch.zeros((rows, hq, hd), dtype=torch.bfloat16, device=DEV)
        b.plan([3], [1], [[0]], n_pages)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            b.append_rope(rope, q, k, v, *pools, q_gain=gains[0], k_gain=gains[1], out_q=out)
        for ctx, new in plans + plans[::-1]:
            need = -(-(ctx + new) // P)
            table = np.full((len(ctx), int(need.max())), -1, np.int32)
            perm = np.random.RandomState(len(ctx)).permutation(n_pages)
            for i in range(len(ctx)):
                table[i, : need[i]] = perm[need[:i].sum(): need[: i + 1].sum()]
            b.plan(ctx, new, table, n_pages)
            T = int(new.sum())
            wanted = [p.clone() for p in pools]
            want = b.append_rope(rope, q, k, v, *wanted, q_gain=gains[0], k_gain=gains[1])
            out.fill_(7.0)
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out[:T], want[:T]) and (out[T:] == 7).all(), (dtype, T)
            assert all(torch.equal(a, c) for a, c in zip(pools, wanted)), (dtype, T)


def test_captured_appends_that_no_cache_holds():
    """A captured append whose plans pass the caches by or do not, with tensors that have room for both: the eager call's bits."""
    s, hq, hkv, hd, rows = synera(), 32, 8, 128, 17500
    rope, b = s.Rope(hd, layout="half"), s.SharedBatch(hq, hkv, hd, 1, rows, 1100)
    n_pages = 1100
    table = np.random.RandomState(1).permutation(n_pages).astype(np.int32)[None]
    pools = [torch.zeros((n_pages, hkv, P, hd), dtype=torch.bfloat16, device=DEV), torch.zeros((n_pages, hkv, hd, P), dtype=torch.bfloat16, device=DEV)]
    x = draw((rows, hq + 2 * hkv, hd), 1, torch.float32)                             # 537 MB moved for all rows, 31 KB for one
    q, k, v = x[:, :hq], x[:, hq: hq + hkv], x[:, hq + hkv:]
    out = torch.zeros((rows, hq, hd), dtype=torch.bfloat16, device=DEV)
    b.plan([3], [1], table[:, :1], n_pages)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.append_rope(rope, q, k, v, *pools, out_q=out)
    for T in (rows - 3, 1, 5001):                                                    # marked, kept, inputs marked
        b.plan([7], [T], table, n_pages)
        wanted = [p.clone() for p in pools]
        want = b.append_rope(rope, q, k, v, *wanted)
        out.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out[:T], want[:T]) and (out[T:] == 7).all(), T
        assert all(torch.equal(a, c) for a, c in zip(pools, wanted)), T


def test_a_scale_that_is_not_finite_in_the_exponent_is_refused():
    """The scale meets log2 e in 32 bits: beyond 2.35e38 there is no such number, and no weight could be formed."""
    s = synera()
    b = s.SharedBatch(2, 1, 64, 1, 1, 1)
    b.plan([4], [1], [[0]], 1)
    kp, vp, q = draw((1, 1, P, 64), 1), draw((1, 1, 64, P), 2), draw((1, 2, 64), 3)
    for scale in (3e38, 2.4e38):
        with pytest.raises(s.SyneraError) as e:
            b.attention(q, kp, vp, scale=scale)
        assert e.value.status == s.EINVAL
    tiny = (q.float() * 2.0 ** -60).to(torch.bfloat16)         # the largest scales weigh the largest score alone
    o = b.attention(tiny, kp, vp, scale=2.0 ** 80)
    best = (tiny[0].double() @ kp[0, 0, :5].double().T).argmax(1)
    # One key has all the weight, p = 2^(s c - m c) with m c rounded to 32 bits: near 2^23 that is up to half a unit off, so p is not 1.  It meets
    # the value as bf16 (2^-8) and is divided by itself unrounded; the output is bf16 (2^-8): (1 + 2^-8)^2 - 1 < 2^-7 + 2^-15, and 32-bit steps.
    want = vp[0, 0].T[best].double()
    assert ((o[0].double() - want).abs() <= want.abs() * (2.0 ** -7 + 2.0 ** -14)).all()


def test_attention_refuses_outputs_on_the_values():
    s, hq, hkv, hd = synera(), 4, 2, 64
    b = s.SharedBatch(hq, hkv, hd, 1, 2, 1)
    b.plan([4], [2], [[0]], 2)
    kp, vp, q, k = draw((2, hkv, P, hd), 1), draw((2, hkv, hd, P), 2), draw((2, hq, hd), 3), draw((2, hkv, hd), 4)
    on_values = vp.view(-1)[: q.numel()].view(q.shape)
    for call in (lambda: b.attention(q, kp, vp, out=on_values), lambda: b.append_rope(s.Rope(hd), q, k, k, kp, vp, out_q=on_values),
                 lambda: b.append_rope(s.Rope(hd), None, k, vp.view(-1, hkv, hd)[:2], kp, vp)):
        with pytest.raises(s.SyneraError) as e:
            call()
        assert e.value.status == s.EINVAL


def test_appends_refuse_outputs_on_gains():
    """Gains are read while queries and pages are written."""
    s, hq, hkv, hd = synera(), 4, 2, 64
    b, rope = s.SharedBatch(hq, hkv, hd, 1, 2, 1), s.Rope(hd)
    b.plan([4], [2], [[0]], 2)
    kp, vp, q, k = draw((2, hkv, P, hd), 1), draw((2, hkv, hd, P), 2), draw((2, hq, hd), 3), draw((2, hkv, hd), 4)
    out, gain = torch.zeros_like(q), torch.ones(hd, dtype=torch.bfloat16, device=DEV)
    for q_gain, k_gain in ((out.view(-1)[64: 128], gain), (gain, out.view(-1)[-64:]), (kp.view(-1)[:64], gain), (gain, vp.view(-1)[-64:]), (None, kp.view(-1)[64: 128])):
        with pytest.raises(s.SyneraError) as e:
            b.append_rope(rope, q, k, k, kp, vp, q_gain=q_gain, k_gain=k_gain, out_q=out)
        assert e.value.status == s.EINVAL
    b.append_rope(rope, q, k, k, kp, vp, q_gain=gain, k_gain=gain, out_q=out)
    torch.cuda.synchronize()


def small_verifier():
    from helpers import drawn_model, small_shape
    shape = small_shape(d_model=256, n_q_heads=4, n_kv_heads=4, head_dim=64, d_ffn=128, vocab=128, n_layers=1)
    head, layers = drawn_model(shape, 1, DEV)
    return synera().Verifier(shape, head, layers, 4, 200, 8)


def test_handles_that_go_while_a_graph_is_captured():
    """A collector may end the life of handles at any time, also while some stream is captured: the capture stands, and what was captured runs."""
    s, hq, hkv, hd = synera(), 4, 2, 64
    b, rope = s.SharedBatch(hq, hkv, hd, 1, 2, 1), s.Rope(hd)
    b.plan([4], [2], [[0]], 1)
    kp, vp, x = draw((1, hkv, P, hd), 1), draw((1, hkv, hd, P), 2), draw((2, hq + 2 * hkv, hd), 3)
    q, k, v = x[:, :hq], x[:, hq: hq + hkv], x[:, hq + hkv:]
    others = [s.Rope(hd), s.SharedBatch(hq, hkv, hd, 1, 2, 1), s.SharedBatch(hq, hkv, hd, 1, 2, 1), small_verifier()]
    others[2].plan([4], [2], [[0]], 1)
    out_q, out = torch.zeros((2, hq, hd), dtype=torch.bfloat16, device=DEV), torch.zeros((2, hq, hd), dtype=torch.bfloat16, device=DEV)
    pools = kp.clone(), vp.clone()
    want_q = b.append_rope(rope, q, k, v, *pools)
    want = b.attention(want_q, *pools)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.append_rope(rope, q, k, v, kp, vp, out_q=out_q)
        for h in others:
            h.close()
        b.attention(out_q, kp, vp, out=out)
    for _ in range(3):
        out.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out_q, want_q) and torch.equal(out, want)


def test_destroys_wait_for_the_device():
    """Handles go behind the work that may still read them, on whatever stream it runs."""
    s = synera()
    for handle in (s.Rope(64), s.SharedBatch(4, 2, 64, 1, 2, 1), small_verifier()):
        torch.cuda.synchronize()
        side, done = torch.cuda.Stream(), torch.cuda.Event()
        with torch.cuda.stream(side):
            torch.cuda._sleep(20_000_000)                      # some milliseconds
            done.record()
        assert not done.query()
        handle.close()
        assert done.query()
