"""Host logic of batches that share pages (no GPU): validation codes, and that a plan covers every (row, KV head, key it sees) exactly
once, with pages of the request itself, inside the capacities, and with partial results that the join finds again."""
import random

import numpy as np
import pytest

import paper_2511_07423_amd as synera

P, TILE = 16, 128


def make_batch(rng, B, max_depth=3, max_new=20, max_own=80, zero=0.1, shuffle=True):
    """A random tree of shared prefixes: each request starts from another one's whole cached pages, or from nothing."""
    ctx, new, rows, n_pages = [], [], [], 0
    for i in range(B):
        row = []
        if i and rng.random() < 0.8:
            j = rng.randrange(i)
            row = rows[j][: rng.randint(0, ctx[j] // P)]
        own = rng.randint(0, max_own)
        c = len(row) * P + own
        n = 0 if rng.random() < zero else rng.randint(1, max_new)
        need = -(-(c + n) // P)
        row = row + list(range(n_pages, n_pages + need - len(row)))
        n_pages = max([n_pages] + [r + 1 for r in row])
        ctx.append(c), new.append(n), rows.append(row)
    order = list(range(B))
    if shuffle:
        rng.shuffle(order)
    perm = list(range(max(n_pages, 1)))
    rng.shuffle(perm)
    cols = max(1, max(len(r) for r in rows)) + rng.randint(0, 2)
    table = np.full((B, cols), -7, np.int32)                   # entries beyond a row's pages are never looked at
    for at, i in enumerate(order):
        table[at, : len(rows[i])] = [perm[p] for p in rows[i]]
    return np.array([ctx[i] for i in order], np.int32), np.array([new[i] for i in order], np.int32), table, len(perm)


def check_plan(hq, hkv, slots, ctx, new, table, max_tokens=None):
    pl = synera.debug_shared_plan(hq, hkv, slots, ctx, new, table, max_tokens)
    G, B, T = hq // hkv, len(ctx), int(new.sum())
    head = pl["head"][0]
    assert head[0] == T and head[1] == len(pl["windows"]) and head[2] == len(pl["joined"])
    assert len(pl["items"]) == 8 * head[3] + 32 * head[4]
    for name, room in zip(("items", "list", "parts", "pages", "windows"), pl["limits"]):
        assert len(pl[name]) <= room, name
    tok0 = np.concatenate([[0], np.cumsum(new)])
    req_of = np.repeat(np.arange(B), new)
    pos = ctx[req_of] + np.arange(T) - tok0[req_of] if T else np.zeros(0, int)
    assert np.array_equal(pl["pos"], pos)
    assert np.array_equal(pl["slot"], [table[r, p // P] * P + p % P for r, p in zip(req_of, pos)])
    covered = []
    for page, row, s0, s1 in pl["windows"]:
        assert 0 <= s0 < s1 <= P
        for s in range(s0, s1):
            assert pl["slot"][row + s - s0] == page * P + s
            covered.append(row + s - s0)
    assert sorted(covered) == list(range(T))

    seen = {}                    # (token, head, kv head) -> list of (first page column, key from, key to, partial row)
    parts = np.zeros(max(1, pl["limits"][5]), np.int32)
    for at_item, item in enumerate(pl["items"]):
        flags, kh, n_rows, row0, tok, page, n_pages, k0, k1, lim0, part = item[:11]
        if n_rows == 0:
            continue
        assert n_rows <= (TILE if at_item < 8 * head[3] else 32)
        assert list(item[16:]) == [pl["pages"][page + min(k0 // P + q, n_pages - 1)] for q in range(16)]
        assert 1 <= n_rows <= TILE and row0 % TILE == 0 and k0 % 128 == 0 and 0 <= k0 < k1 <= n_pages * P and 0 <= kh < hkv
        ids = pl["pages"][page: page + n_pages]
        assert len(ids) == n_pages
        if part >= 0:
            assert part + n_rows <= pl["limits"][5]
            parts[part: part + n_rows] += 1
        for r in range(n_rows):
            j, g = divmod(row0 + r, G)
            t = tok + j if flags & 1 else pl["list"][tok + j]
            i = req_of[t]
            own = list(table[i, : -(-(ctx[i] + new[i]) // P)])
            col = own.index(ids[0])                            # the node's pages are a run of the request's own
            assert own[col: col + n_pages] == list(ids)
            end = k1
            if flags & 1:
                assert t - tok0[i] == j and lim0 == ctx[i] - col * P
                end = min(end, lim0 + j + 1)                   # what the kernel's mask leaves
            seen.setdefault((t, g, kh), []).append((col * P + k0, col * P + end, part + r if part >= 0 else -1))
    assert parts.max(initial=0) <= 1                           # no partial row is written twice
    joined = {int(t): (int(first), int(n)) for t, first, n, _ in pl["joined"]}
    assert len(joined) == len(pl["joined"])
    for t in range(T):
        i = req_of[t]
        for kh in range(hkv):
            for g in range(G):
                # a tile's other rows may see keys that this one does not: such ranges hold nothing for it
                ranges = sorted(r for r in seen[(t, g, kh)] if r[1] > r[0])
                at = 0
                for a, b, _ in ranges:
                    assert a == at
                    at = b
                assert at == pos[t] + 1
                if t not in joined:
                    assert len(seen[(t, g, kh)]) == 1 and ranges[0][2] == -1
                    continue
                first, n = joined[t]
                mine = {row + kh * step + g for row, step in pl["parts"][first: first + n]}
                assert len(mine) == n and {p for _, _, p in ranges} <= mine <= {p for _, _, p in seen[(t, g, kh)]}
    return pl


@pytest.mark.parametrize("seed", range(24))
def test_plan_covers_every_key_once(seed):
    rng = random.Random(seed)
    B = rng.choice((1, 2, 3, 9, 24))
    hkv = rng.choice((1, 2, 3))
    hq = hkv * rng.choice((1, 3, 4, 12))
    ctx, new, table, n_pages = make_batch(rng, B, max_new=rng.choice((1, 5, 40)), max_own=rng.choice((0, 40, 900)))
    assert synera.validate_shared(ctx, new, table, n_pages, B, int(new.sum())) == synera.OK
    check_plan(hq, hkv, rng.choice((1, 16, 512)), ctx, new, table)
    check_plan(hq, hkv, 4, ctx, new, table, max_tokens=int(new.sum()) + 100)


def test_plan_shares_where_it_is_shorter():
    # 64 requests of one token behind 2048 common ones: the common pages are read once
    B, shared = 64, 128
    ctx = np.full(B, shared * P + 5, np.int32)
    table = np.concatenate([np.tile(np.arange(shared), (B, 1)), shared + np.arange(B)[:, None]], 1).astype(np.int32)
    pl = check_plan(32, 8, 512, ctx, np.ones(B, np.int32), table)
    shared_items = pl["items"][((pl["items"][:, 0] & 1) == 0) & (pl["items"][:, 2] > 0)]
    assert len(pl["pages"]) == shared + B and len(pl["list"]) == B
    assert {int(r) for r in shared_items[:, 2]} == {128}       # 64 x 4 rows are two full tiles
    # two levels: behind 9600 common tokens, halves of the batch share more
    shared = 600
    table = np.concatenate([np.tile(np.arange(shared), (B, 1)), 3000 + np.arange(B)[:, None]], 1).astype(np.int32)
    ctx2 = np.full(B, (shared + 64) * P + 5, np.int32)
    more = np.concatenate([np.tile(1000 + np.arange(64), (B // 2, 1)), np.tile(2000 + np.arange(64), (B // 2, 1))])
    table2 = np.concatenate([table[:, :shared], more, table[:, shared:]], 1).astype(np.int32)
    pl = check_plan(32, 8, 512, ctx2, np.ones(B, np.int32), table2)
    assert len(pl["pages"]) == shared + 2 * 64 + B


def test_plan_of_long_chunks_reads_for_itself():
    # prompts of 512 tokens fill their tiles alone: nothing is gained by one pass for both
    ctx, new = np.array([160, 160], np.int32), np.array([512, 512], np.int32)
    table = np.concatenate([np.tile(np.arange(10), (2, 1)), 10 + np.arange(64).reshape(2, 32)], 1).astype(np.int32)
    pl = check_plan(8, 1, 512, ctx, new, table)
    assert (pl["items"][pl["items"][:, 2] > 0, 0] & 1).all()


@pytest.mark.parametrize("block_groups,wave_groups", [(0, 0), (1, 0), (0, 3), (5, 2), (2, 5), (70, 33), (200, 31), (64, 64), (3, 400)])
@pytest.mark.parametrize("run", [1, 2, 32])
def test_blocks_take_every_item_once(block_groups, wave_groups, run):
    """The order in which blocks take the two lists (as the kernel's sh_block has it)."""
    taken, whole_before = [], 0
    for b in range(8 * (block_groups + wave_groups)):
        at, whole = synera.debug_shared_block(block_groups, wave_groups, run, b)
        assert whole == (at < 8 * block_groups)
        assert at % 8 == b % 8 or not whole                    # the XCD that the item was queued for
        taken += [at] if whole else range(at, at + 4)
    assert sorted(taken) == list(range(8 * block_groups + 32 * wave_groups))


def test_plan_without_rows():
    ctx, new, table, n = np.array([20, 0], np.int32), np.zeros(2, np.int32), np.array([[0, 1], [5, 5]], np.int32), 2
    assert synera.validate_shared(ctx, new, table, n, 2, 1) == synera.OK
    pl = check_plan(4, 4, 64, ctx, new, table, max_tokens=1)
    assert not pl["head"].any()


def test_validation_codes():
    ok = dict(ctx_len=[40, 37, 0], n_new=[3, 1, 16], block_table=np.array([[0, 1, 2, 9], [0, 1, 3, -5], [4, -1, -1, 99]], np.int32),
              n_pages_in_pool=10, max_batch=3, max_tokens=20)
    s = synera
    v = s.validate_shared
    assert v(**ok) == s.OK

    def table(**at):
        t = ok["block_table"].copy()
        for k, x in at.items():
            t[int(k[1]), int(k[2])] = x
        return t
    assert v(**dict(ok, n_new=[3, -1, 16])) == s.EINVAL
    assert v(**dict(ok, n_new=[3, 0, 16])) == s.OK
    assert v(**dict(ok, ctx_len=[40, -1, 0])) == s.ERANGE
    assert v(**dict(ok, ctx_len=[40, 2 ** 31 - 100, 0])) == s.ERANGE                 # positions are int32
    assert v(**dict(ok, max_batch=2)) == s.ENOSPC
    assert v(**dict(ok, max_tokens=19)) == s.ENOSPC
    assert v(**dict(ok, ctx_len=[62, 37, 0])) == s.ENOSPC                            # 65 positions, four columns
    assert v(**dict(ok, n_pages_in_pool=1 << 27)) == s.EUNSUP
    assert v(**dict(ok, n_pages_in_pool=0)) == s.EINVAL
    assert v(**dict(ok, block_table=table(_02=10))) == s.ERANGE                      # outside the pool
    assert v(**dict(ok, block_table=table(_11=-1))) == s.ERANGE
    assert v(**dict(ok, block_table=table(_12=2))) == s.ERANGE                       # both append to page 2
    assert v(**dict(ok, block_table=table(_20=0))) == s.ERANGE                       # request 2 appends to a cached page
    assert v(**dict(ok, block_table=table(_10=1, _11=0))) == s.ERANGE                # the same pages, another order
    assert v(**dict(ok, block_table=table(_10=5))) == s.ERANGE                       # page 1 behind another page
    assert v(**dict(ok, block_table=table(_01=0))) == s.ERANGE                       # twice in one row
    assert v(**dict(ok, ctx_len=[40, 30, 0])) == s.ERANGE                            # request 1 appends inside page 1
    one = dict(ctx_len=[32], n_new=[1], block_table=np.array([[0, 1, 0]], np.int32), n_pages_in_pool=4, max_batch=1, max_tokens=1)
    assert v(**one) == s.ERANGE
