"""Whole steps over trees of drafted tokens where something gives out on the way: pools that run dry, counts out of range, replayed plans of other
sizes; and the shapes of trees and paths that the tests of the single operators leave out."""
import gc
import random

import numpy as np
import pytest
import torch

import shared_reference as ref
import tree_reference as tree
from test_gpu_tree import DEV, P, Server, grow, i32, same, synera

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
