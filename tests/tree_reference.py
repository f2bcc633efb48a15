"""The operators of include/synera_tree.h in plain Python and float64 numpy, from their definitions, and the error their kernels may have."""
import math

import numpy as np

from shared_reference import PAGE, U, keys_of

OK, EINVAL, ERANGE, ENOSPC = 0, -1, -2, -3


def update_pages(table, held, free, n_free, ctx, new, n_rows, shared=None):
    """In place on numpy arrays -> cu, pos, slot, status.  One request after another, one page after another."""
    B, columns = table.shape
    stack = list(free[:n_free])
    status, count = np.zeros(B, np.int32), np.zeros(B, np.int64)
    asked, given, returned = 0, [], []
    for i in range(B):
        l, n, h = int(ctx[i]), int(new[i]), int(held[i])
        count[i] = n if 0 <= n <= PAGE * columns else 0
        need = -(-(l + n) // PAGE)
        if l < 0 or n < 0 or l + n > 2 ** 31 - 1:
            status[i] = ERANGE
        elif h < 0 or h > columns:
            status[i] = EINVAL
        elif need > columns:
            status[i] = ENOSPC
        else:
            keep = max(need, min(max(int(shared[i]), 0), h) if shared is not None else 0)
            if keep > h:
                asked += keep - h
                if asked > n_free:
                    status[i] = ENOSPC
                else:
                    given += [(i, c) for c in range(h, keep)]
            else:
                returned += [(i, c) for c in range(keep, h)]
            if status[i] == OK:
                held[i] = keep
    for i, c in given:
        table[i, c] = stack.pop()
    for i, c in reversed(returned):
        stack.append(table[i, c])
    free[: len(stack)] = stack
    cu = np.concatenate([[0], np.cumsum(count)])
    pos, slot = np.full(n_rows, -7, np.int64), np.full(n_rows, -7, np.int64)
    for i in range(B):
        for j in range(count[i]):
            if cu[i] + j < n_rows:
                p = int(ctx[i]) + j
                pos[cu[i] + j], slot[cu[i] + j] = (p, table[i, p // PAGE] * PAGE + p % PAGE) if status[i] == OK else (-1, -1)
    return cu, pos, slot, status, len(stack)


def paths(parent):
    """Nodes of one tree -> the nodes on each one's path, itself last."""
    out = []
    for j, p in enumerate(parent):
        out.append((out[p] if p >= 0 else []) + [j])
    return out


def attention(q, pool_k, pool_v, ctx, trees, table, scale):
    """float64 q [T, Hq, hd], pools of one layer, trees: the parents of each request's nodes -> o, lse, allowed error of o (a bf16 output) and
    of lse."""
    T, hq, hd = q.shape
    hkv = pool_k.shape[1]
    G = hq // hkv
    o, lse = np.zeros((T, hq, hd)), np.zeros((T, hq))
    eo, el = np.zeros_like(o), np.zeros_like(lse)
    t = 0
    with np.errstate(all="ignore"):
        for i, parent in enumerate(trees):
            L, n = int(ctx[i]), len(parent)
            for h in range(hkv):
                if n == 0:
                    continue
                k_all, v_all = keys_of(pool_k, pool_v, table[i], L + n, h)
                for j, path in enumerate(paths(parent)):
                    at = np.concatenate([np.arange(L), L + np.array(path, np.int64)])
                    k, v = k_all[at], v_all[at]
                    qq = q[t + j, h * G: (h + 1) * G]
                    x = qq @ k.T * scale
                    m = x.max(-1, keepdims=True)
                    p = np.exp(x - m)
                    l = p.sum(-1, keepdims=True)
                    size = (np.abs(qq) @ np.abs(k).T * scale).max(-1, keepdims=True)      # of a score's terms
                    e = (hd + 4) * U * size + 4 * U                                       # of an exponent
                    sl = slice(h * G, (h + 1) * G)
                    o[t + j, sl] = (p @ v) / l
                    lse[t + j, sl] = (m + np.log(l))[:, 0]
                    mean = (p @ np.abs(v)) / l
                    keys = L + n
                    # probabilities and output are bf16; 2 e: numerator and sum; all keys' terms are added in 32 bits, hidden ones as zeros
                    eo[t + j, sl] = 2.0 ** -8 * np.abs(o[t + j, sl]) + mean * (2.0 ** -8 + 2 * e + (keys + 64) * 2 * U)
                    el[t + j, sl] = (e + (keys + 64) * U)[:, 0] + 4 * U * (np.abs(lse[t + j, sl]) + np.abs(m[:, 0]) + 1)
            t += n
    return o, lse, eo, el


def accept(trees, tokens, target, anchor=None, given=None):
    """-> accept_len, token, path (-1 behind its end), n_path"""
    out, t = [], 0
    path_rows = []
    for i, parent in enumerate(trees):
        n = len(parent)
        g = min(max(int(given[i]), 0), n) if given is not None else 0
        path = list(range(g))
        want = int(target[t + g - 1]) if g else (int(anchor[i]) if anchor is not None and n else -1)
        while g or (anchor is not None and n):
            at = path[-1] if path else -1
            nxt = [c for c in range(g, n) if parent[c] == at and tokens[t + c] == want]
            if not nxt:
                break
            path.append(nxt[0])
            want = int(target[t + nxt[0]])
        out.append((len(path) - g, want, len(path)))
        path_rows += path + [-1] * (n - len(path))
        t += n
    a = np.array(out, np.int64).reshape(-1, 3)
    return a[:, 0], a[:, 1], np.array(path_rows, np.int64), a[:, 2]


def adjust(x, req, history, history_len, n_prompt, rho, pres, freq, bias_id, bias, allowed, path_tokens):
    """x float64 [R, V]; per-request arrays or None; allowed bool [R, V] or None; path_tokens: a list of tokens for each row -> (y, the error
    that 32-bit steps may leave)."""
    y = x.copy()
    size = np.abs(x)
    V = x.shape[1]
    with np.errstate(all="ignore"):
        for r in range(len(x)):
            i = req[r]
            seen, made = set(), {}
            if history is not None:
                for e, t in enumerate(history[i][: min(max(int(history_len[i]), 0), len(history[i]))]):
                    if 0 <= t < V:
                        seen.add(int(t))
                        if e >= (n_prompt[i] if n_prompt is not None else 0):
                            made[int(t)] = made.get(int(t), 0) + 1
            for t in path_tokens[r]:
                if 0 <= t < V:
                    seen.add(int(t))
                    made[int(t)] = made.get(int(t), 0) + 1
            for t in seen:
                if rho is not None:
                    y[r, t] = y[r, t] / rho[i] if y[r, t] > 0 else y[r, t] * rho[i]
                size[r, t] = abs(y[r, t])
            for t, g in made.items():
                pen = (freq[i] * g if freq is not None else 0.0) + (pres[i] if pres is not None else 0.0)
                size[r, t] += 2 * (abs(freq[i] * g) if freq is not None else 0.0) + 2 * (abs(pres[i]) if pres is not None else 0.0)
                y[r, t] -= pen
            if bias_id is not None:
                last = {int(t): e for e, t in enumerate(bias_id[i]) if 0 <= t < V}
                for t, e in last.items():
                    y[r, t] += bias[i][e]
                    size[r, t] += abs(bias[i][e])
        if allowed is not None:
            y[~allowed] = -math.inf
    # a quotient or product, a fused product and sum, a difference and a sum: each rounds once, to half a step of what is there
    return y, 4 * U * np.where(np.isfinite(size), size, 0)
