"""The operators of include/synera_shared.h in float64 numpy, from their definitions, and the error their kernels may have: half a
step of each rounding to fewer bits, and the roundings of 32-bit sums over as many terms as there are."""
import math

import numpy as np
import torch

PAGE = 16
U = 2.0 ** -24                                       # half a step of f32


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def to64(t):
    return t.detach().to("cpu", torch.float32).numpy().astype(np.float64)


def frequencies(rot, base=10000.0, scaling=None):
    f = np.array([base ** (-2.0 * i / rot) for i in range(rot // 2)])
    if scaling is None:
        return f
    if scaling[0] == "linear":
        return f / scaling[1]
    _, factor, low, high, original = scaling
    out = []
    for v in f:
        r = original * v / (2 * math.pi)
        t = min(1.0, max(0.0, (r - low) / (high - low)))
        out.append((1 - t) * v / factor + t * v)
    return np.array(out)


def turn(x, pos, freq, layout, magnitude=1.0, gain=None, eps=0.0):
    """x [T, H, hd] float64 -> (turned, allowed 32-bit error): the error of a pair's sum, of the angle (half a turn in f32, and the
    64-bit product's own at far positions), and of the norm's sum over hd squares."""
    with np.errstate(all="ignore"):
        hd, slack = x.shape[-1], 0.0
        if gain is not None:
            x = x * gain / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
            slack = (hd + 8) * U
        half = len(freq)
        turns = np.abs(pos.astype(np.float64))[:, None] * freq / (2 * math.pi)
        ang = (pos.astype(np.float64)[:, None] * freq)[:, None]
        c, s = np.cos(ang) * magnitude, np.sin(ang) * magnitude
        off = (2 * math.pi * (turns * 2.0 ** -51) + 16 * U)[:, None] * abs(magnitude)
        y, err = x.copy(), np.abs(x) * slack
        a, b = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if layout == "interleaved" else (slice(0, half), slice(half, 2 * half))
        xa, xb = x[..., a], x[..., b]
        y[..., a], y[..., b] = xa * c - xb * s, xb * c + xa * s
        size = np.abs(xa) + np.abs(xb)
        err[..., a] = err[..., b] = size * (off + abs(magnitude) * (slack + 4 * U))
    return y, err


def keys_of(pool_k, pool_v, row, n, h):
    """The first n keys and values of KV head h of a request with page-table row `row`: [n, hd] each."""
    ids = row[: -(-n // PAGE)]
    return pool_k[ids, h].reshape(-1, pool_k.shape[-1])[:n], pool_v[ids, h].transpose(0, 2, 1).reshape(-1, pool_v.shape[2])[:n]


def attention(q, pool_k, pool_v, ctx, new, table, scale):
    """float64 q [T, Hq, hd], pools of one layer -> o, lse, allowed error of o (a bf16 output) and of lse."""
    T, hq, hd = q.shape
    hkv = pool_k.shape[1]
    G = hq // hkv
    o, lse = np.zeros((T, hq, hd)), np.zeros((T, hq))
    eo, el = np.zeros_like(o), np.zeros_like(lse)
    t = 0
    with np.errstate(all="ignore"):
        for i in range(len(ctx)):
            for h in range(hkv):
                if new[i] == 0:
                    continue
                k_all, v_all = keys_of(pool_k, pool_v, table[i], ctx[i] + new[i], h)
                for j in range(new[i]):
                    k, v = k_all[: ctx[i] + j + 1], v_all[: ctx[i] + j + 1]
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
                    n = len(k)
                    # probabilities and output are bf16; 2 e: numerator and sum; n terms are added in 32 bits
                    eo[t + j, sl] = 2.0 ** -8 * np.abs(o[t + j, sl]) + mean * (2.0 ** -8 + 2 * e + (n + 64) * 2 * U)
                    el[t + j, sl] = (e + (n + 64) * U)[:, 0] + 4 * U * (np.abs(lse[t + j, sl]) + np.abs(m[:, 0]) + 1)
            t += new[i]
    return o, lse, eo, el


def close(got, want, allowed, name):
    """Element by element; infinities and NaN where they are wanted and nowhere else."""
    got = np.asarray(got, np.float64)
    assert got.shape == want.shape, f"{name}: {got.shape}, wanted {want.shape}"
    fine = np.isfinite(want)
    assert np.array_equal(np.isnan(got), np.isnan(want)), f"{name}: NaN at {np.argwhere(np.isnan(got) != np.isnan(want))[:4].tolist()}"
    assert np.array_equal(got[~fine & ~np.isnan(want)], want[~fine & ~np.isnan(want)]), f"{name}: infinities differ"
    off = np.abs(np.where(fine, got, 0) - np.where(fine, want, 0)) - np.where(fine, allowed, 0)
    worst = np.unravel_index(np.argmax(off), off.shape) if off.size else None
    assert not off.size or off[worst] <= 0, f"{name}: {got[worst]} at {worst}, wanted {want[worst]} +- {np.broadcast_to(allowed, want.shape)[worst]:.3e}"
