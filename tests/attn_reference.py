"""64-bit definitions of the operators of include/qknorm_attn.h for the tests: plain loops over sequences and heads,
no code shared with the library."""
import math

import numpy as np
import torch

F8, BF16 = torch.float8_e4m3fn, torch.bfloat16
HALF_STEP = {BF16: 2.0 ** -8, F8: 2.0 ** -4}       # relative, half a step
F8_TINY = 2.0 ** -10                               # half a step of E4M3's subnormals


def widen(t):
    return t.detach().cpu().double()


def rotate(x, positions, inv_freq, head_dim, interleaved, inverse=False, mscale=1.0):
    """x [T, heads*head_dim] float64 -> (rotated, magnitude |a| + |b| of every element's pair)."""
    T = x.shape[0]
    x = x.reshape(T, -1, head_dim).clone()
    y, mag = x.clone(), x.abs()
    for i, f in enumerate(inv_freq.tolist()):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + len(inv_freq))
        ang = positions.double() * f * (-1.0 if inverse else 1.0)
        c, s = torch.cos(ang)[:, None], torch.sin(ang)[:, None]
        y[:, :, a] = (x[:, :, a] * c - x[:, :, b] * s) * mscale
        y[:, :, b] = (x[:, :, b] * c + x[:, :, a] * s) * mscale
        mag[:, :, a] = mag[:, :, b] = (x[:, :, a].abs() + x[:, :, b].abs()) * abs(mscale)
    return y.reshape(T, -1), mag.reshape(T, -1)


def norm(x, gamma, eps, width):
    T = x.shape[0]
    h = x.reshape(T, -1, width)
    r = 1.0 / torch.sqrt((h * h).mean(-1, keepdim=True) + eps)
    return (h * r).reshape(T, -1) * gamma


def sees(pos, L, causal, window):
    """Boolean [L]: the keys a row at `pos` sees."""
    j = np.arange(L)
    ok = np.ones(L, dtype=bool)
    if causal:
        ok &= j <= pos
    if window:
        ok &= j > pos - window
    return ok


def attention(q, k_pool, v_pool, table, kv_lens, q_starts, heads_q, *, scale, causal=True, window=0, k_scale=1.0, v_scale=1.0,
              max_kv=None):
    """numpy float64; q [T, heads_q*D], pools [pages, page, H, D].  Returns out (NaN in rows of no sequence), lse, and per
    element the pieces of the error bound: A = sum p |v|, S = largest scale * sum |q||k| over the keys seen, V = sum |v|."""
    q = q.numpy()
    k_pool, v_pool = k_pool.numpy() * k_scale, v_pool.numpy() * v_scale
    pages, page, H, D = k_pool.shape
    G = heads_q // H
    T = q.shape[0]
    out = np.full((T, heads_q, D), np.nan)
    A, V = np.zeros((T, heads_q, D)), np.zeros((T, heads_q, D))
    S, lse, n_keys = np.zeros((T, heads_q)), np.full((T, heads_q), np.nan), np.zeros((T, heads_q))
    q = q.reshape(T, heads_q, D)
    for b, L in enumerate(kv_lens):
        r0, r1 = q_starts[b], q_starts[b + 1]
        if max_kv is not None:
            keys = min(L, max_kv)
        else:
            keys = L
        keys = max(0, min(keys, len(table[b]) * page))
        ids = [table[b][j // page] for j in range(0, keys, page)]
        kk, vv = np.zeros((len(ids) * page, H, D)), np.zeros((len(ids) * page, H, D))
        for n, e in enumerate(ids):
            if 0 <= e < pages:
                kk[n * page:(n + 1) * page], vv[n * page:(n + 1) * page] = k_pool[e], v_pool[e]
        for i in range(r1 - r0):
            pos = L - (r1 - r0) + i
            ok = np.nonzero(sees(pos, keys, causal, window))[0]
            for h in range(heads_q):
                if len(ok) == 0:
                    out[r0 + i, h], lse[r0 + i, h] = 0.0, -math.inf
                    continue
                K, W = kk[ok, h // G], vv[ok, h // G]
                s = K @ q[r0 + i, h] * scale
                m = s.max()
                p = np.exp(s - m)
                l = p.sum()
                out[r0 + i, h] = p @ W / l
                lse[r0 + i, h] = m + math.log(l)
                A[r0 + i, h] = p @ np.abs(W) / l
                V[r0 + i, h] = np.abs(W).sum(0)
                S[r0 + i, h] = scale * (np.abs(K) @ np.abs(q[r0 + i, h])).max()
                n_keys[r0 + i, h] = len(ok)
    return dict(out=out, lse=lse, A=A, S=S, V=V, n=n_keys)


def attention_bounds(ref, D, e4m3):
    """How far out and lse may be off.  A score is a sum of D products in fp32: off by at most e = (D + 4) 2^-24 S, which moves
    every weight by a factor e^(+-e) and with the normalisation twice that.  A weight is rounded to bf16 (2^-8) or, with an
    FP8 cache, fp16 (2^-11, and 2^-25 absolute below its normal range against a largest weight of at least 1); the sum of
    n weights in fp32 adds n/32 + 16 steps; the result is rounded to bf16."""
    e = (D + 4) * 2.0 ** -24 * ref["S"][..., None] + 2.0 ** -21
    steps = (ref["n"] / 32 + 16)[..., None] * 2.0 ** -24
    w = 2.0 ** -11 if e4m3 else 2.0 ** -8
    tol = (w + 3 * e + 2 * steps) * ref["A"] + 2.0 ** -8 * np.abs(ref["out"]) * 1.01 + 1e-30
    if e4m3:
        tol = tol + 2.0 ** -25 * ref["V"]
    tol_lse = e[..., 0] + steps[..., 0] + 2.0 ** -22 * np.abs(np.where(np.isfinite(ref["lse"]), ref["lse"], 0.0))
    return tol, tol_lse
