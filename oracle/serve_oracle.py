"""fp64 oracle of the serving step and of the per-head norm + rotation, from
their definitions: one request, token and row at a time, numpy only."""
from __future__ import annotations

import math

import numpy as np

PAGE = 64


def rotate(z, cos, sin, interleaved):
    """z [d] with its first 2 len(cos) entries turned pair by pair."""
    y = np.array(z, dtype=np.float64)
    half = len(cos)
    for i in range(half):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
        y[a] = z[a] * cos[i] - z[b] * sin[i]
        y[b] = z[b] * cos[i] + z[a] * sin[i]
    return y


def norm_rope_row(x, w, cos, sin, eps, interleaved):
    r = 1.0 / math.sqrt(float(np.mean(x * x)) + eps)
    return rotate(w * x * r, cos, sin, interleaved)


def norm_rope_row_grad(x, w, cos, sin, eps, interleaved, dy):
    """(dx, the row's term of dw)."""
    r = 1.0 / math.sqrt(float(np.mean(x * x)) + eps)
    xh = x * r
    dz = rotate(dy, cos, -np.asarray(sin), interleaved)   # the transposed rotation
    u = w * dz
    return r * (u - xh * float(np.mean(u * xh))), dz * xh


def qk_norm_rope(qkv, wq, wk, cos, sin, positions, Hq, eps, interleaved):
    """qkv [T, Hq + 2 Hkv, d], positions [T] -> (Q [T, Hq, d], K, V [T, Hkv, d])."""
    T, H, _ = qkv.shape
    Hkv = (H - Hq) // 2
    out = np.array(qkv, dtype=np.float64)
    for t in range(T):
        p = positions[t]
        for h in range(Hq + Hkv):
            out[t, h] = norm_rope_row(qkv[t, h], wq if h < Hq else wk, cos[p], sin[p], eps, interleaved)
    return out[:, :Hq], out[:, Hq:Hq + Hkv], out[:, Hq + Hkv:]


def qk_norm_rope_grad(qkv, wq, wk, cos, sin, positions, Hq, eps, interleaved, dY):
    """dY [T, Hq + 2 Hkv, d] -> (dqkv, dwq, dwk)."""
    T, H, d = qkv.shape
    Hkv = (H - Hq) // 2
    dx = np.array(dY, dtype=np.float64)
    dw = np.zeros((2, d))
    for t in range(T):
        p = positions[t]
        for h in range(Hq + Hkv):
            k = int(h >= Hq)
            dx[t, h], term = norm_rope_row_grad(qkv[t, h], wk if k else wq, cos[p], sin[p], eps, interleaved, dY[t, h])
            dw[k] += term
    return dx, dw[0], dw[1]


def plan(seq_lens, new_lens, free_pages, free_begin, table, T, held_lens=None):
    """(kv_lens, cu, positions, slots, free_end, table) of a plan that fits."""
    table = np.array(table)
    at = free_begin
    cu, positions, slots = [0], [], []
    for b, (s, n) in enumerate(zip(seq_lens, new_lens)):
        for p in range(s, s + n):
            if p % PAGE == 0 and (held_lens is None or p >= held_lens[b]):   # a block no held page covers
                table[b, p // PAGE] = free_pages[at]
                at += 1
            positions.append(p)
            slots.append(int(table[b, p // PAGE]) * PAGE + p % PAGE)
        cu.append(len(slots))
    pad = [-1] * (T - len(slots))
    return ([s + n for s, n in zip(seq_lens, new_lens)], cu, positions + pad, slots + pad, at, table)


def chunk_attention(Q, K_cache, V_cache, table, cu, kv_lens, scale):
    """Q [T, Hq, d], caches [P, Hkv, 64, d] -> O [T, Hq, d], LSE [T, Hq], the same on |V|, and per row the
    largest sum |q||k| over its keys (rows of no request: NaN)."""
    T, Hq, d = Q.shape
    Hkv = K_cache.shape[1]
    O, A = np.full((T, Hq, d), np.nan), np.full((T, Hq, d), np.nan)
    LSE, S = np.full((T, Hq), np.nan), np.full((T, Hq), np.nan)
    for b, L in enumerate(kv_lens):
        n = cu[b + 1] - cu[b]
        if n == 0:
            continue
        pages = table[b][:-(-L // PAGE)]
        for g in range(Hkv):
            K = np.concatenate([K_cache[p, g] for p in pages])[:L]
            V = np.concatenate([V_cache[p, g] for p in pages])[:L]
            for i in range(n):
                m = L - n + i + 1
                for h in range(g * (Hq // Hkv), (g + 1) * (Hq // Hkv)):
                    q = Q[cu[b] + i, h]
                    z = scale * (K[:m] @ q)
                    top = z.max()
                    e = np.exp(z - top)
                    t = cu[b] + i
                    O[t, h] = e @ V[:m] / e.sum()
                    A[t, h] = e @ np.abs(V[:m]) / e.sum()
                    LSE[t, h] = top + math.log(e.sum())
                    S[t, h] = (np.abs(K[:m]) @ np.abs(q)).max()
    return O, LSE, A, S


def verify(tokens, cu, target, draft, u, noise, max_draft):
    """draft None: certain drafts.  Returns (accepted, tokens [B, max_draft + 1])."""
    accepted, out = [], []
    for b in range(len(cu) - 1):
        n, row = cu[b + 1] - cu[b], []
        w = None
        for j in range(n):
            x, p = int(tokens[cu[b] + j]), target[cu[b] + b + j]
            if draft is None:
                q = np.zeros_like(p)
                if 0 <= x < len(p):
                    q[x] = np.inf
                qx = 1.0
            else:
                q = draft[cu[b] + j]
                qx = q[x] if 0 <= x < len(p) else np.nan
            if not (0 <= x < len(p) and u[cu[b] + j] * qx < p[x]):
                w = np.where(p > q, p - q, 0.0)
                if not (w > 0).any():
                    w = p
                break
            row.append(x)
        if w is None:
            w = target[cu[b] + b + n]
        accepted.append(len(row))
        ok = (w > 0) & (noise[b] > 0)
        score = np.where(ok, w / np.where(ok, noise[b], 1), 0)
        row.append(int(score.argmax()) if ok.any() else -1)   # argmax: the lowest of equal ones
        out.append(row + [-1] * (max_draft + 1 - len(row)))
    return np.array(accepted), np.array(out)


def page_scale(amax):
    """Least power of two s, 2^-64 <= s <= 2^120, with amax <= 448 s."""
    k = -64
    while amax > 448.0 * 2.0 ** k and k < 120:
        k += 1
    return 2.0 ** k


def round_e4m3(x):
    """To the nearest e4m3 number (4 significant bits, least step 2^-9, largest 448), ties to even; what is not finite
    becomes NaN."""
    x = np.asarray(x, dtype=np.float64)
    finite = np.isfinite(x)
    a = np.abs(np.where(finite, x, 0.0))
    _, e = np.frexp(np.where(a > 0, a, 1.0))
    step = np.ldexp(1.0, np.maximum(e - 4, -9))
    r = np.minimum(np.round(a / step) * step, 448.0)
    return np.where(finite, np.copysign(r, np.where(finite, x, 0.0)), np.nan)


def append8(qkv, wq, wk, cos, sin, positions, slots, Hq, eps, interleaved, K_cache, V_cache, K_scale, V_scale):
    """Caches [P, Hkv, 64, d] of e4m3 numbers, scales [P, Hkv].  Returns Q, the new caches before rounding (in units of the
    new scales), and the new scales.  Tokens of slot -1 are left out."""
    live = [t for t, s in enumerate(slots) if s >= 0]
    Q, K, V = qk_norm_rope(qkv, wq, wk, cos, sin, np.maximum(positions, 0), Hq, eps, interleaved)
    out = []
    for new, cache, scale in ((K, K_cache, K_scale), (V, V_cache, V_scale)):
        cache, scale = np.array(cache, dtype=np.float64), np.array(scale, dtype=np.float64)
        for page in sorted({slots[t] // PAGE for t in live}):
            ts = [t for t in live if slots[t] // PAGE == page]
            for g in range(scale.shape[1]):
                y = np.array([new[t, g] for t in ts])
                s = page_scale(float(np.abs(y[np.isfinite(y)]).max(initial=0.0)))
                if all(slots[t] % PAGE != 0 for t in ts):
                    s = max(s, scale[page, g])
                    cache[page, g] *= scale[page, g] / s
                for t in ts:
                    cache[page, g, slots[t] % PAGE] = new[t, g] / s
                scale[page, g] = s
        out += [cache, scale]
    return Q, out[0], out[2], out[1], out[3]
