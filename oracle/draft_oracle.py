"""fp64 CPU oracle for speculative decoding on the ring and the state, and for rotary positions on several axes.
TEST INFRASTRUCTURE ONLY: imported by the tests and by nothing in the product.

Attention of a tree of drafts is defined through what it stands for: node n's output is the output of the operator's last
row on the sequence (history, path of n), which rattn_oracle evaluates directly.  So there is no ring, no state and no tree
mask here: a caller hands over the whole history.  Verification follows the sequential description word by word, in fp64 or in
exact rational arithmetic."""
from __future__ import annotations

from fractions import Fraction

import numpy as np

from . import rattn_oracle as O


def path_of(parents, i):
    """Nodes from the root down to i, or None where i is no part of the tree."""
    line = [i]
    while True:
        p = int(parents[line[0]])
        if p == -1:
            return line
        if p < 0 or p >= line[0]:
            return None
        line.insert(0, p)


def draft_attention(q, k, v, parents, k_hist, v_hist, w, scale=1.0, eps=O.DEFAULT_EPS, gs=None, gr=None, phi=O.PHI_SOFTMAX):
    """One batch entry: q [Hq,N,d], k, v [Hkv,N,d], parents [N], k_hist, v_hist [Hkv,pos,d].  Rows of no node are NaN."""
    Hq, N, d = q.shape
    G = Hq // k.shape[0]
    out = np.full(q.shape, np.nan)
    for i in range(N):
        line = path_of(parents, i)
        if line is None:
            continue
        for h in range(Hq):
            keys = np.concatenate([k_hist[h // G], k[h // G, line]])
            vals = np.concatenate([v_hist[h // G], v[h // G, line]])
            t = np.array([len(keys) - 1])
            row = q[h, i][None]
            o_swa, _ = O.swa_rows(row, t, keys, vals, w, scale)
            o_rla, _ = O.rla_rows(row, t, keys, vals, w, phi)
            y = O.rmsnorm(o_swa, None if gs is None else gs[h], eps) + O.rmsnorm(o_rla, None if gr is None else gr[h], eps)
            out[h, i] = y[0]
    return out


def cache_of(k_hist, v_hist, w, phi=O.PHI_SOFTMAX, fill=0.0):
    """(k_ring, v_ring, state) of a history [Hkv,pos,d]; unused slots hold `fill`."""
    Hkv, pos, d = k_hist.shape
    rings = []
    for x in (k_hist, v_hist):
        r = np.full((Hkv, w, d), fill)
        for j in range(max(0, pos - w), pos):
            r[:, j % w] = x[:, j]
        rings.append(r)
    state = np.zeros((Hkv, d, d))
    for h in range(Hkv):
        for j in range(max(0, pos - w)):
            state[h] += np.outer(O.feature_map(k_hist[h, j][None], phi)[0], v_hist[h, j])
    return rings[0], rings[1], state


def verify(tokens, parents, p, q, u):
    """One batch entry: (accepted nodes, token).  p, q [N,V] (q may be None), u [N]; Fractions stay exact."""
    N = len(tokens)
    if parents[0] != -1:
        return [], -1
    V = len(p[0])
    clean = lambda row: [x if x > 0 else 0 * u[0] for x in row]  # noqa: E731
    line, c = [0], 0
    r, Z = clean(p[0]), 1
    for i in range(1, N):
        if parents[i] != c or not 0 <= tokens[i] < V:
            continue
        x = tokens[i]
        qc = None if q is None else clean(q[c])
        if u[i] * (1 if q is None else qc[x]) * Z < r[x]:
            line.append(i)
            c = i
            r, Z = clean(p[c]), 1
        elif q is None:
            Z = Z - r[x]
            r = [0 * y if j == x else y for j, y in enumerate(r)]
        else:
            less = [max(y - Z * s, 0 * y) for y, s in zip(r, qc)]
            if sum(less) * 2 ** 40 > Z:
                r, Z = less, sum(less)
    if not sum(r) > 0:
        r = clean(p[c])
    total, run = sum(r), 0
    for x, y in enumerate(r):
        run += y
        if run > u[0] * total:
            return line, x
    return line, -1


def rational(row):
    return [Fraction(float(x)) for x in row]


def commit(k, v, path, n, k_ring, v_ring, state, pos, phi=O.PHI_SOFTMAX):
    """One batch entry: n single steps' effect on copies of ring and state."""
    k_ring, v_ring, state = k_ring.copy(), v_ring.copy(), state.copy()
    w = k_ring.shape[1]
    for a in range(n):
        at = (pos + a) % w
        if pos + a >= w:
            for h in range(k.shape[0]):
                state[h] += np.outer(O.feature_map(k_ring[h, at][None], phi)[0], v_ring[h, at])
        k_ring[:, at], v_ring[:, at] = k[:, path[a]], v[:, path[a]]
    return k_ring, v_ring, state


def axes_angles(at, sections, order, theta, d):
    """Angles [B,T,d/2]: at [n_axes,B,T], order "runs", "own" or "dealt"."""
    A, B, T = at.shape
    ang = np.zeros((B, T, d // 2))
    if order == "dealt":
        owners, left = [], list(sections)
        while sum(left):
            for a in range(A):
                if left[a]:
                    left[a] -= 1
                    owners.append(a)
    else:
        owners = [a for a in range(A) for _ in range(sections[a])]
    seen = [0] * A
    for i, a in enumerate(owners):
        exponent = seen[a] / sections[a] if order == "own" else 2 * i / d
        seen[a] += 1
        ang[..., i] = at[a].astype(np.float64) * theta ** -exponent
    return ang


def axes_rotate(x, ang):
    """x [B,H,T,d] turned by ang [B,T,d/2]."""
    half = x.shape[-1] // 2
    c, s = np.cos(ang)[:, None], np.sin(ang)[:, None]
    lo, hi = x[..., :half], x[..., half:]
    return np.concatenate([lo * c - hi * s, hi * c + lo * s], -1)


def qk_prologue_axes(x, gain, ang, eps=O.DEFAULT_EPS):
    return axes_rotate(O.rmsnorm(x, gain, eps), ang)


def qk_prologue_axes_bwd(x, gain, ang, dy, eps=O.DEFAULT_EPS):
    """(dx, dgain) of qk_prologue_axes."""
    d = x.shape[-1]
    dn = axes_rotate(dy, -ang)
    r = 1.0 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    dgain = (dn * x * r).sum((0, 1, 2))
    dn = dn if gain is None else dn * gain
    return r * dn - x * r ** 3 * (dn * x).sum(-1, keepdims=True) / d, dgain
