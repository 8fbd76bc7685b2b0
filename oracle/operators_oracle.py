"""Plain fp64 definitions of what stands around the multi-LoRA layers: products with 8-bit operands, counter-based dropout, block
edges (norms, gate, residual scale) and the preference loss.  numpy only; shares no code with the library."""
from __future__ import annotations

import numpy as np


# ---- dropout -------------------------------------------------------------------------------------------------------------------

def philox(counter, key) -> list:
    """Four 32-bit words (uint64 arrays) of ten Philox 4x32 rounds; counter: four arrays, key: two numbers."""
    m = np.uint64(0xFFFFFFFF)
    c = [np.asarray(x, dtype=np.uint64) & m for x in counter]
    k = [int(key[0]) & 0xFFFFFFFF, int(key[1]) & 0xFFFFFFFF]
    for _ in range(10):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> np.uint64(32)) ^ c[1] ^ np.uint64(k[0]), b & m, (a >> np.uint64(32)) ^ c[3] ^ np.uint64(k[1]), a & m]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return c


def threshold(p: float) -> int:
    return int(round(65536.0 * float(np.float32(p))))


def keep_mask(rows: int, cols: int, p: float, seed: int, counter: int) -> np.ndarray:
    """Truth values [rows, cols] of one segment."""
    pieces = -(-cols // 8)
    r, c = np.meshgrid(np.arange(rows), np.arange(pieces), indexing="ij")
    w = philox([c, r, np.full_like(c, counter & 0xFFFFFFFF), np.full_like(c, (counter >> 32) & 0xFFFFFFFF)], [seed & 0xFFFFFFFF, seed >> 32])
    numbers = np.stack([(w[j // 2] >> np.uint64(16 * (j % 2))) & np.uint64(0xFFFF) for j in range(8)], axis=-1)
    return numbers.reshape(rows, 8 * pieces)[:, :cols] >= threshold(p)


def dropout(X, offsets, rates, seeds, counter, add=None) -> np.ndarray:
    Y = np.zeros(X.shape)
    for i, (p, seed) in enumerate(zip(rates, seeds)):
        a, b = offsets[i], offsets[i + 1]
        if threshold(p) == 65536:
            continue
        keep = keep_mask(b - a, X.shape[1], p, seed, counter)
        with np.errstate(invalid="ignore"):
            Y[a:b] = np.where(keep, X[a:b] * (65536 / (65536 - threshold(p))), 0.0)
    return Y if add is None else Y + add


# ---- block edges ---------------------------------------------------------------------------------------------------------------

def _row(v, i):
    return v[i] if v.ndim == 2 else v


def edge(h, y, offsets, post, gate, scale, pre, eps_post=1e-5, eps_pre=1e-5):
    """(h_out, x).  post / gate / pre [d] or [N, d] or None, scale [N] or None."""
    h_out = h.copy()
    x = None if pre is None else np.empty(h.shape)
    for i in range(len(offsets) - 1):
        rows = slice(offsets[i], offsets[i + 1])
        if post is not None:
            u = y[rows] / np.sqrt((y[rows] ** 2).mean(1, keepdims=True) + eps_post) * _row(post, i)
            h_out[rows] += (1.0 if scale is None else scale[i]) * (1.0 if gate is None else _row(gate, i)) * u
        if pre is not None:
            x[rows] = h_out[rows] / np.sqrt((h_out[rows] ** 2).mean(1, keepdims=True) + eps_pre) * _row(pre, i)
    return h_out, x


def edge_grads(h, y, offsets, post, gate, scale, pre, dx, dh_out, eps_post=1e-5, eps_pre=1e-5):
    """Gradients by the chain rule, and next to each the same expression with every term's magnitude (what rounding is relative to).
    dict name -> (value, magnitude); per-adapter parameter gradients [N, d], shared ones [d]."""
    N, d = len(offsets) - 1, h.shape[1]
    h_out, _ = edge(h, y, offsets, post, gate, scale, pre, eps_post, eps_pre)
    terms = np.abs(h) + np.abs(h_out - h)
    dh, dh_m = np.zeros(h.shape), np.zeros(h.shape)
    out = {"dh": (dh, dh_m)}
    if post is not None:
        dy, dy_m = np.zeros(h.shape), np.zeros(h.shape)
        out["dy"] = (dy, dy_m)
    C, Cm, D, Dm = (np.zeros((N, d)) for _ in range(4))
    S, Sm = np.zeros(N), np.zeros(N)
    for i in range(N):
        rows = slice(offsets[i], offsets[i + 1])
        e = np.zeros((offsets[i + 1] - offsets[i], d)) if dh_out is None else dh_out[rows].copy()
        em = np.abs(e)
        if pre is not None:
            rh = 1 / np.sqrt((h_out[rows] ** 2).mean(1, keepdims=True) + eps_pre)
            xh, xm, v = h_out[rows] * rh, terms[rows] * rh, _row(pre, i) * dx[rows]
            e += rh * (v - xh * (v * xh).mean(1, keepdims=True))
            em += rh * (np.abs(v) + xm * (np.abs(v) * xm).mean(1, keepdims=True))
            D[i], Dm[i] = (dx[rows] * xh).sum(0), (np.abs(dx[rows]) * xm).sum(0)
        dh[rows], dh_m[rows] = e, em
        if post is not None:
            ry = 1 / np.sqrt((y[rows] ** 2).mean(1, keepdims=True) + eps_post)
            yh, q, s = y[rows] * ry, (1.0 if gate is None else _row(gate, i)) * _row(post, i), 1.0 if scale is None else scale[i]
            dy[rows] = s * ry * (q * e - yh * (q * e * yh).mean(1, keepdims=True))
            dy_m[rows] = abs(s) * ry * (np.abs(q) * em + np.abs(yh) * (np.abs(q) * em * np.abs(yh)).mean(1, keepdims=True))
            C[i], Cm[i] = (e * yh).sum(0), (em * np.abs(yh)).sum(0)
            S[i], Sm[i] = (q * e * yh).sum(), (np.abs(q) * em * np.abs(yh)).sum()

    def shared(p, v):
        return v if p.ndim == 2 else v.sum(0)

    if pre is not None:
        out["d_pre"] = (shared(pre, D), shared(pre, Dm))
    if post is not None:
        s = np.ones((N, 1)) if scale is None else scale[:, None]
        g = 1.0 if gate is None else gate
        out["d_post"] = (shared(post, s * g * C), shared(post, np.abs(s * g) * Cm))
        if gate is not None:
            out["d_gate"] = (shared(gate, s * post * C), shared(gate, np.abs(s * post) * Cm))
        if scale is not None:
            out["d_scale"] = (S, Sm)
    return out


# ---- preference loss -------------------------------------------------------------------------------------------------------------

def row_logp(z, targets):
    """(log-probability of each row's target, lse), zeros where the target is outside the vocabulary.  The log-probability comes from differences to the
    row's maximum, which a row of very large or very low logits still has: its lse does not hold the logarithm of the sum."""
    l, lse = np.zeros(len(z)), np.zeros(len(z))
    for t, v in enumerate(targets):
        if 0 <= v < z.shape[1]:
            m = z[t].max()
            m = 0.0 if m == -np.inf else m
            with np.errstate(divide="ignore", invalid="ignore"):
                log_sum = np.log(np.exp(z[t] - m).sum())
                l[t], lse[t] = (z[t, v] - m) - log_sum, m + log_sum
    return l, lse


def preference(z, targets, seq_offsets, owner, params, ref=None, dloss=None):
    """dict of logp [2 P], margin [P], loss [N], coef [2 P] (gradient of the summed losses by a sequence's log-probability) and dz.
    params: (beta, smoothing, nll) per adapter."""
    row, lse = row_logp(z, targets)
    S = len(seq_offsets) - 1
    ref = np.zeros(S) if ref is None else ref
    dloss = np.ones(len(params)) if dloss is None else dloss
    V = z.shape[1]
    counted = np.array([0 <= v < V for v in targets], dtype=bool)
    logp = np.array([row[a:b].sum() for a, b in zip(seq_offsets, seq_offsets[1:])])
    n = np.array([counted[a:b].sum() for a, b in zip(seq_offsets, seq_offsets[1:])])
    margin, coef, loss = np.zeros(S // 2), np.zeros(S), np.zeros(len(params))
    for j, i in enumerate(owner):
        beta, a, w = params[i]
        w = w / n[2 * j] if n[2 * j] else 0.0
        m = beta * ((logp[2 * j] - ref[2 * j]) - (logp[2 * j + 1] - ref[2 * j + 1]))
        margin[j] = m
        P = sum(1 for o in owner if o == i)
        f = ((1 - a) * np.logaddexp(0, -m) if a < 1 else 0.0) + (a * np.logaddexp(0, m) if a > 0 else 0.0)      # a term without weight has no part
        loss[i] += (f - (w * logp[2 * j] if w else 0.0)) / P
        up, down = np.exp(-np.logaddexp(0, -m)), np.exp(-np.logaddexp(0, m))        # sigma(m), sigma(-m)
        dm = beta * (a * up - (1 - a) * down)
        coef[2 * j], coef[2 * j + 1] = dloss[i] * (dm - w) / P, -dloss[i] * dm / P
    dz = np.zeros(z.shape)
    for q in range(S):
        for t in range(seq_offsets[q], seq_offsets[q + 1]):
            if counted[t]:
                m = z[t].max()
                with np.errstate(invalid="ignore"):
                    e = np.exp(z[t] - (0.0 if m == -np.inf else m))
                    dz[t] = -coef[q] * (e / e.sum())
                dz[t, targets[t]] += coef[q]
    return {"logp": logp, "row": row, "margin": margin, "loss": loss, "coef": coef, "dz": dz, "counted": counted, "lse": lse}


# ---- products with 8-bit operands --------------------------------------------------------------------------------------------------

def e4m3_values() -> np.ndarray:
    """The finite magnitudes that 4 exponent and 3 mantissa bits hold, ascending; the index is the code."""
    v = [m * 2.0 ** -9 for m in range(8)]
    v += [(1 + m / 8) * 2.0 ** (e - 7) for e in range(1, 16) for m in range(8)]
    return np.array(v[:-1])            # the last code is NaN


def quantise_block(x: np.ndarray) -> np.ndarray:
    """What a block stands for under its own scale, that of its largest finite magnitude: the nearest value, ties to the even code; NaN for what is not
    finite."""
    finite = np.isfinite(x)
    if not finite.all():
        return np.where(finite, quantise_block(np.where(finite, x, 0.0)), np.nan)
    amax = np.abs(x).max() if x.size else 0.0
    if amax == 0.0:
        return np.zeros(x.shape)
    scale = 2.0 ** -127
    while amax > 448.0 * scale:
        scale *= 2.0
    tab = e4m3_values()
    v = np.abs(x) / scale
    hi = np.minimum(np.searchsorted(tab, v), len(tab) - 1)
    lo = np.maximum(hi - 1, 0)
    up = (tab[hi] - v < v - tab[lo]) | ((tab[hi] - v == v - tab[lo]) & (hi % 2 == 0)) | (tab[hi] == v)
    return np.sign(x) * np.where(up, tab[hi], tab[lo]) * scale


def quantise_rows(x: np.ndarray) -> np.ndarray:
    out = np.empty(x.shape)
    for r in range(x.shape[0]):
        for c in range(0, x.shape[1], 128):
            out[r, c:c + 128] = quantise_block(x[r, c:c + 128])
    return out


def quantise_weight(w: np.ndarray) -> np.ndarray:
    out = np.empty(w.shape)
    for r in range(0, w.shape[0], 128):
        for c in range(0, w.shape[1], 128):
            out[r:r + 128, c:c + 128] = quantise_block(w[r:r + 128, c:c + 128])
    return out
