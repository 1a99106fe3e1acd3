"""Float64 definitions of the decoder-block operators: RMSNorm with the residual
added, rotary positions, sliding-window attention with sinks (training and single
tokens), and what a rolling cache holds.  Test infrastructure only: plain numpy
over the full score matrix, nothing shared with the HIP path.

These operators are not in the paper; their formulas are stated here.
"""

from __future__ import annotations

import numpy as np

E4M3_MAX = 448.0


def _f64(x):
    return np.asarray(x, dtype=np.float64)


# ---------------------------------------------------------------------------
# RMSNorm
# ---------------------------------------------------------------------------
def rmsnorm_fwd(x, gamma, residual=None, eps=1e-5):
    """(y, h, rstd) of h = x + residual, rstd = 1 / sqrt(mean(h^2) + eps), y = h rstd gamma."""
    h = _f64(x) if residual is None else _f64(x) + _f64(residual)
    rstd = 1.0 / np.sqrt(np.mean(h * h, axis=-1) + eps)
    return h * rstd[..., None] * _f64(gamma), h, rstd


def rmsnorm_bwd(h, gamma, rstd, dy, dh=None):
    """(dx, dgamma) for given h and rstd: xhat = h rstd, g = dy gamma."""
    h, gamma, rstd, dy = _f64(h), _f64(gamma), _f64(rstd), _f64(dy)
    xhat = h * rstd[:, None]
    g = dy * gamma
    dx = rstd[:, None] * (g - xhat * np.mean(g * xhat, axis=1, keepdims=True))
    return dx + (0.0 if dh is None else _f64(dh)), np.sum(dy * xhat, axis=0)


def q8_scales(y, group=0):
    """Scale of each group of consecutive columns: max(max|y| / 448, 2^-126)."""
    y = _f64(y)
    R, C = y.shape
    G = group or C
    return np.stack([np.maximum(np.abs(y[:, c:c + G]).max(axis=1) / E4M3_MAX, 2.0 ** -126) for c in range(0, C, G)], 1)


# ---------------------------------------------------------------------------
# Rotary positions
# ---------------------------------------------------------------------------
def rope_frequencies(rot, base=10000.0, scaling="none", factor=1.0, context=0.0, low=1.0, high=32.0):
    i = np.arange(rot // 2)
    if scaling == "ntk":
        base = base * factor ** (rot / (rot - 2))
    f = base ** (-2.0 * i / rot)
    if scaling == "linear":
        return f / factor
    if scaling == "ramp":
        turns = context * f / (2 * np.pi)
        keep = np.where(turns <= low, 0.0, np.where(turns >= high, 1.0, (turns - low) / (high - low)))
        return keep * f + (1 - keep) * f / factor
    return f


def rope(x, positions, freqs, interleaved=False, amplitude=1.0, inverse=False):
    """x [B, H, S, D] with its first 2 len(freqs) columns turned; positions [B, S]."""
    x = _f64(x)
    half = len(freqs)
    ang = _f64(positions)[:, None, :, None] * _f64(freqs) * (-1.0 if inverse else 1.0)
    c, s = amplitude * np.cos(ang), amplitude * np.sin(ang)
    a_at, b_at = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if interleaved else (slice(0, half), slice(half, 2 * half))
    out = x.copy()
    out[..., a_at] = x[..., a_at] * c - x[..., b_at] * s
    out[..., b_at] = x[..., b_at] * c + x[..., a_at] * s
    return out


def cache_slots(length, cap, window=0, sinks=0, rolling=False):
    """{position: slot} of what a cache holds of a sequence of `length` tokens."""
    if not rolling:
        return {p: p for p in range(min(length, cap))}
    held = [p for p in range(length) if p < sinks or p >= length - window]
    return {p: p if p < sinks else sinks + (p - sinks) % window for p in held}


# ---------------------------------------------------------------------------
# Sliding-window attention with sinks
# ---------------------------------------------------------------------------
def visible(n, window, sinks):
    """[n, n] truth values: query i sees key j."""
    i, j = np.arange(n)[:, None], np.arange(n)[None]
    return (j <= i) & ((i - j < window) | (j < sinks))


def _probabilities(q, k, scale, keep):
    z = np.where(keep, scale * (q @ k.T), -np.inf)
    m = z.max(axis=1, keepdims=True)
    e = np.exp(z - m)
    l = e.sum(axis=1, keepdims=True)
    return e / l, (m + np.log(l))[:, 0]


def swa(q, k, v, scale, window, sinks=0, lens=None, do=None):
    """Forward, and with `do` [B, Hq, S, D] the backward, of q [B, Hq, S, D] over k, v
    [B, Hkv, S, D]: a dict of o, lse (dq, dk, dv), and, for error bounds, the sums of the
    absolute values of the terms each element adds (attn_oracle.head_term_magnitudes):
    m_o, m_dv, g_dq, g_dk, h_dq, h_dk.  Rows from lens[b] on: 0, lse -inf; they are not
    looked at."""
    q, k, v = _f64(q), _f64(k), _f64(v)
    B, Hq, S, D = q.shape
    Hkv = k.shape[1]
    group = Hq // Hkv
    out = {"o": np.zeros_like(q), "lse": np.full((B, Hq, S), -np.inf), "m_o": np.zeros_like(q)}
    if do is not None:
        do = _f64(do)
        for n in ("dq", "g_dq", "h_dq"):
            out[n] = np.zeros_like(q)
        for n in ("dk", "dv", "m_dv", "g_dk", "h_dk"):
            out[n] = np.zeros_like(k)
    for b in range(B):
        n = S if lens is None else min(max(int(lens[b]), 0), S)
        if n == 0:
            continue
        keep = visible(n, window, sinks)
        for h in range(Hq):
            a = h // group
            qh, kh, vh = q[b, h, :n], k[b, a, :n], v[b, a, :n]
            p, lse = _probabilities(qh, kh, scale, keep)
            o = p @ vh
            out["o"][b, h, :n], out["lse"][b, h, :n], out["m_o"][b, h, :n] = o, lse, p @ np.abs(vh)
            if do is None:
                continue
            g = do[b, h, :n]
            ds = p * (g @ vh.T - np.sum(g * o, axis=1)[:, None])
            out["dq"][b, h, :n] = scale * (ds @ kh)
            out["dk"][b, a, :n] += scale * (ds.T @ qh)
            out["dv"][b, a, :n] += p.T @ g
            ap = np.sum(np.abs(g) * out["m_o"][b, h, :n], axis=1)[:, None] * p
            out["m_dv"][b, a, :n] += p.T @ np.abs(g)
            out["g_dq"][b, h, :n], out["h_dq"][b, h, :n] = np.abs(ds) @ np.abs(kh), ap @ np.abs(kh)
            out["g_dk"][b, a, :n] += np.abs(ds).T @ np.abs(qh)
            out["h_dk"][b, a, :n] += ap.T @ np.abs(qh)
    return out


def swa_decode(q, k_seq, v_seq, scale, window, sinks=0):
    """(o [Hq, D], lse [Hq], m_o) of the newest token's query over its sequence's keys and
    values [Hkv, n, D] (n >= 1), in position order."""
    q, k_seq, v_seq = _f64(q), _f64(k_seq), _f64(v_seq)
    n = k_seq.shape[1]
    keep = visible(n, window, sinks)[n - 1:]
    o, m_o, lse = np.empty_like(q), np.empty_like(q), np.empty(q.shape[0])
    for h in range(q.shape[0]):
        a = h // (q.shape[0] // k_seq.shape[0])
        p, l = _probabilities(q[h:h + 1], k_seq[a], scale, keep)
        o[h], lse[h], m_o[h] = p[0] @ v_seq[a], l[0], p[0] @ np.abs(v_seq[a])
    return o, lse, m_o
