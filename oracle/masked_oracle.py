"""Plain fp64 statement of masked attention, its gradients, and attention over a paged cache.

Test infrastructure only, written from the definitions: which keys a row sees is decided pair by pair, from the
documents' borders.  Beside each result stands what bounds a kernel's distance to it: the sums of absolute terms that
roundings of the weights, of the scores' gradients and of the forward pass's output are multiplied by.
"""
from __future__ import annotations

import numpy as np


def visible(batch, q_len, kv_len, causal=False, doc_offsets=None, prefix=None):
    """Truth values [batch, q_len, kv_len]."""
    pos = np.arange(q_len) + kv_len - q_len
    key = np.arange(kv_len)
    see = np.zeros((batch, q_len, kv_len), bool)
    for b in range(batch):
        borders = [(0, kv_len)] if doc_offsets is None else list(zip(doc_offsets[b][:-1], doc_offsets[b][1:]))
        for c, (first, end) in enumerate(borders):
            rows = np.ones(q_len, bool) if doc_offsets is None else (pos >= first) & (pos < end)
            keys = (key >= first) & (key < end)
            pair = rows[:, None] & keys[None, :]
            if causal:
                ahead = 0 if prefix is None else max(0, int(prefix[b][c]))
                pair &= (key[None, :] <= pos[:, None]) | (key[None, :] < first + ahead)
            see[b] |= pair
    return see


def scores(q, k, scale, softcap=0.0, slope=None, pos=None):
    """(z, dz/ds) of one head: q [n, d], k [m, d]."""
    s = (q @ k.T) * scale
    gain = np.ones_like(s)
    if softcap:
        t = np.tanh(s / softcap)
        s, gain = softcap * t, 1 - t * t
    if slope is not None:
        s = s - slope * np.abs(pos[:, None] - np.arange(k.shape[0])[None, :])
    return s, gain


def softmax_rows(z, see):
    """(p, lse) over the seen keys; rows that see none: p = 0, lse = -inf."""
    z = np.where(see, z, -np.inf)
    top = z.max(axis=1, keepdims=True) if z.shape[1] else np.full((z.shape[0], 1), -np.inf)
    top0 = np.where(np.isfinite(top), top, 0.0)
    e = np.where(see, np.exp(z - top0), 0.0)
    total = e.sum(axis=1, keepdims=True)
    with np.errstate(divide="ignore"):
        lse = (top0 + np.log(total))[:, 0]
    return e / np.where(total == 0, 1.0, total), lse


def attention(q, k, v, see, scale, softcap=0.0, slopes=None, dout=None):
    """q [b, h, n, d], k, v [b, kvh, m, d] (fp64), see [b, n, m].  Returns a dict: out, lse, and `mass` = sum p |v|;
    with dout also dq, dk, dv and the sums their bounds are made of (see `gradient_bounds`)."""
    b, h, n, d = q.shape
    kvh, m = k.shape[1], k.shape[2]
    pos = np.arange(n) + m - n
    res = {x: np.zeros(q.shape) for x in ("out", "mass")}
    res["lse"] = np.full((b, h, n), -np.inf)
    res["zmax"] = 0.0
    if dout is not None:
        for x in ("dq", "dq_mass", "dq_weight"):
            res[x] = np.zeros(q.shape)
        for x in ("dk", "dv", "dk_mass", "dv_mass", "dk_weight"):
            res[x] = np.zeros(k.shape)
        res["weight_max"] = 0.0
    for i in range(b):
        for j in range(h):
            g = j // (h // kvh)
            K, V, Q = k[i, g], v[i, g], q[i, j]
            z, gain = scores(Q, K, scale, softcap, None if slopes is None else slopes[j], pos)
            p, lse = softmax_rows(z, see[i])
            Vs = np.where(see[i].any(0)[:, None], V, 0.0)      # values that no row sees may be anything
            res["out"][i, j], res["lse"][i, j], res["mass"][i, j] = p @ Vs, lse, p @ np.abs(Vs)
            if see[i].any():
                res["zmax"] = max(res["zmax"], float(np.abs(z[see[i]]).max()), float((np.abs(Q) @ np.abs(K).T)[see[i]].max() * scale))
            if dout is None:
                continue
            rows = see[i].any(1)[:, None]
            G, Qs = np.where(rows, dout[i, j], 0.0), np.where(rows, Q, 0.0)
            Ks = np.where(see[i].any(0)[:, None], K, 0.0)
            dp = G @ Vs.T
            delta = (G * res["out"][i, j]).sum(1, keepdims=True)
            ds = p * (dp - delta) * gain
            res["dq"][i, j] = scale * (ds @ Ks)
            res["dk"][i, g] += scale * (ds.T @ Qs)
            res["dv"][i, g] += p.T @ G
            res["dq_mass"][i, j] = scale * (np.abs(ds) @ np.abs(Ks))
            res["dk_mass"][i, g] += scale * (np.abs(ds).T @ np.abs(Qs))
            res["dv_mass"][i, g] += p.T @ np.abs(G)
            # |terms| that an error of p, dp or delta of relative size 1 would be multiplied by
            size = (np.abs(G) @ np.abs(Vs).T + np.abs(G * res["out"][i, j]).sum(1, keepdims=True)) * p * gain
            res["dq_weight"][i, j] = scale * (size @ np.abs(Ks))
            res["dk_weight"][i, g] += scale * (size.T @ np.abs(Qs))
            # delta is made from the stored out: its error is |dout| . |error of out|
            res.setdefault("delta_terms", []).append((i, j, g, np.abs(G), p * gain, np.abs(Ks), np.abs(Qs)))
    return res


def forward_bounds(res, eps, n_terms):
    """How far a kernel's out may be off: its weights rounded to the type (eps / 2 relative, of which sums of p |v|
    remain), out rounded once, and in fp32 n_terms roundings of 2^-24 in the scores (each of the size of the largest
    score), the weights and the sums."""
    f32 = 2.0 ** -24 * n_terms * (1 + res["zmax"])
    half = eps / 2
    return half * 1.01 * (res["mass"] + np.abs(res["out"])) + f32 * res["mass"] + 1e-30


def gradient_bounds(res, eps, n_terms, scale):
    """The same for dq, dk, dv: ds (or p) rounded to the type, the result rounded once, delta from a rounded out, fp32."""
    half = eps / 2 * 1.01
    f32 = 2.0 ** -24 * n_terms * (1 + res["zmax"])
    out_err = forward_bounds(res, eps, n_terms)
    b = {"dq": half * (res["dq_mass"] + np.abs(res["dq"])) + f32 * res["dq_weight"],
         "dk": half * (res["dk_mass"] + np.abs(res["dk"])) + f32 * res["dk_weight"],
         "dv": half * (res["dv_mass"] + np.abs(res["dv"])) + f32 * res["dv_mass"]}
    for i, j, g, G, pg, K, Q in res["delta_terms"]:
        e = pg * (G * out_err[i, j]).sum(1, keepdims=True)
        b["dq"][i, j] += scale * (e @ K)
        b["dk"][i, g] += scale * (e.T @ Q)
    return {x: y * 1.01 + 1e-30 for x, y in b.items()}
