"""fp64 CPU oracle of the operators on a target's top logits and of the logits
processing.

TEST INFRASTRUCTURE ONLY, as ``aal_oracle``: a plain, literal transcription of
the definitions in ``include/aal.h``, sharing no code with the HIP library.
Pinned by ``tests/test_oracle_toplist.py`` against sorting in Python, finite
differences, hand-computed cases and the full-vocabulary oracle.
"""
from __future__ import annotations

import math

import numpy as np

from .aal_oracle import window_length_coefficients, window_rows

__all__ = ["top_logits", "top_loss", "process_logits", "process_logits_bwd"]


def _lse(x: np.ndarray) -> float:
    m = x.max() if x.size else -math.inf
    return -math.inf if m == -math.inf else float(m + np.log(np.exp(x - m).sum()))


def _softmax(x: np.ndarray) -> np.ndarray:
    """Zeros where nothing is finite.  Not exp(x - lse): where all of x is -3e38 the lse rounds
    to it and every entry would get 1."""
    m = x.max()
    e = np.exp(x - m) if m > -math.inf else np.zeros(len(x))
    return e / e.sum() if m > -math.inf else e


def top_logits(z, k: int, T: float = 1.0):
    """(values [R, k], ids [R, k], rest [R]): larger first, lower id first among equal ones."""
    z = np.asarray(z, np.float64)
    z = z.reshape(-1, z.shape[-1])
    R, V = z.shape
    vals, ids, rest = np.empty((R, k)), np.empty((R, k), np.int64), np.empty(R)
    for r in range(R):
        order = np.lexsort((np.arange(V), -(z[r] + 0.0)))
        ids[r] = order[:k]
        vals[r] = z[r][order[:k]]
        rest[r] = _lse(z[r][np.sort(order[k:])] / T)
    return vals, ids, rest


def top_loss(z_draft, top, ids, rest, T_draft: float, T_target: float, weights, layout: int, B: int, S: int, K: int,
             grad_scale: float = 1.0):
    """The objectives against lists [R, k] with a remainder [R] (or None).

    Beside the results: `bound` [R, V], what a relative error of every q and p
    of one can change in a gradient entry, and `near` [R], the smallest
    |q / p - 1| over the row's entries (a sign of q < p within rounding of it
    may go either way)."""
    z = np.asarray(z_draft, np.float64)
    z = z.reshape(-1, z.shape[-1])
    R, V = z.shape
    top, ids = np.asarray(top, np.float64).reshape(R, -1), np.asarray(ids, np.int64).reshape(R, -1)
    w_wtv, w_eal, w_kl, w_tv = (float(x) for x in weights)
    a_tv, a_eal, kl, xstar = np.zeros(R), np.zeros(R), np.zeros(R), np.full(R, -1)
    near = np.full(R, math.inf)
    parts = []
    for r in range(R):
        ok = (ids[r] >= 0) & (ids[r] < V) & (top[r] > -math.inf)
        at, t = ids[r][ok], top[r][ok] / T_target
        tr = -math.inf if rest is None else float(np.asarray(rest, np.float64).reshape(R)[r])
        pp = _softmax(np.append(t, tr))
        p, pr = pp[:-1], float(pp[-1])
        has = pp.any()
        q = _softmax(z[r] / T_draft)
        others = np.ones(V, bool)
        others[at] = False
        qr = float(q[others].sum()) if rest is not None else 0.0
        qi = q[at]
        with np.errstate(divide="ignore", invalid="ignore"):
            terms = np.where(p > 0, p * (np.log(p) - np.log(qi)), 0.0)
            kl[r] = terms.sum() + (pr * (np.log(pr) - np.log(qr)) if pr > 0 else 0.0)
        a_tv[r] = np.minimum(p, qi).sum() + min(pr, qr)
        if len(at):
            xstar[r] = at[top[r][ok] == top[r][ok].max()].min()
            a_eal[r] = q[xstar[r]] if has else 0.0
        m, mr = qi < p, qr < pr
        Q = float(qi[m].sum()) + (qr if mr else 0.0)
        # (an empty list: all of q against all of p, where either sign of q < p gives m - Q = 0)
        pairs = np.append(qi[p > 0] / p[p > 0], qr / pr if pr > 0 and len(at) else 2.0)
        near[r] = np.abs(pairs - 1).min()
        share = pr / qr if qr > 0 else 0.0
        parts.append((at, p, q, m, mr, Q, share, has))
    win = window_rows(layout, B, S, K)
    W = len(win)
    E_tv, d_tv = window_length_coefficients(a_tv, win)
    E_eal, d_eal = window_length_coefficients(a_eal, win)
    count = np.zeros(R)
    np.add.at(count, win.reshape(-1), 1.0)
    terms = np.array([-E_tv.sum() / W if W else 0.0, -E_eal.sum() / W if W else 0.0, kl.sum() / R,
                      (count * (1 - a_tv)).sum() / (W * K) if W else 0.0])
    used = np.array([w != 0 for w in (w_wtv, w_eal, w_kl, w_tv)])
    terms = np.where(used, terms, 0.0)
    grad, bound = np.zeros((R, V)), np.zeros((R, V))
    f = grad_scale / T_draft
    for r, (at, p, q, m, mr, Q, share, has) in enumerate(parts):
        c_tv = f * (-w_wtv * d_tv[r] - w_tv * count[r] / K) / W if W else 0.0
        c_eal = f * -w_eal * d_eal[r] / W * a_eal[r] if W else 0.0
        c_kl = f * w_kl / R if has else 0.0
        grad[r] = q * (c_tv * (mr - Q) - c_eal + c_kl * (1 - share))
        grad[r][at] = q[at] * (c_tv * (m - Q) - c_eal + c_kl) - c_kl * p
        bound[r] = q * (abs(c_tv) + abs(c_eal) + abs(c_kl) * (1 + share))
        bound[r][at] += abs(c_kl) * p
        if xstar[r] >= 0:
            grad[r][xstar[r]] += c_eal
            bound[r][xstar[r]] += abs(c_eal)
    return {"loss": float((terms * (w_wtv, w_eal, w_kl, w_tv)).sum()), "terms": terms, "E_tv": E_tv, "E_eal": E_eal,
            "accept_tv": a_tv, "accept_eal": a_eal, "xstar": xstar, "kl": kl, "grad": grad, "bound": bound,
            "near": near}


def _row_rules(rules, r: int, V: int):
    """(seen [V], generated [V], bias [V], allowed [V], repetition, frequency, presence) of row r."""
    seen, times, bias, allowed = np.zeros(V, bool), np.zeros(V), np.zeros(V), np.ones(V, bool)
    get = lambda name, default: default if rules.get(name) is None else float(rules[name][r])  # noqa: E731
    if rules.get("tokens") is not None:
        tokens = list(rules["tokens"])
        h0 = min(max(int(rules["hist_start"][r]), 0), len(tokens))
        n = min(max(int(rules["hist_len"][r]), 0), len(tokens) - h0)
        prompt = 0 if rules.get("prompt_len") is None else min(max(int(rules["prompt_len"][r]), 0), n)
        for i in range(n):
            t = int(tokens[h0 + i])
            if 0 <= t < V:
                seen[t] = True
                times[t] += i >= prompt
    if rules.get("bias_offsets") is not None:
        for i in range(int(rules["bias_offsets"][r]), int(rules["bias_offsets"][r + 1])):
            t = int(rules["bias_ids"][i])
            if 0 <= t < V:
                bias[t] = float(rules["bias_values"][i])
    if rules.get("mask") is not None:
        masks = np.asarray(rules["mask"]).reshape(-1, (V + 31) // 32)
        row = rules.get("mask_row")
        m = int(row[r]) if row is not None else 0 if len(masks) == 1 else r
        if 0 <= m < len(masks):
            v = np.arange(V)
            allowed = (masks[m].astype(np.int64)[v // 32] >> (v % 32) & 1) != 0
    return seen, times, bias, allowed, get("repetition", 1.0), get("frequency", 0.0), get("presence", 0.0)


def process_logits(z, rules) -> np.ndarray:
    z = np.asarray(z, np.float64)
    out = np.empty_like(z)
    for r in range(len(z)):
        seen, times, bias, allowed, rep, freq, pres = _row_rules(rules, r, z.shape[1])
        with np.errstate(invalid="ignore"):
            x = z[r] + bias
            x = np.where(seen, np.where(x > 0, x / rep, x * rep), x)
            x = x - np.where(times > 0, freq * times + pres, 0.0)
        out[r] = np.where(allowed, x, -math.inf)
    return out


def process_logits_bwd(grad_out, z, rules) -> np.ndarray:
    z, g = np.asarray(z, np.float64), np.asarray(grad_out, np.float64)
    out = np.empty_like(g)
    for r in range(len(z)):
        seen, _, bias, allowed, rep, _, _ = _row_rules(rules, r, z.shape[1])
        d = np.where(seen, np.where(z[r] + bias > 0, g[r] / rep, g[r] * rep), g[r])
        out[r] = np.where(allowed, d, 0.0)
    return out
