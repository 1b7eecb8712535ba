"""Cross attention, its gradient and attention with a shared prefix, in numpy fp64.

Definitions only (test infrastructure; imports nothing from the library), and with
them bounds on what fp32 sums and the stated roundings may be off by.
"""
from __future__ import annotations

import numpy as np


def attend(q, k, v, scale, see=None):
    """q [n, H, d] against k, v [Hkv, len, d]; see [n, len] (None: all).  o, lse, and per row and head
    the largest scale * sum |q k| and |v| seen."""
    n, H, d = q.shape
    kv, length, _ = k.shape
    per = H // kv
    o, lse, xm, vm = np.zeros((n, H, d)), np.full((n, H), -np.inf), np.zeros((n, H)), np.zeros((n, H))
    if length == 0:
        return o, lse, xm, vm
    see = np.ones((n, length), bool) if see is None else see
    some = see.any(1)
    for h in range(H):
        kk, vv = k[h // per], v[h // per]
        x = np.where(see, scale * (q[:, h] @ kk.T), -np.inf)
        top = np.where(some, x.max(1), 0.0)
        w = np.exp(x - top[:, None])
        total = w.sum(1)
        o[:, h] = np.where(some[:, None], (w @ vv) / np.where(some, total, 1)[:, None], 0)
        lse[:, h] = np.where(some, top + np.log(np.where(some, total, 1)), -np.inf)
        xm[:, h] = np.where(see, abs(scale) * (np.abs(q[:, h]) @ np.abs(kk).T), 0).max(1)
        vm[:, h] = np.where(see[..., None], np.abs(vv)[None], 0).max((1, 2)) if n * length * d < 1 << 22 else np.abs(vv).max()
    return o, lse, xm, vm


def gradient(q, k, v, d_o, scale, unit, least):
    """d_q, d_k, d_v of one sequence and bounds on their errors.

    unit: half a step of the type relative to a value; least: half its smallest step.  A
    logit is off by d 2^-23 X (X = scale sum |q k|, sums of d products in fp32), as is
    the log sum; p by that share, then by `unit` where it is rounded; <d_o, v> by d 2^-23 of
    its absolute sum; D = <d_o, o> by that and by o's rounding."""
    n, H, d = q.shape
    kv, length, _ = k.shape
    per = H // kv
    out = [np.zeros(q.shape), np.zeros(k.shape), np.zeros(v.shape)]
    tol = [np.zeros(q.shape), np.zeros(k.shape), np.zeros(v.shape)]
    if length == 0 or n == 0:
        return out, tol
    e = d * 2.0 ** -23
    for h in range(H):
        kk, vv, qq, g = k[h // per], v[h // per], q[:, h], d_o[:, h]
        x = scale * (qq @ kk.T)
        top = x.max(1, keepdims=True)
        w = np.exp(x - top)
        p = w / w.sum(1, keepdims=True)
        o = p @ vv
        dp = g @ vv.T
        D = (g * o).sum(1, keepdims=True)
        t = p * (dp - D)
        X = abs(scale) * (np.abs(qq) @ np.abs(kk).T)
        share = 2 * e * X.max(1, keepdims=True) + 2.0 ** -20 * (1 + np.abs(top) + np.log(length))
        p_off = p * (share + unit) + least
        # what enters t: fp32 p, dp, D with o off by its own share and rounding
        vmax = np.abs(vv).max()
        o_off = unit * np.abs(o) + (share + unit + 2.0 ** -16) * vmax
        d_off = (np.abs(g) * o_off).sum(1, keepdims=True) + e * (np.abs(g) * np.abs(o)).sum(1, keepdims=True)
        dp_off = e * (np.abs(g) @ np.abs(vv).T)
        t_off = p * (share + 2.0 ** -20) * np.abs(dp - D) + p * (1 + share) * (d_off + dp_off)
        t_off = t_off + unit * (np.abs(t) + t_off) + least
        out[0][:, h] = scale * (t @ kk)
        tol[0][:, h] = abs(scale) * (t_off @ np.abs(kk) + 2.0 ** -16 * (np.abs(t) @ np.abs(kk)))
        out[1][h // per] += scale * (t.T @ qq)
        tol[1][h // per] += abs(scale) * (t_off.T @ np.abs(qq) + 2.0 ** -16 * (np.abs(t).T @ np.abs(qq)))
        out[2][h // per] += p.T @ g
        tol[2][h // per] += p_off.T @ np.abs(g) + 2.0 ** -16 * (p.T @ np.abs(g))
    for i in range(3):
        tol[i] += unit * (np.abs(out[i]) + tol[i]) + least
    return out, tol


def gradient_norms(q, k, v, d_o, scale, unit, least, of_d=None, exact=False):
    """d_q, d_k, d_v of one sequence, and for each KV head what the norm of their errors may be.

    Every rounding is taken as an error of its own, evenly spread over half a step (`unit` of the value, `least`
    at the bottom of the type): its variance is a third of its square, and the squares add up.  t and p
    are rounded before the products over them (of t in d_q, what all of a row's t lose together is put back: its
    part along the row's mean key is gone), then the results.  fp32 sums are off by `d` 2^-24 of their absolute
    sums, far less.  The norm of independent errors lies close to the root of their variance; 2.5 times that is
    past any one error's largest size (3^0.5 of it), and a gradient with a term left out is beyond it.

    of_d: D = <d_o, o> of [n, H] to be used instead (mistakes to be refused).  exact: every partial sum of a
    logit fits fp32."""
    n, H, d = q.shape
    kv, length, _ = k.shape
    per = H // kv
    out = [np.zeros(q.shape), np.zeros(k.shape), np.zeros(v.shape)]
    var = np.zeros((3, kv))
    for h in range(H if length and n else 0):
        kk, vv, qq, g = k[h // per], v[h // per], q[:, h], d_o[:, h]
        x = scale * (qq @ kk.T)
        w = np.exp(x - x.max(1, keepdims=True))
        p = w / w.sum(1, keepdims=True)
        D = (g * (p @ vv)).sum(1, keepdims=True) if of_d is None else of_d[:, h, None]
        dp = g @ vv.T
        t = p * (dp - D)
        # of a logit, the weight's share; 2^-15: the log-sum-exp's up to 2^9
        off = 2.0 ** -15 + (0 if exact else abs(scale) * np.sqrt(d) * 2.0 ** -23 * (np.abs(qq) @ np.abs(kk).T))
        t_var = (unit * t) ** 2 / 3 + least ** 2 / 3 + (off * t) ** 2 + (p * d * 2.0 ** -23) ** 2 * (g * g).sum(1, keepdims=True) * (vv * vv).sum(1)
        p_var = (unit * p) ** 2 / 3 + least ** 2 / 3 + (off * p) ** 2
        far = (kk * kk).sum(1) - 2 * (p @ kk) @ kk.T + ((p @ kk) ** 2).sum(1, keepdims=True)      # |k_j - mean k|^2
        out[0][:, h] = scale * (t @ kk)
        out[1][h // per] += scale * (t.T @ qq)
        out[2][h // per] += p.T @ g
        var[0, h // per] += scale ** 2 * (t_var * np.maximum(far, 0)).sum()
        var[1, h // per] += scale ** 2 * (t_var * (qq * qq).sum(1, keepdims=True)).sum()
        var[2, h // per] += (p_var * (g * g).sum(1, keepdims=True)).sum()
    heads = [out[0].reshape(n, kv, per, d).transpose(1, 0, 2, 3), out[1], out[2]]
    for i in range(3):
        for h in range(kv):
            var[i, h] += unit ** 2 / 3 * (heads[i][h] ** 2).sum() + least ** 2 / 3 * heads[i][h].size
    return out, 2.5 * np.sqrt(var)
