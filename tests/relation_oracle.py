"""The relation head's operators in 64 bits (numpy), from their definitions: attention
among boxes with its gradients, the 8-bit memory, the gated norms.  Only the decisions that
the definitions make in binary32 (buckets, codes) are taken in binary32.

Besides the results, `attn` returns sums of absolute contributions, from which the tests
derive how far a result in fewer bits may be off.
"""
from __future__ import annotations

import numpy as np

F = np.float32


def axis_buckets(cq, ck, side, n, first_exp, steps):
    """[Nq, Nk] signed buckets of one axis by counting the edges that |r| has reached."""
    with np.errstate(all="ignore"):
        inv = F(1) / np.fmax(side, F(1))
        r = ((ck[None, :] - cq[:, None]).astype(F) * inv[:, None]).astype(F)
        m = np.zeros(r.shape, dtype=np.int64)
        for i in range(n):
            edge = F(2.0 ** (first_exp + i // steps) * (1.0 + (i % steps) / steps))
            m += ~(np.abs(r) < edge)              # not a number: every edge
        return np.where(r < 0, -m, m)


def buckets(qb, kb, nb, first_exp, steps):
    """[Nq, Nk] index into the nb x nb table of one image's boxes [N, 4] (binary32)."""
    n = (nb - 1) // 2
    qb, kb = qb.astype(F), kb.astype(F)
    with np.errstate(all="ignore"):
        c = [((b[:, i] + b[:, i + 2]).astype(F) * F(0.5)) for b in (qb, kb) for i in (0, 1)]
        side = [(qb[:, i + 2] - qb[:, i]).astype(F) for i in (0, 1)]
    bx = axis_buckets(c[0], c[2], side[0], n, first_exp, steps)
    by = axis_buckets(c[1], c[3], side[1], n, first_exp, steps)
    return (by + n) * nb + bx + n


def attn(q, k, v, scale, idx=None, bias=None, q_len=None, k_len=None, k_mask=None, g=None):
    """q [B, Nq, H, D], k, v [B, Nk, Hkv, D] float64; idx [B, Nq, Nk]; bias [H, nb * nb].
    Returns a dict: out, lse, and with g grad_q, grad_k, grad_v, grad_bias; and for each
    result r (lse excepted) r + "_abs" (the same sums over absolute values: of ds, of p) and
    r + "_big" (with |ds| replaced by p (|dp| + sum p |dp|), what ds is a difference of), and
    "logit": the largest sum of absolute contributions to a logit."""
    B, nq, H, D = q.shape
    nk, hkv = k.shape[1], k.shape[2]
    group = H // hkv
    r = {"out": np.zeros(q.shape), "lse": np.full((B, H, nq), -np.inf), "logit": 0.0}
    names = ["out"]
    if g is not None:
        r.update(grad_q=np.zeros(q.shape), grad_k=np.zeros(k.shape), grad_v=np.zeros(k.shape))
        names += ["grad_q", "grad_k", "grad_v"]
        if bias is not None:
            r["grad_bias"] = np.zeros(bias.shape)
            names.append("grad_bias")
    for n in names:
        for s in ("_abs", "_big"):
            r[n + s] = np.zeros(r[n].shape)
    for b in range(B):
        ql = nq if q_len is None else int(np.clip(q_len[b], 0, nq))
        kl = nk if k_len is None else int(np.clip(k_len[b], 0, nk))
        keep = np.arange(nk) < kl
        if k_mask is not None:
            keep &= k_mask[b] != 0
        cols = np.nonzero(keep)[0]
        if ql == 0 or cols.size == 0:
            continue
        for h in range(H):
            ki, vi, qi = k[b, cols, h // group], v[b, cols, h // group], q[b, :ql, h]
            s = scale * (qi @ ki.T)
            r["logit"] = max(r["logit"], float((abs(scale) * (np.abs(qi) @ np.abs(ki).T)).max()))
            if bias is not None:
                at = idx[b][:ql][:, cols]
                s = s + bias[h][at]
                fin = bias[h][np.isfinite(bias[h])]
                if fin.size:
                    r["logit"] = max(r["logit"], float(np.abs(fin).max()))
            top = s.max(1, keepdims=True)
            ref = np.where(np.isfinite(top), top, 0.0)
            p = np.exp(s - ref)
            tot = p.sum(1, keepdims=True)
            with np.errstate(divide="ignore"):
                r["lse"][b, h, :ql] = (ref + np.log(tot))[:, 0]
            p = p / np.where(tot == 0, 1.0, tot)
            o = p @ vi
            r["out"][b, :ql, h] = o
            r["out_abs"][b, :ql, h] = r["out_big"][b, :ql, h] = p @ np.abs(vi)
            if g is None:
                continue
            gi = g[b, :ql, h]
            dp = gi @ vi.T
            big = np.abs(gi) @ np.abs(vi).T
            ds = p * (dp - (p * dp).sum(1, keepdims=True))
            dsb = p * (big + (p * big).sum(1, keepdims=True))
            for name, w, wa, wb in (("", ds, np.abs(ds), dsb),):
                r["grad_q"][b, :ql, h] = scale * (w @ ki)
                r["grad_q_abs"][b, :ql, h] = abs(scale) * (wa @ np.abs(ki))
                r["grad_q_big"][b, :ql, h] = abs(scale) * (wb @ np.abs(ki))
                r["grad_k"][b, cols, h // group] += scale * (w.T @ qi)
                r["grad_k_abs"][b, cols, h // group] += abs(scale) * (wa.T @ np.abs(qi))
                r["grad_k_big"][b, cols, h // group] += abs(scale) * (wb.T @ np.abs(qi))
            r["grad_v"][b, cols, h // group] += p.T @ gi
            r["grad_v_abs"][b, cols, h // group] += p.T @ np.abs(gi)
            r["grad_v_big"][b, cols, h // group] += p.T @ np.abs(gi)
            if bias is not None:
                nb = bias.shape[1]
                r["grad_bias"][h] += np.bincount(at.ravel(), ds.ravel(), nb)
                r["grad_bias_abs"][h] += np.bincount(at.ravel(), np.abs(ds).ravel(), nb)
                r["grad_bias_big"][h] += np.bincount(at.ravel(), dsb.ravel(), nb)
    return r


def encode(x):
    """Codes (int8) and scales (binary32) of x [..., D] (binary32 values)."""
    x = np.asarray(x, dtype=F)
    with np.errstate(all="ignore"):
        a = np.where(np.isfinite(x), np.abs(x), F(0)).max(-1)
        scale = (a / F(127)).astype(F)
        q = np.clip(np.rint((x / scale[..., None]).astype(F)), -127, 127)
        q = np.where(np.isnan(x) | (scale[..., None] == 0), 0, q)
    return q.astype(np.int8), scale


def norm(x, branch, gate, alpha, w1, c1, w2, c2, layer, eps, gy=None, gu=None):
    """The gated norms and (with gy or gu) their gradients by the formulas, float64.
    gate: [rows, channels] or None.  Returns a dict."""
    C = x.shape[1]

    def n(t, w, c):
        t = t - t.mean(1, keepdims=True) if layer else t
        rstd = 1.0 / np.sqrt((t * t).mean(1, keepdims=True) + eps)
        return t * rstd, rstd, t * rstd * w + c

    def back(g, hat, rstd, w):
        g = g * w
        t = g - hat * (g * hat).mean(1, keepdims=True)
        if layer:
            t = t - g.mean(1, keepdims=True)
        return rstd * t

    one, zero = np.ones(C), np.zeros(C)
    w1, w2 = (one if w is None else w for w in (w1, w2))
    c1, c2 = (zero if c is None else c for c in (c1, c2))
    gt = 1.0 if gate is None else gate
    y = x
    if branch is not None:
        hat1, rstd1, z = n(branch, w1, c1)
        y = x + alpha * gt * z
    hat2, rstd2, u = n(y, w2, c2)
    r = {"y": y, "u": u}
    if gy is None and gu is None:
        return r
    t = np.zeros_like(x) if gy is None else gy
    if gu is not None:
        t = t + back(gu, hat2, rstd2, w2)
        r["pre_weight"], r["pre_bias"] = (gu * hat2).sum(0), gu.sum(0)
    else:
        r["pre_weight"], r["pre_bias"] = zero, zero
    r["x"] = t
    if branch is not None:
        gz = alpha * gt * t
        r["branch"] = back(gz, hat1, rstd1, w1)
        r["gate"] = alpha * t * z
        r["post_weight"], r["post_bias"] = (gz * hat1).sum(0), gz.sum(0)
    return r
