"""Plain 64-bit implementations (numpy) of attention between all tokens and of rotary positions, with bounds of what a 32-bit
implementation on the same stored values may be off by.

TEST INFRASTRUCTURE ONLY, like the rest of this package: written from the definitions, sharing no code with the product.  Every
function takes and returns float64 arrays that hold the stored values exactly.
"""
from __future__ import annotations

import numpy as np

U = 2.0 ** -24  # half a step of fp32, relative


def _pairs(d, layout):
    c = np.arange(d // 2)
    return (2 * c, 2 * c + 1) if layout == "pairs" else (c, c + d // 2)


def rotary(x, coords, freq, layout="pairs", back=False):
    """x [B,N,H,d] turned by coords [B,N,A] . freq [d/2,A]."""
    a, b = _pairs(x.shape[-1], layout)
    t = (coords @ freq.T)[:, :, None, :] * (-1 if back else 1)
    y = np.empty_like(x)
    y[..., a] = x[..., a] * np.cos(t) - x[..., b] * np.sin(t)
    y[..., b] = x[..., a] * np.sin(t) + x[..., b] * np.cos(t)
    return y


def rotary_spin(y, dy, layout="pairs"):
    """Derivative of <dy, y> by every pair's angle, summed over heads [B,N,d/2], and the sum of its terms' absolute values."""
    a, b = _pairs(y.shape[-1], layout)
    terms = y[..., a] * dy[..., b], y[..., b] * dy[..., a]
    return (terms[0] - terms[1]).sum(2), (np.abs(terms[0]) + np.abs(terms[1])).sum(2)


def hidden(q_doc, k_doc):
    return (q_doc[:, :, None] != k_doc[:, None, :]) | (q_doc[:, :, None] < 0) | (k_doc[:, None, :] < 0)


def attn(q, k, v, scale, cap=0.0, q_xy=None, k_xy=None, slope=None, q_doc=None, k_doc=None, dout=None, half=0.0, given=None, puts_right=False):
    """out, lse and, with dout, dq, dk, dv (and dslope): name -> (values, bound).  `half`: rounding of the storage type; what a bf16
    implementation rounds on the way (p, dS) is counted with it, U stands for a type that it need not round.
    `given`: the stored output that the backward pass got, whose rounding goes into D.  `puts_right`: of an implementation that works out
    what D lacks, r = sum_j p (dP - D), and takes r sum_j p (1 - tanh^2) k_j off dq and gives D + r to dk: then what `given` was rounded by
    is left only where dS and p were rounded for dq's two products, at `on_way` each."""
    B, Nq, H, d = q.shape
    Nk, Hk = k.shape[1:3]
    G = H // Hk
    on_way = half if half > U else 0.0
    r = {n: (np.zeros(s), np.zeros(s)) for n, s in (("out", q.shape), ("lse", (B, Nq, H)))}
    if dout is not None:
        r.update({n: (np.zeros(s), np.zeros(s)) for n, s in (("dq", q.shape), ("dk", k.shape), ("dv", v.shape))})
        if slope is not None:
            r["dslope"] = (np.zeros(H), np.zeros(H))
    out_of = hidden(q_doc, k_doc) if q_doc is not None else np.zeros((B, Nq, Nk), dtype=bool)
    n_sum = 2 * U * (Nk + 16)
    for b in range(B):
        # padding may hold anything
        qb, kb, vb = (np.where(np.asarray(doc)[b][:, None, None] < 0, 0.0, x[b]) if doc is not None else x[b] for x, doc in ((q, q_doc), (k, k_doc), (v, k_doc)))
        gone = out_of[b]
        dist = None
        if slope is not None:
            xy = [np.where(doc[b][:, None] < 0, 0.0, c[b]) if doc is not None else c[b] for c, doc in ((q_xy, q_doc), (k_xy, k_doc))]
            dist = np.sqrt(((xy[0][:, None] - xy[1][None]) ** 2).sum(-1))
        for h in range(H):
            Q, K, V = qb[:, h], kb[:, h // G], vb[:, h // G]
            z = scale * (Q @ K.T)
            off = 2 * U * (d + 6) * abs(scale) * (np.abs(Q) @ np.abs(K).T) + 4 * U * np.abs(z)
            bend = None
            if cap:
                bend = np.tanh(z / cap)
                bend_off = off / cap + 8 * U
                z = cap * bend
                off = off + 8 * U * cap
            if slope is not None:
                z = z - slope[h] * dist
                off = off + 8 * U * abs(slope[h]) * dist
            off = off + 4 * U * np.abs(z)
            zm = np.where(gone, -np.inf, z)
            top = zm.max(1)
            sees = top > -np.inf
            top = np.where(sees, top, 0.0)
            e = np.where(gone, 0.0, np.exp(zm - top[:, None]))
            total = e.sum(1)
            p = e / np.where(sees, total, 1.0)[:, None]
            lse = np.where(sees, top + np.log(np.where(sees, total, 1.0)), -np.inf)
            # a score's error and the largest one of its row, the exponent's rounding and the sum
            worst = np.where(gone, 0.0, off).max(1)
            flat = np.where(sees, lse, 0.0)
            eps = off + worst[:, None] + n_sum + 8 * U * (1 + np.abs(z - flat[:, None]) + np.abs(flat)[:, None])
            out = p @ V
            tol = (p * (eps + on_way + n_sum)) @ np.abs(V)
            tol = tol + max(half, U) * (np.abs(out) + tol)
            r["out"][0][b, :, h], r["out"][1][b, :, h] = out, tol
            r["lse"][0][b, :, h], r["lse"][1][b, :, h] = lse, worst + n_sum + 8 * U * (1 + np.abs(flat))
            if dout is None:
                continue
            g = dout[b, :, h] if q_doc is None else np.where(q_doc[b][:, None] < 0, 0.0, dout[b, :, h])
            dP = g @ V.T
            dP_off = 2 * U * (d + 6) * (np.abs(g) @ np.abs(V).T)
            D = (g * out).sum(1)
            stored = tol if given is None else np.abs(np.where(sees[:, None], given[b, :, h], 0.0) - out)
            D_off = (np.abs(g) * stored).sum(1) + 2 * U * (d + 6) * (np.abs(g) * np.abs(out)).sum(1)
            dZ = p * (dP - D[:, None])
            pair_off = (eps + 4 * U) * np.abs(dP - D[:, None]) + dP_off
            gap = np.zeros(Nq)
            if puts_right:
                # with D - gap for D a row's dZ sum to gap (1 + a row's error of sum p) and the sum of what their own are off by
                if given is not None:
                    gap = np.abs((g * np.where(sees[:, None], given[b, :, h] - out, 0.0)).sum(1)) + 2 * U * (d + 6) * (np.abs(g) * np.abs(out)).sum(1)
                gap_sum = n_sum * (p * (np.abs(dP - D[:, None]) + gap[:, None])).sum(1) + (np.where(gone, 0.0, eps).max(1) + 4 * U) * gap + 4 * U * np.abs(D)
                dZ_off = p * (pair_off + ((p * pair_off).sum(1) + gap_sum + 4 * U * gap)[:, None])
            else:
                dZ_off = p * (pair_off + D_off[:, None])
            if slope is not None:
                r["dslope"][0][h] -= (dZ * dist).sum()
                # D enters as the sum of p dP, so its storage's rounding does not: only the sums that put it right
                once = p * (2 * (eps + 4 * U) * (np.abs(dP) + np.abs(D)[:, None]) + 2 * dP_off)
                sums = 2 * U * (Nk + Nq * B // 512 + 32) * (np.abs(dZ) + p * D_off[:, None])
                r["dslope"][1][h] += ((once + sums) * dist).sum() + ((once + sums).sum(1) * (p * dist).sum(1)).sum()
            dS, dS_off = dZ, dZ_off
            if cap:
                dS = dZ * (1 - bend ** 2)
                dS_off = dZ_off + np.abs(dZ) * (2 * np.abs(bend) * bend_off + bend_off ** 2 + 4 * U)
            dS_off = dS_off + on_way * (np.abs(dS) + dS_off)
            dq = scale * (dS @ K)
            twice = 2 * (on_way + n_sum + 4 * U) * p * gap[:, None]  # in dS and in p times what D lacks
            dq_off = abs(scale) * ((dS_off + twice + n_sum * np.abs(dS)) @ np.abs(K))
            r["dq"][0][b, :, h], r["dq"][1][b, :, h] = dq, dq_off + max(half, U) * (np.abs(dq) + dq_off) + 4 * U * np.abs(dq)
            r_sum = 2 * U * (Nq * G + 16)
            p_off = p * (eps + on_way)
            for name, w, w_off, x, f in (("dk", dS, dS_off, Q, scale), ("dv", p, p_off, g, 1.0)):
                r[name][0][b, :, h // G] += f * (w.T @ x)
                r[name][1][b, :, h // G] += abs(f) * ((w_off + r_sum * np.abs(w)).T @ np.abs(x))
    if dout is not None:
        for name in ("dk", "dv"):
            x, tol = r[name]
            r[name] = (x, tol + max(half, U) * (np.abs(x) + tol) + 4 * U * np.abs(x))
    return r
