"""fp64 CPU oracle of attention with modified scores, from the definition, row by row over tokens (no blocks, no tables):

    z = scale q.k;  y = cap tanh(z / cap) (cap > 0);  s = y - slope_h |pos_i - pos_j|;  softmax over the visible keys of a row

and its gradient.  Beside every result stands a bound on what an implementation may be off that keeps P and dS as bf16 operands
and everything else in fp32: a bf16 rounding is off by at most HALF = 2^-8 of the value, an exponent x in fp32 by 2^-22 |x| or so.
Bounds are an element's own: keys that have no weight in a row loosen none of its."""
from __future__ import annotations

import numpy as np

HALF = 2.0 ** -8        # half a step of bf16


def layout(seq_lens, block, mask="causal", cut=None, owned=None):
    """Token tables of a plan's buffers: (q_seq, q_pos, kv_seq, kv_pos), int arrays.  Blocks end at multiples of `block` from a
    sequence's start and, with `cut`, at the cut and at multiples of `block` from it; owned: (seq, idx) rows."""
    q_seq, q_pos, kv_seq, kv_pos = [], [], [], []
    keep = None if owned is None else {(int(s), int(i)) for s, i in owned}
    for s, n in enumerate(seq_lens):
        c = 0 if cut is None else int(cut[s])
        starts = list(range(0, c, block)) + list(range(c, int(n), block))
        kv_seq += [s] * int(n)
        kv_pos += range(int(n))
        for i, a in enumerate(starts):
            b = starts[i + 1] if i + 1 < len(starts) else int(n)
            if keep is None or (s, i) in keep:
                q_seq += [s] * (b - a)
                q_pos += range(a, b)
    return tuple(np.asarray(x, dtype=np.int64) for x in (q_seq, q_pos, kv_seq, kv_pos))


def visible(q_seq, q_pos, kv_seq, kv_pos, mask="causal", cut=None):
    """bool [T_q, T_kv]; mask: "causal", "full" or "prefix" (tokens before cut[seq] are seen by the whole sequence)."""
    same = q_seq[:, None] == kv_seq[None]
    if mask == "full":
        return same
    see = kv_pos[None] <= q_pos[:, None]
    if mask == "prefix":
        see = see | (kv_pos < np.asarray(cut, dtype=np.int64)[kv_seq])[None]
    return same & see


def attention(q, k, v, see, dist, cap=0.0, slopes=None, scale=None, d_o=None, o_bf16=False, grad_bf16=False):
    """q, d_o [T_q, Hq, d], k, v [T_kv, Hkv, d] fp64; see, dist [T_q, T_kv].  Returns dict name -> (value, bound)."""
    t_q, hq, d = q.shape
    t_kv, hkv = k.shape[:2]
    group = hq // hkv
    scale = 1.0 / np.sqrt(d) if scale is None else scale
    o, eo, lse, el = np.zeros_like(q), np.zeros_like(q), np.full((t_q, hq), -np.inf), np.zeros((t_q, hq))
    g = {n: (np.zeros_like(x), np.zeros_like(x)) for n, x in (("dq", q), ("dk", k), ("dv", v))}
    for h in range(hq):
        kh, vh, qh = k[:, h // group], v[:, h // group], q[:, h]
        z = qh @ kh.T * scale
        t = np.tanh(z / cap) if cap else np.zeros_like(z)
        s = cap * t if cap else z
        big = np.abs(qh) @ np.abs(kh).T * scale         # of the terms that fp32 sums up to z
        if slopes is not None:
            b = float(np.float32(slopes[h])) * dist
            s, big = s - b, big + b
        s = np.where(see, s, -np.inf)
        with np.errstate(invalid="ignore", divide="ignore"):
            top = s.max(1) if t_kv else np.full(t_q, -np.inf)
            p = np.where(see, np.exp(s - np.where(np.isfinite(top), top, 0)[:, None]), 0.0)
            tot = p.sum(1)
            lse[:, h] = np.where(tot > 0, np.log(tot) + top, -np.inf)
            p = np.where(tot[:, None] > 0, p / np.where(tot > 0, tot, 1)[:, None], 0.0)
        # What fp32 does to the exponent of an element, as a relative error of its P: sums and products of this size, the LSE that is taken off, and
        # a bias that is formed along the 64 columns of a tile, 64 slopes from their first to their last.
        fin = np.where(np.isfinite(lse[:, h]), lse[:, h], 0)
        ex = 2.0 ** -20 + 2.0 ** -21 * (big + 2 * cap + np.abs(fin)[:, None]) + (2.0 ** -17 * float(np.float32(slopes[h])) if slopes is not None else 0.0)
        r = HALF + ex
        pr = p * r
        o[:, h] = p @ vh
        # Every P_j V_j carries a rounding (1 + r_j), |r_j| <= r.  Divided by the sum of P as it is, O is off by |sum P_j r_j V_j|
        # <= (P r)|V|.  Divided by the sum of the rounded P it is sum P_j (1 + r_j) V_j / sum P_j (1 + r_j), off by
        # |sum P_j r_j (V_j - O)| / |1 + sum P_j r_j| <= ((P r)|V| + sum(P r)|O|) / (1 - sum(P r)), the larger one.
        all_r = pr.sum(1)[:, None]
        eo[:, h] = (pr @ np.abs(vh) + all_r * np.abs(o[:, h])) / (1 - all_r) + (HALF * np.abs(o[:, h]) if o_bf16 else 0)
        el[:, h] = (p * ex).sum(1) + 2.0 ** -21 * np.abs(fin)
        if d_o is None:
            continue
        do = d_o[:, h]
        dp, dsum = do @ vh.T, (do * o[:, h]).sum(1)
        f = (1 - t * t) * scale if cap else np.full_like(z, scale)
        ds = p * (dp - dsum[:, None]) * f
        # P is formed anew, against the LSE that was stored; D comes from the O that was stored; dP and D are sums in fp32
        r = r + el[:, h][:, None]
        pr = p * r
        e_d = (np.abs(do) * eo[:, h]).sum(1)
        e_ds = r * np.abs(ds) + p * f * (e_d[:, None] + 2.0 ** -18 * (np.abs(do) @ np.abs(vh).T))
        if cap:
            e_ds += p * np.abs(dp - dsum[:, None]) * scale * 2.0 ** -20          # 1 - tanh^2 in absolute terms
        for name, val, err in (("dq", ds @ kh, e_ds @ np.abs(kh)),):
            g[name][0][:, h] += val
            g[name][1][:, h] += err
        for name, val, err in (("dk", ds.T @ qh, e_ds.T @ np.abs(qh)), ("dv", p.T @ do, pr.T @ np.abs(do))):
            g[name][0][:, h // group] += val
            g[name][1][:, h // group] += err
    out = {"o": (o, eo + 1e-7), "lse": (lse, el)}
    if d_o is not None:
        for name, (val, err) in g.items():
            out[name] = (val, err + 1e-7 + (HALF * np.abs(val) if grad_bf16 else 0))
    return out
