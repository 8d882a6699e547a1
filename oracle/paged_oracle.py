"""Plain CPU oracle of the operators over a page pool (slow, obvious, 64-bit).

TEST INFRASTRUCTURE, as ``entmtp_oracle``: only the tests import it, and it
shares no code with the kernels.  Every function follows the definition that
``include/entmtp.h`` gives for the entry point of the same name.
"""
from __future__ import annotations

import math

import numpy as np

from oracle import entmtp_oracle as orc

OK, NONE, RANGE, FULL, BAD = range(5)
SEEN = np.int32(-2 ** 31)    # bit 31 of a history entry


def page_map(trees, topo, prefix_len, table, page, n_pages, rows_cap, free=None, n_free=0):
    """(table, row_off, slots, status, n_free): slots lists the rows [0, row_off[-1])."""
    table = table.copy()
    B, max_pages = table.shape
    n_free = min(max(int(n_free), 0), 0 if free is None else len(free))
    left, taken, end = n_free, 0, 0
    short = False              # an earlier sequence asked for more than there was
    row_off, status, slots = [0], [], []
    for b in range(B):
        named = 0 <= topo[b] < len(trees)
        T = len(trees[topo[b]]) if named else 0
        L = int(prefix_len[b])
        end += T
        st = OK if named else NONE
        if named and (end > rows_cap or L < 0 or L + T > max_pages * page):
            st = RANGE
        if st == OK:
            entries = list(range(L // page, (L + T - 1) // page + 1))
            lack = [e for e in entries if table[b, e] < 0]
            if any(table[b, e] >= n_pages for e in entries) or (L % page and entries[0] in lack):
                st = BAD
            elif lack:
                short = short or len(lack) > left
                if short:
                    st = FULL
                else:
                    ids = [int(free[left - 1 - k]) for k in range(len(lack))]
                    left -= len(lack)
                    if all(0 <= i < n_pages for i in ids):
                        table[b, lack] = ids
                    else:
                        st = BAD
        for i in range(min(end, rows_cap) - row_off[-1]):
            pos = L + i
            slots.append(int(table[b, pos // page]) * page + pos % page if st == OK else -1)
        row_off.append(min(end, rows_cap))
        status.append(st)
    return table, np.array(row_off, np.int32), np.array(slots, np.int32), np.array(status, np.int32), left


def kv_compact_paged(pool, path, accept_len, row_off, slots):
    """pool [layers, pages, Hkv, page, d] after the accepted paths moved."""
    new, page = pool.copy(), pool.shape[3]
    n_slots = pool.shape[1] * page
    for b, a in enumerate(accept_len):
        for j in range(min(int(a), path.shape[1] - 1, orc.D_MAX) + 1):
            n, node = row_off[b + 1] - row_off[b], path[b, j]
            if not (0 <= node < n and j < n):
                continue
            src, dst = slots[row_off[b] + node], slots[row_off[b] + j]
            if 0 <= src < n_slots and 0 <= dst < n_slots:
                new[:, dst // page, :, dst % page] = pool[:, src // page, :, src % page]
    return new


def history_prompt(history, tokens, tok_off):
    h, V = history.copy(), history.shape[1]
    for b in range(h.shape[0]):
        for t in tokens[tok_off[b]:tok_off[b + 1]]:
            if 0 <= t < V:
                h[b, t] |= SEEN
    return h


def history_accept(history, row_off, tok, path, accept_len, bonus):
    h, V = history.copy(), history.shape[1]
    for b, a in enumerate(accept_len):
        if a < 0:
            continue
        said = [int(bonus[b])]
        for j in range(1, min(int(a), path.shape[1] - 1, orc.D_MAX) + 1):
            if 0 <= path[b, j] < row_off[b + 1] - row_off[b]:
                said.append(int(tok[row_off[b] + path[b, j]]))
        for t in said:
            if 0 <= t < V:
                h[b, t] += 1
    return h


def adjusted_row(z, parent, node, tok, params, history, bias, allowed):
    """One row's adjusted logits in 64 bits (the tree's drafted tokens ``tok``;
    history, bias and allowed are rows of the vocabulary or None)."""
    rep, freq, pres = (float(x) for x in params[:3])
    V = z.shape[0]
    z = z.astype(np.float64)
    count = np.zeros(V) if history is None else (history & 0x7FFFFFFF).astype(np.float64)
    for k in orc.ancestors_or_self(parent, node)[1:]:
        if 0 <= tok[k] < V:
            count[tok[k]] += 1
    seen = count > 0 if history is None else (count > 0) | (history < 0)
    z = np.where(seen, np.where(z > 0, z / rep, z * rep), z)
    z = np.where(count > 0, z - freq * count - pres, z)
    if bias is not None:
        z = z + bias
    if allowed is not None:
        z = np.where(allowed, z, -np.inf)
    return z


def row_stats(z, inv_temp):
    """(entropy, top-1 probability, argmax) of a row of logits, -inf ones apart."""
    if np.isnan(z).any() or np.isposinf(z).any():
        with np.errstate(invalid="ignore"):
            best = np.nanmax(z) if not np.isnan(z).all() else -np.inf
        return math.nan, math.nan, int(np.argmax(z == best)) if best > -np.inf else -1
    if not (z > -np.inf).any():
        return 0.0, 0.0, -1
    y = z[z > -np.inf] * inv_temp
    e = np.exp(y - y.max())
    p = e / e.sum()
    return float(-(p[p > 0] * np.log(p[p > 0])).sum()), float(p.max()), int(np.argmax(z))


def tree_attention_paged(q, kt, vt, k_pool, v_pool, table, L, parent, scale, theta, softcap=0.0,
                         window=0, slopes=None):
    """One sequence: out [T, Hq, d] in 64 bits, the tree's rotated keys as bf16
    bits [T, Hkv, d], and how far roundings to bf16 can move out.  q, kt, vt,
    pools: bf16 bits; table: its pages.

    The last: a rounding to bf16 is off by at most u = 2^-8 of the value.  The
    weights and a split's partial are rounded (u sum p |v| each), so is out (u
    |out|); the rounding of a rotated or scaled query (scale in base 2 taken
    into it: u of every element, whatever the scale), and the cap's own error
    (softcap 2^-21), move a score by at most d_k = u scale
    sum |q_c k_c| (a score cap bends by at most one), all of a row's by at most
    D, and with it out by at most (e^(2 D) - 1) sum p |v - out|."""
    T, Hq, d = q.shape
    Hkv, page = k_pool.shape[1:3]
    depth = orc.depths(parent)
    n_pre = -(-L // page)
    dense = lambda pool: np.concatenate([pool[p] for p in table[:n_pre]], axis=1)[:, :L] if n_pre else \
        np.zeros((Hkv, 0, d), np.uint16)    # noqa: E731
    k_pre, v_pre = orc.bf16_to_f64(dense(k_pool)), orc.bf16_to_f64(dense(v_pool))
    qf, kf, vf = orc.bf16_to_f64(q), orc.bf16_to_f64(kt), orc.bf16_to_f64(vt)
    if theta > 0:
        qf = np.stack([orc.rope(qf[i], L + depth[i], theta) for i in range(T)])
        kf = orc.round_to_bf16(np.stack([orc.rope(kf[i], L + depth[i], theta) for i in range(T)]))
    pos = np.concatenate([np.arange(L), L + np.array(depth)])
    out, off = np.zeros((T, Hq, d)), np.zeros((T, Hq, d))
    u = 2.0 ** -8
    for i in range(T):
        see = np.concatenate([np.ones(L, bool), np.isin(np.arange(T), orc.ancestors_or_self(parent, i))])
        dist = L + depth[i] - pos
        if window:
            see &= dist < window
        for h in range(Hq):
            g = h // (Hq // Hkv)
            k, v = np.concatenate([k_pre[g], kf[:, g]])[see], np.concatenate([v_pre[g], vf[:, g]])[see]
            z = k @ qf[i, h] * scale
            if softcap:
                z = softcap * np.tanh(z / softcap)
            if slopes is not None:
                z = z - float(slopes[h]) * dist[see]
            p = np.exp(z - z.max())
            p /= p.sum()
            out[i, h] = p @ v
            D = u * scale * float((np.abs(k) @ np.abs(qf[i, h])).max()) + softcap * 2.0 ** -21
            off[i, h] = 2 * u * (p @ np.abs(v)) + u * np.abs(out[i, h]) + (math.exp(2 * D) - 1) * (p @ np.abs(v - out[i, h]))
    return out, orc.f64_to_bf16_bits(kf) if theta > 0 else kt, off
