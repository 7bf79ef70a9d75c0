"""The verification of drafted tokens in 64 bits and plain Python (test infrastructure only): attention of a tree of nodes
over paged, un-rotated K/V, the tables of a step's new tokens, the move of a kept path."""
from __future__ import annotations

import numpy as np

E4M3_MAX = 448.0


def path_of(parents, j):
    """The node numbers from node j up to its root; a parent that does not precede its node makes the node a root."""
    path = []
    while j >= 0:
        path.append(j)
        p = int(parents[j])
        j = p if 0 <= p < j else -1
    return path


def _rotate(x, pos, theta, interleaved):
    """x [n, H, D] float64 at positions pos [n]."""
    D = x.shape[-1]
    z = np.exp(1j * np.asarray(pos, dtype=np.float64)[:, None, None] * theta ** (-2.0 * np.arange(D // 2) / D))
    re, im = (x[..., 0::2], x[..., 1::2]) if interleaved else (x[..., : D // 2], x[..., D // 2:])
    w = (re + 1j * im) * z
    out = np.empty_like(x)
    if interleaved:
        out[..., 0::2], out[..., 1::2] = w.real, w.imag
    else:
        out[..., : D // 2], out[..., D // 2:] = w.real, w.imag
    return out


def _lengths(x, interleaved):
    """The length of each rotary pair of x [..., D]."""
    D = x.shape[-1]
    a, b = (x[..., 0::2], x[..., 1::2]) if interleaved else (x[..., : D // 2], x[..., D // 2:])
    return np.sqrt(a * a + b * b)


def tree_attention(q, k_pages, v_pages, block_tables, kv_lens, q_positions, cu_q_lens, parents, *, theta, k_scales=None, v_scales=None,
                   block_positions=None, block_valid_mask=None, sm_scale=0.0, interleaved=False):
    """q [n, Hq, D], k_pages [N, Hkv, D/X, P, X], v_pages [N, Hkv, D, P] in float64. parents: [n] or None (chains).
    Returns out [n, Hq, D], the weighted mean of |v| [n, Hq, D], and [n, Hq] the largest scale * sum over rotary pairs of the product of
    the query's and the key's length in the pair that a row sees (no rotation changes these lengths)."""
    n_q, Hq, D = q.shape
    Hkv, P = k_pages.shape[1], v_pages.shape[3]
    G, scale = Hq // Hkv, sm_scale if sm_scale > 0 else D ** -0.5
    out, mean, size = np.zeros((n_q, Hq, D)), np.zeros((n_q, Hq, D)), np.zeros((n_q, Hq))
    for b in range(len(kv_lens)):
        q0, T, L = int(cu_q_lens[b]), int(cu_q_lens[b + 1] - cu_q_lens[b]), int(kv_lens[b])
        C = L - T
        idx = np.asarray(block_tables[b][: -(-L // P)], dtype=np.int64)
        wide = lambda pages, s: pages[idx] * (1.0 if s is None else np.asarray(s, np.float64)[idx].reshape(-1, *[1] * (pages.ndim - 1)))  # noqa: E731
        k = wide(k_pages, k_scales).transpose(0, 3, 1, 2, 4).reshape(-1, Hkv, D)[:L]
        v = wide(v_pages, v_scales).transpose(0, 3, 1, 2).reshape(-1, Hkv, D)[:L]
        slots = np.arange(L)
        valid = np.ones(L, bool)
        pos = slots.copy()
        if block_positions is not None:
            pos = np.asarray(block_positions[b])[slots // P] + slots % P
        if block_valid_mask is not None:
            valid = ((np.asarray(block_valid_mask[b], dtype=np.uint64)[slots // P] >> (slots % P).astype(np.uint64)) & np.uint64(1)).astype(bool)
        pos[max(C, 0):] = np.asarray(q_positions)[q0 + max(-C, 0): q0 + T]
        par = np.arange(-1, T - 1) if parents is None else np.asarray(parents)[q0: q0 + T]
        kr = _rotate(k, pos, theta, interleaved)
        qr = _rotate(np.asarray(q[q0: q0 + T]), np.asarray(q_positions)[q0: q0 + T], theta, interleaved)
        for i in range(T):
            sees = valid.copy()
            sees[max(C, 0):] = False
            for j in path_of(par, i):
                if C + j >= 0:
                    sees[C + j] = valid[C + j]
            if not sees.any():
                continue
            ks, vs = kr[sees], v[sees]
            for h in range(Hq):
                s = scale * (ks[:, h // G] @ qr[i, h])
                w = np.exp(s - s.max())
                w /= w.sum()
                out[q0 + i, h] = w @ vs[:, h // G]
                mean[q0 + i, h] = w @ np.abs(vs[:, h // G])
                size[q0 + i, h] = scale * (_lengths(ks[:, h // G], interleaved) @ _lengths(qr[i, h], interleaved)).max()
    return out, mean, size


def tables_extend(kv_lens, new_lens, block_tables, P, *, num_pages, n_blocks=None, free_pages=None, free_head=0, first_positions=None,
                  token_offsets=None, block_positions=None, block_valid_mask=None, max_tokens=None):
    """Request by request. Returns a dict of everything the call writes; tokens not served and entries not written are absent
    (token arrays are lists of (index, value))."""
    B, max_blocks = np.shape(block_tables)
    bt = np.array(block_tables, dtype=np.int64)
    bp = None if block_positions is None else np.array(block_positions, dtype=np.int64)
    bm = None if block_valid_mask is None else np.array(block_valid_mask, dtype=np.uint32)
    cu, run, first, status, kv_out, held_out = [0], [], [], [], [], []
    slots, positions, requests = {}, {}, {}
    asked, used = 0, 0
    for b in range(B):
        kv, new, held = int(kv_lens[b]), int(new_lens[b]), 0 if n_blocks is None else int(n_blocks[b])
        bad = kv < 0 or new < 0 or held < 0
        n = 0 if bad else new
        blocks = -(-(kv + n) // P)
        st = 3 if bad else 1 if blocks > max_blocks else 0
        need = max(0, blocks - held) if st == 0 and n_blocks is not None else 0
        asked += need
        if need and asked > len(free_pages) - free_head:
            st = 2
        t0 = cu[-1]
        cu.append(t0 + n)
        status.append(st)
        run.append(b if st == 0 else -1)
        first.append(kv if st == 0 else -1)
        kv_out.append(kv + n if st == 0 else kv)
        held_out.append(held + need if st == 0 else held)
        if st == 0:
            for j in range(need):
                bt[b, held + j] = free_pages[free_head + used + j]
            used += need
        for i in range(n):
            t = t0 + i
            if max_tokens is not None and t >= max_tokens:
                break
            if st:
                slots[t] = positions[t] = requests[t] = -1
                continue
            j, s = (kv + i) // P, (kv + i) % P
            base = kv if first_positions is None else int(first_positions[b])
            slots[t] = int(bt[b, j]) * P + s if 0 <= bt[b, j] < num_pages else -1
            positions[t] = base + (i if token_offsets is None else int(token_offsets[t]))
            requests[t] = b
            if bp is not None and s == 0:
                bp[b, j] = base + i
            if bm is not None and (s == 0 or i == 0):
                bits = sum(1 << x for x in range(s, min(P, s + n - i)))
                bm[b, j] = bits if s == 0 else int(bm[b, j]) | bits
    return dict(block_tables=bt, kv_lens=kv_out, n_blocks=held_out, free_head=free_head + used, cu=cu, run_request=run, run_first_slot=first,
                status=status, slots=slots, positions=positions, requests=requests, block_positions=bp, block_valid_mask=bm)


def kv_keep(k, v, block_tables, first_slots, cu_tree, kept, cu_kept, *, P, requant=None):
    """Moves tokens one after another in arrays of page contents k [N, Hkv, D/X, P, X], v [N, Hkv, D, P] (storage words), in place.
    requant(words, from_page, to_page, is_k): the words as the destination holds them. Returns kv_lens_out (None: left out)."""
    N, max_blocks = k.shape[0], np.shape(block_tables)[1]
    lens = []
    for b, first in enumerate(first_slots):
        if first < 0:
            lens.append(None)
            continue
        nodes = cu_tree[b + 1] - cu_tree[b]
        mine = kept[cu_kept[b]: cu_kept[b + 1]]
        lens.append(int(first) + len(mine))
        for r, node in enumerate(mine):
            at, to = int(first) + int(node), int(first) + r
            if (r and node <= mine[r - 1]) or node <= r or node >= nodes or at // P >= max_blocks:
                continue
            pa, pt = int(block_tables[b][at // P]), int(block_tables[b][to // P])
            if not (0 <= pa < N and 0 <= pt < N):
                continue
            kw, vw = k[pa, :, :, at % P, :].copy(), v[pa, :, :, at % P].copy()
            if requant is not None:
                kw, vw = requant(kw, pa, pt, True), requant(vw, pa, pt, False)
            k[pt, :, :, to % P, :], v[pt, :, :, to % P] = kw, vw
    return lens
