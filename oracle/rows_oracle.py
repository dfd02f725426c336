"""Slow CPU oracle of the operators on the rows of a token tree, written from their definitions: numpy, loops, 64 bits.

Row 0 of a sequence is the token sampled last, row 1 + i is node i; row r sees the cached tokens, row 0, its ancestors and
itself.  Test infrastructure only."""
from __future__ import annotations

import numpy as np

MAX_CHAIN = 8   # nodes of a path that are followed, the row's own among them


def path_of(parent, row):
    """Nodes on the path of a row, the row's own first."""
    nodes, node = [], row - 1
    while node >= 0 and len(nodes) < MAX_CHAIN:
        nodes.append(node)
        up = int(parent[node])
        node = up if up < node else -1
    return nodes


def attention(q, k_new, v_new, k_cache, v_cache, table, ctx, parent, n_nodes, scale):
    """(out, weighted) [batch, R, q_heads, D] float64; weighted = sum_k p_k |v_k|, which error bounds are stated in, and the largest
    sum_d |q_d k_d| * scale and number of keys.  Rows that do not exist hold NaN."""
    b, R, H, D = q.shape
    n_blocks, page, KH, _ = k_cache.shape
    out, weighted = np.full((b, R, H, D), np.nan), np.full((b, R, H, D), np.nan)
    products, most = 0.0, 0
    for s in range(b):
        where = [(int(table[s][t // page]), t % page) for t in range(int(ctx[s]))]
        where = [(x, y) for x, y in where if 0 <= x < n_blocks]
        for r in range(int(n_nodes[s]) + 1):
            rows = [0] + [x + 1 for x in path_of(parent[s] if R > 1 else [], r)]
            for h in range(H):
                g = h // (H // KH)
                k = np.array([k_cache[x, y, g] for x, y in where] + [k_new[s, x, g] for x in rows], np.float64)
                v = np.array([v_cache[x, y, g] for x, y in where] + [v_new[s, x, g] for x in rows], np.float64)
                x = q[s, r, h].astype(np.float64)
                z = k @ x * scale
                products = max(products, float((np.abs(k) @ np.abs(x)).max() * abs(scale)))
                most = max(most, len(z))
                p = np.exp(z - z.max())
                p /= p.sum()
                out[s, r, h], weighted[s, r, h] = p @ v, p @ np.abs(v)
    return out, weighted, products, most


def extend(ctx, add, table, ring, state, page, cap, path=None, seq_rows=0):
    """Everything spec_cache_extend writes, as a dict of int lists / arrays."""
    table, ring = np.array(table), np.array(ring)
    (head, count), n, width = state, len(ring), table.shape[1]
    free = [int(ring[(head + i) % n]) for i in range(count)]
    new, added, start, back, full = [], [], [], [], False
    slot, pos, src = [], [], []
    taken = asked = rows = 0
    for q, (c, a) in enumerate(zip(ctx, add)):
        c, a = int(c), int(a)
        start.append(len(slot))
        need = -(-(c + max(a, 0)) // page) - -(-c // page)
        if a < 0:
            n_new = max(c + a, 0)
            back += [int(x) for x in table[q, -(-n_new // page):-(-c // page)]]
            new.append(n_new), added.append(n_new - c)
            continue
        if a > 0 and c + a <= width * page:
            asked, rows = asked + need, rows + a
            full = full or asked > count or rows > cap
        if a == 0 or full or c + a > width * page:
            new.append(c), added.append(0)
            continue
        for i in range(need):
            table[q, -(-c // page) + i] = free[taken]
            taken += 1
        for j in range(a):
            t = c + j
            x = int(table[q, t // page])
            slot.append(x * page + t % page if 0 <= x < n else -1)
            pos.append(t)
            if path is not None:
                r = int(path[q][j]) if j < len(path[q]) else -1
                src.append(q * seq_rows + r if 0 <= r < seq_rows else -1)
        new.append(c + a), added.append(a)
    start.append(len(slot))
    for i, x in enumerate(back):
        ring[(head + count + i) % n] = x
    pad = [-1] * (cap - len(slot))
    got = dict(new_len=new, added=added, block_table=table, ring=ring, ring_state_new=[(head + taken) % n, count - taken + len(back)],
               row_start=start, slot=slot + pad, pos=pos + pad)
    if path is not None:
        got["src_row"] = src + pad
    return got


def store(k_new, slot, cache, src=None):
    """cache [L, n_blocks, page, ...] with rows k_new [L, rows, ...] in their slots."""
    cache = np.array(cache)
    L, n_blocks, page = cache.shape[:3]
    for t, s in enumerate(slot):
        r = t if src is None else int(src[t])
        if 0 <= s < n_blocks * page and 0 <= r < k_new.shape[1]:
            cache[:, s // page, s % page] = k_new[:, r]
    return cache


def bit(words, t):
    return (int(words[t // 32]) >> (t % 32)) & 1


def processed(logits, pen, tok, parent, n_nodes, dt=np.float64):
    """Processed rows [batch, R, V] in `dt`, and the sum of the sizes of all intermediate values (for error bounds); rows
    that do not exist hold NaN."""
    b, R, V = logits.shape
    out, sizes = np.full((b, R, V), np.nan, dt), np.zeros((b, R, V))
    for q in range(b):
        for r in range(int(n_nodes[q]) + 1):
            path = [int(tok[q][x]) for x in path_of(parent[q], r)] if tok is not None else []
            for t in range(V):
                v = dt(logits[q, r, t])
                listed = pen.get("seen") is not None and bit(pen["seen"][q], t)
                c = int(pen["counts"][q][t]) if pen.get("counts") is not None and (pen.get("seen") is None or listed) else 0
                c += path.count(t)
                if listed or c > 0:
                    rep = dt(pen["repetition"][q]) if pen.get("repetition") is not None else dt(1)
                    v = v / rep if v > 0 else v * rep
                size = abs(float(v))
                v = v - dt(pen["frequency"][q] if pen.get("frequency") is not None else 0) * dt(c)
                size += 2 * abs(float(v))
                if c > 0:
                    v = v - dt(pen["presence"][q] if pen.get("presence") is not None else 0)
                    size += abs(float(v))
                if pen.get("bias") is not None and 0 <= pen["bias_row"][q] < len(pen["bias"]):
                    v = v + dt(pen["bias"][pen["bias_row"][q]][t])
                    size += abs(float(v))
                if pen.get("allowed") is not None and 0 <= pen["mask_row"][q][r] < len(pen["allowed"]):
                    if not bit(pen["allowed"][pen["mask_row"][q][r]], t):
                        v = dt(-np.inf)
                out[q, r, t], sizes[q, r, t] = v, size
    return out, sizes


def first_maximum(row):
    best = 0
    for t, v in enumerate(row):
        if v > row[best] or (np.isnan(row[best]) and not np.isnan(v)):
            best = t
    return best if row[best] > -np.inf else 0


def verify_tree(rows, cand, cand_node, n_nodes, n_cand=None):
    """rows: processed logits [batch, R, V].  A dict of what spec_verify_tree writes."""
    b, R, _ = rows.shape
    Bc, n = cand.shape[1:]
    got = {k: [] for k in ("greedy", "accept_len", "best_cand", "out_tokens", "n_out", "path_row", "accept_all")}
    for q in range(b):
        live = int(n_nodes[q]) + 1
        greedy = [first_maximum(rows[q, r]) if r < live else -1 for r in range(R)]
        got["greedy"].append(greedy)
        lengths = []
        for c in range(Bc):
            a = 0
            if live > 0 and (n_cand is None or c < n_cand[q]):
                for p in range(n):
                    before = 0 if p == 0 else int(cand_node[q, c, p - 1]) + 1
                    mine = int(cand_node[q, c, p]) + 1
                    if not (0 <= before < live and 1 <= mine < live and greedy[before] == cand[q, c, p]):
                        break
                    a += 1
            lengths.append(a)
        a, best = max(lengths), lengths.index(max(lengths))
        path = [0] + [int(x) + 1 for x in cand_node[q, best, :a]] if live > 0 else []
        out = [int(x) for x in cand[q, best, :a]] + [greedy[path[-1]]] if live > 0 else []
        got["accept_len"].append(a), got["best_cand"].append(best), got["n_out"].append(len(out))
        got["out_tokens"].append(out + [-1] * (n + 1 - len(out)))
        got["path_row"].append(path + [-1] * (n + 1 - len(path)))
        got["accept_all"].append(lengths)
    return {k: np.array(v, np.int32) for k, v in got.items()}
