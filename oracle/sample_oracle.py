"""Slow CPU oracle of the verification against the base model's probabilities, written from its definition: numpy, loops; logits are
processed in float32, each operation by itself, as their definition says, everything else in 64 bits.  Test infrastructure only."""
from __future__ import annotations

import numpy as np

from oracle.rows_oracle import path_of

F = np.float32


def processed(logits, s, row, node_tok, parent, pen):
    """One row's processed logits (float32); pen: dict as the binding takes it, of numpy arrays, or None."""
    x = logits[s, row].astype(F)
    V = len(x)
    if pen is None:
        return np.where(np.isnan(x), F(-np.inf), x)
    bits = np.arange(V)
    seen = ((pen["seen"][s].view(np.uint32)[bits // 32] >> (bits % 32).astype(np.uint32)) & 1) > 0 if pen.get("seen") is not None else None
    c = np.zeros(V, np.int64)
    if pen.get("counts") is not None:
        c = np.where(seen, pen["counts"][s], 0) if seen is not None else pen["counts"][s].astype(np.int64)
    c = c.copy()
    for node in path_of(parent[s] if parent is not None else [], row):
        t = int(node_tok[s][node])
        if 0 <= t < V:
            c[t] += 1
    touched = (c > 0) | (seen if seen is not None else False)
    rep, pres, freq = (F(pen[k][s]) if pen.get(k) is not None else F(d) for k, d in (("repetition", 1), ("presence", 0), ("frequency", 0)))
    with np.errstate(all="ignore"):
        x = np.where(touched, np.where(x > 0, x / rep, x * rep), x).astype(F)
        x = np.where(touched, x - (freq * c.astype(F)).astype(F), x).astype(F)
        x = np.where(c > 0, x - pres, x).astype(F)
        if pen.get("bias") is not None and 0 <= pen["bias_row"][s] < len(pen["bias"]):
            x = (x + pen["bias"][pen["bias_row"][s]]).astype(F)
    if pen.get("allowed") is not None and 0 <= pen["mask_row"][s][row] < len(pen["allowed"]):
        m = pen["allowed"][pen["mask_row"][s][row]].view(np.uint32)
        x = np.where((m[bits // 32] >> (bits % 32).astype(np.uint32)) & 1, x, F(-np.inf))
    return np.where(np.isnan(x), F(-np.inf), x)


def weights(x, T):
    """Weights of processed logits; None where nothing is above -inf.  (+inf is taken as the largest finite number.)"""
    x = np.minimum(x, np.finfo(F).max)
    top = x.max()
    if top == -np.inf:
        return None
    if not T > 0:
        w = np.zeros(len(x))
        w[int(x.argmax())] = 1
        return w
    return np.exp((x.astype(np.float64) - float(top)) / float(F(T)))


def verify(logits, node_tok, parent, n_nodes, temperature, uniform, pen):
    """Everything spec_verify_sampled writes, as lists per sequence: (tokens, rows, logps), and by how much of the mass the nearest
    end of a stretch was missed in the closest of its choices."""
    b, R, V = logits.shape
    n = uniform.shape[1] - 1
    got = []
    for s in range(b):
        nodes = R - 1 if n_nodes is None else min(max(int(n_nodes[s]), -1), R - 1)
        if nodes < 0:
            got.append(([], [], [], 1.0))
            continue
        T = 1.0 if temperature is None else temperature[s]
        tokens, rows, logps, row, near = [], [], [], 0, 1.0
        for level in range(n + 1):
            w = weights(processed(logits, s, row, node_tok, parent, pen), T)
            children, order = [], []
            if level < n:
                for i in range(nodes):
                    up = int(parent[s][i])
                    t = int(node_tok[s][i])
                    if (up + 1 if 0 <= up < i else 0) == row and 0 <= t < V and t not in order:
                        children.append(i)
                        order.append(t)
            rows.append(row)
            if w is None:
                token, logp = 0, -np.inf
                down = [i for i, t in zip(children, order) if t == 0]
            else:
                S = w.sum()
                u = float(uniform[s][level])
                u = min(u, 1 - 2.0 ** -24) if u > 0 else 0.0
                rest = np.ones(V, bool)
                rest[order] = False
                line = np.array(order + list(np.flatnonzero(rest)), np.int64)
                ends = np.cumsum(w[line])
                at = u * S
                hit = np.flatnonzero((ends > at) & (w[line] > 0))
                k = int(hit[0]) if len(hit) else int(np.flatnonzero(w[line] > 0)[-1])
                near = min(near, float(np.abs(ends[:-1][w[line][1:] > 0] - at).min() / S) if V > 1 and (w[line][1:] > 0).any() and T > 0 else 1.0)
                token, logp = int(line[k]), float(np.log(w[line[k]] / S))
                down = [i for i, t in zip(children, order) if t == token]
            tokens.append(token)
            logps.append(logp)
            if not down:
                break
            row = down[0] + 1
        got.append((tokens, rows, logps, near))
    return got
