"""Operators around the base model's forward over a candidate tree, for a server whose cache holds four bits an element and whose
users sample.

A case is a dict of plain values.  `kind` names the operator:

  rotate     spec_rotate_rows: norms of queries and keys for each head and the position rotation, in one pass
  append     spec_cache_append: keys and values into a paged cache, the keys' norm and rotation on the way
  pack       spec_packed_append: the same into a cache of four bits; what it holds is read back (spec_packed_load)
  load       spec_packed_load: tokens of a cache of four bits as bfloat16 rows
  attention  spec_packed_attention: the rows of a token tree attend to a cache of four bits and to their own ancestors
  sampled    spec_verify_sampled: drafted tokens against the target's probabilities, from given random numbers

Sequence q has `R` rows: row 0 is the token sampled last, row 1 + i is node i of its tree.  `tree` is the branching per
stage and `B` the candidates kept, whose distinct prefixes are the nodes; tree "" is plain decoding of one token.
Lengths follow from the case alone and are dealt out to the sequences by the seed.

A cache of four bits holds, for each token, key/value head and group of 32 elements, a scale 2^(s - 127) (s one byte) and 32 codes: the
lowest three bits stand for 0, 0.5, 1, 1.5, 2, 3, 4, 6, the highest one for the sign, the element with the even number in the low half of a byte.
"""
import math
import random

import torch

own = False
DEV = "cuda"
INF = math.inf
I32 = dict(dtype=torch.int32, device=DEV)
TREES = [("", 1), ("5,3,2", 16), ("6,3,2", 16), ("4,3,2", 24), ("6,4,3", 32), ("6,4,3,2", 16), ("2,2,1,1,1,1,1", 4),
         ("1,1,1,1,1,1,1", 1), ("1,1,1,1,1", 1), ("4,2", 8), ("3,1,1", 3)]
HEADS = [(32, 32), (40, 40), (64, 8), (48, 1), (32, 8), (12, 4), (7, 1)]
EPS = 1e-5


def _rotate(name, q_heads, kv_heads, D, rot, pairs, norm, tree, B, batch, tokens, dtype="bf16"):
    """batch > 0: trees over up to `tokens` tokens each; batch = 0: `tokens` tokens of prompts, packed"""
    return {"name": name, "kind": "rotate", "q_heads": q_heads, "kv_heads": kv_heads, "D": D, "rot": rot, "pairs": pairs,
            "norm": norm, "tree": tree, "B": B, "batch": batch, "tokens": tokens, "dtype": dtype}


def _append(name, layers, kv_heads, D, rot, pairs, norm, tokens, rows, page, dtype="bf16"):
    """rows = 0: every row is kept; otherwise kept rows of trees of so many rows, up to four of each"""
    return {"name": name, "kind": "append", "layers": layers, "kv_heads": kv_heads, "D": D, "rot": rot, "pairs": pairs,
            "norm": norm, "tokens": tokens, "rows": rows, "page": page, "dtype": dtype}


def _pack(name, layers, kv_heads, D, rot, norm, tokens, rows, page):
    return {"name": name, "kind": "pack", "layers": layers, "kv_heads": kv_heads, "D": D, "rot": rot, "pairs": False,
            "norm": norm, "tokens": tokens, "rows": rows, "page": page, "dtype": "bf16"}


def _load(name, kv_heads, D, tokens, page):
    return {"name": name, "kind": "load", "kv_heads": kv_heads, "D": D, "tokens": tokens, "page": page}


def _attention(name, q_heads, kv_heads, D, tree, B, batch, ctx, page):
    return {"name": name, "kind": "attention", "q_heads": q_heads, "kv_heads": kv_heads, "D": D, "tree": tree, "B": B,
            "batch": batch, "ctx": ctx, "page": page}


def _sampled(name, V, tree, B, batch, past, dtype):
    return {"name": name, "kind": "sampled", "V": V, "tree": tree, "B": B, "batch": batch, "past": past, "dtype": dtype}


def listed():
    return [
        # one user of a 7B model, a layer's queries and keys of the tree: latency
        _rotate("rotate_7b_b1", 32, 32, 128, 128, False, False, "5,3,2", 16, 1, 600),
        # a chunk of prompts of a model with grouped heads and norms
        _rotate("rotate_prompt", 64, 8, 128, 128, False, True, "", 1, 0, 16000),
        # plain decoding of a loaded server: one token of each sequence, a layer
        _append("append_step", 1, 8, 128, 128, False, True, 64, 0, 16),
        # a chunk of prompts, half of each head rotated, neighbours as pairs
        _append("append_prompt", 1, 8, 128, 64, True, False, 16000, 0, 64),
        # a chunk of prompts into the cache of four bits
        _pack("pack_prompt", 1, 8, 128, 128, True, 16000, 0, 64),
        # the kept rows of one user's step, all layers at once, rotated before the attention: their values read back
        _pack("pack_step_b1", 32, 32, 128, 0, False, 3, 49, 16),
        # long files of several requests
        _load("load_long", 8, 128, 60000, 64),
        # one user of a 7B model, a short conversation: latency
        _attention("attention_7b_b1", 32, 32, 128, "5,3,2", 16, 1, 600, 16),
        # a full batch of the largest model, grouped heads, a wide tree: the matrix cores' work
        _attention("attention_70b_b32", 64, 8, 128, "6,4,3,2", 16, 32, 4000, 64),
        # the same model with speculation off, long conversations: the cache's bytes
        _attention("attention_decode_b64", 64, 8, 128, "", 1, 64, 8000, 64),
        # one user's tree, sampled: the smallest verification
        _sampled("sampled_7b_b1", 32000, "5,3,2", 16, 1, 500, "f32"),
        # a full batch of the largest vocabulary, most with a temperature
        _sampled("sampled_70b_b32", 128256, "6,4,3,2", 16, 32, 2000, "bf16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choices(["rotate", "append", "pack", "load", "attention", "sampled"], [15, 15, 15, 5, 30, 20])[0]
    tree, B = rng.choice(TREES)
    q_heads, kv_heads = rng.choice(HEADS)
    D = rng.choice([128, 128, 64, 16 * rng.randint(2, 16)])
    rot = rng.choice([D, D, 16 * rng.randint(1, D // 16)])
    pairs, norm = rng.random() < 0.3, rng.random() < 0.5
    page = rng.choice([16, 32, 64, 128, 256, rng.randint(1, 200)])
    if kind == "rotate":
        batch = rng.choice([0, _log_int(rng, 1, 64)])
        c = _rotate("", q_heads, kv_heads, D, rot, pairs, norm, tree, B, batch, _log_int(rng, 1, 16000 if batch == 0 else 30000),
                    rng.choice(["bf16", "bf16", "f32"]))
        while c["batch"] == 0 and c["tokens"] * (q_heads + kv_heads) * D * (2 if c["dtype"] == "bf16" else 4) > 3e8:
            c["tokens"] = max(1, c["tokens"] // 2)
    elif kind in ("append", "pack"):
        rows, layers = rng.choice([0, 8, 49, 65]), rng.choice([1, 1, rng.randint(2, 40)])
        tokens = _log_int(rng, 1, 16000) if rows == 0 else _log_int(rng, 1, 250)
        kv_heads = rng.choice([1, 4, 8, 32, 40])
        if kind == "append":
            c = _append("", layers, kv_heads, D, rot, pairs, norm, tokens, rows, page, rng.choice(["bf16", "bf16", "f32"]))
        else:
            D = rng.choice([128, 128, 64, 32 * rng.randint(1, 8)])
            c = _pack("", layers, kv_heads, D, rng.choice([D, D, 0, 16 * rng.randint(1, D // 16)]), norm, tokens, rows, page)
        size = 2 if c["dtype"] == "bf16" else 4
        while c["layers"] * kv_heads * D * size * max(c["tokens"], 8 * rows) > 3.3e7:
            if c["layers"] == c["tokens"] == 1:
                break
            c["layers"], c["tokens"] = max(1, c["layers"] // 2), max(1, c["tokens"] // 2)
    elif kind == "load":
        c = _load("", kv_heads, rng.choice([128, 128, 64, 32 * rng.randint(1, 8)]), _log_int(rng, 1, 60000), page)
        while c["tokens"] * kv_heads * c["D"] > 6e7:
            c["tokens"] //= 2
    elif kind == "attention":
        D = rng.choice([128, 128, 64, 32 * rng.randint(1, 8)])
        c = _attention("", q_heads, kv_heads, D, tree, B, _log_int(rng, 1, 64), _log_int(rng, 1, 40000), page)
        # (no dearer than the largest listed ones)
        while c["batch"] * c["ctx"] * max(q_heads * _rows(c) / 4e10, kv_heads / 3e8) * D > 1.0:
            c["ctx"], c["batch"] = max(1, c["ctx"] * 2 // 3), max(1, c["batch"] * 3 // 4)
    else:
        c = _sampled("", rng.choice([32000, 32016, 49152, 128256, rng.randint(1000, 130000)]), tree, B, _log_int(rng, 1, 64),
                     _log_int(rng, 1, 8000), rng.choice(["f32", "bf16"]))
        while c["batch"] * _rows(c) * c["V"] * (4 if c["dtype"] == "f32" else 2) > 5e8:
            c["batch"] = max(1, c["batch"] * 2 // 3)
    del c["name"]
    return c


# ---- trees, lengths and pages ---------------------------------------------------------------------------------

def _stages(case):
    return [int(k) for k in case["tree"].split(",")] if case["tree"] else []


def _rows(case):
    return 1 + case["B"] * len(_stages(case))


def _trees(case, rng):
    """Per sequence its candidates, as ranks per stage: B distinct leaves of the full tree, the likely ones more often."""
    ks, got = _stages(case), []
    for _ in range(case["batch"]):
        leaves = set()
        while len(leaves) < case["B"] and ks:
            leaves.add(tuple(min(k - 1, int(rng.expovariate(1.0))) if rng.random() < 0.8 else rng.randrange(k) for k in ks))
        leaves = sorted(leaves)
        rng.shuffle(leaves)
        got.append(leaves)
    return got


def _key(case):
    return ";".join("%s=%s" % (k, case[k]) for k in sorted(case) if k != "name")


def _shape(case):
    """The trees and cached lengths of a case: its lengths spread over a factor of eight and more, one of them whole, and
    one new sequence with nothing cached."""
    rng = random.Random(_key(case))
    most = case.get("ctx", case.get("tokens", 1))
    ctx = [max(1, int(most * math.exp(-2.2 * rng.random() ** 2))) for _ in range(case["batch"])]
    ctx[0] = most
    if case["batch"] > 4:
        ctx[1] = 0
    return _trees(case, rng), ctx


def _nodes(leaves):
    """Distinct prefixes in order of first appearance: {prefix: number}."""
    node = {}
    for leaf in leaves:
        for p in range(len(leaf)):
            node.setdefault(leaf[:p + 1], len(node))
    return node


def _metadata(case, trees, V, rng):
    """The token trees' tables, as spec_tree_metadata writes them, and each node's rank among its siblings."""
    b, M = case["batch"], _rows(case) - 1
    tok, parent = torch.full((b, M), -1, dtype=torch.int32), torch.full((b, M), -1, dtype=torch.int32)
    depth, rank = torch.zeros((b, M), dtype=torch.int32), torch.zeros((b, M), dtype=torch.int32)
    count = torch.zeros((b,), dtype=torch.int32)
    for q, leaves in enumerate(trees):
        node, token = _nodes(leaves), {}
        count[q] = len(node)
        for prefix, i in node.items():
            family = token.setdefault(prefix[:-1], rng.sample(range(V), 8))
            tok[q, i], rank[q, i] = family[prefix[-1]], prefix[-1]
            parent[q, i], depth[q, i] = node.get(prefix[:-1], -1), len(prefix)
    return {k: v.to(DEV) for k, v in dict(tok=tok, parent=parent, depth=depth, rank=rank, count=count).items()}


def _pages(lengths, page, spare, g):
    """Block tables over a shuffled pool, and the pool's size."""
    width = max(1, -(-max(lengths) // page))
    need = [-(-n // page) for n in lengths]
    pool = sum(need) + spare
    at = torch.randperm(pool, generator=g, device=DEV).to(torch.int32)
    table = torch.full((len(lengths), width), -1, **I32)
    first = 0
    for q, n in enumerate(need):
        table[q, :n] = at[first:first + n]
        first += n
    return table, pool


def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


# ---- what a program has in hand ---------------------------------------------------------------------------------

def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return {"case": case, **_PREPARE[case["kind"]](case, g, random.Random(seed))}


def _rand(g, *shape, dtype=torch.float32):
    return torch.randn(shape, generator=g, device=DEV).to(dtype)


def _heads(g, dtype, *shape):
    """Rows of heads as projections give them: a few elements of a head stand out."""
    loud = 1 + 4 * (torch.rand(shape[-2:], generator=g, device=DEV) < 0.05).float()
    return (torch.randn(shape, generator=g, device=DEV) * loud).to(dtype)


def _angles(rot, positions):
    """The model's table: cosines and sines of the pairs' angles at every position."""
    a = torch.arange(positions, device=DEV).double()[:, None] * 10000.0 ** (-torch.arange(rot // 2, device=DEV).double() * 2 / max(rot, 1))
    return torch.cos(a).float(), torch.sin(a).float()


def _prepare_rotate(case, g, rng):
    dt, D, b = _dtype(case), case["D"], max(1, case["batch"])
    st = {}
    if case["batch"]:
        trees, ctx = _shape(case)
        rng.shuffle(trees)
        rng.shuffle(ctx)
        meta = _metadata(case, trees, 32000, rng)
        R, most = _rows(case), max(ctx) + 8
        st |= {"ctx": torch.tensor(ctx, **I32), "depth": meta["depth"], "count": meta["count"]}
    else:
        # prompts one behind the other, each from its first token on, the first one from a chunk before
        R, pos = case["tokens"], []
        at = rng.randint(0, 2000)
        while len(pos) < R:
            n = min(R - len(pos), max(1, int(R * rng.random() ** 2)))
            pos += range(at, at + n)
            at = 0
        most = max(pos) + 1
        st["pos"] = torch.tensor([pos], **I32)
    st["q"], st["k"] = _heads(g, dt, b, R, case["q_heads"], D), _heads(g, dt, b, R, case["kv_heads"], D)
    st["q_out"], st["k_out"] = torch.zeros_like(st["q"]), torch.zeros_like(st["k"])
    st["cos"], st["sin"] = _angles(case["rot"], most)
    st["q_weight"], st["k_weight"] = (1 + 0.1 * _rand(g, D) if case["norm"] else None for _ in range(2))
    return st


def _slots(case, g):
    """Rows and slots of an append: consecutive slots within a page, pages in any order; two entries behind the last token."""
    T, page = case["tokens"], case["page"]
    rows = T + 2 if case["rows"] == 0 else case["rows"] * -(-T // 4)
    pages = -(-T // page) + 2
    order = torch.randperm(pages, generator=g, device=DEV)[: -(-T // page)]
    slots = (order[:, None] * page + torch.arange(page, device=DEV)).reshape(-1)[:T]
    slot = torch.cat([slots, torch.full((2,), -1, device=DEV)]).to(torch.int32)
    src = None
    if case["rows"]:
        src = torch.randperm(rows, generator=g, device=DEV)[:T].sort()[0]
        src = torch.cat([src, torch.zeros((2,), device=DEV, dtype=src.dtype)]).to(torch.int32)
    return rows, pages, slot, src


def _prepare_append(case, g, rng):
    dt, L, H, D, T = _dtype(case), case["layers"], case["kv_heads"], case["D"], case["tokens"]
    rows, pages, slot, src = _slots(case, g)
    first = rng.randint(0, 3000)
    st = {"k_new": _heads(g, dt, L, rows, H, D), "v_new": _heads(g, dt, L, rows, H, D), "slot": slot, "src": src, "cos": None, "sin": None,
          "pos": torch.cat([first + torch.arange(T, device=DEV), torch.full((2,), -1, device=DEV)]).to(torch.int32)}
    if case["rot"]:
        st["cos"], st["sin"] = _angles(case["rot"], first + T)
    st["k_weight"] = 1 + 0.1 * _rand(g, L, D) if case["norm"] else None
    if case["kind"] == "append":
        st["k_cache"], st["v_cache"] = (_rand(g, L, pages, case["page"], H, D, dtype=dt) for _ in range(2))
    else:
        st |= _packed(g, L, pages, H, case["page"], D)
        st["k_out"], st["v_out"] = (torch.zeros((L, T, H, D), dtype=dt, device=DEV) for _ in range(2))
        st["kept"] = slot[:T].contiguous()
    return st


def _packed(g, L, pages, H, page, D):
    """A cache of four bits, the tokens of a head in a block one behind the other: [layers, blocks, slots, heads, bytes] as views."""
    st = {}
    for x in "kv":
        codes = torch.randint(0, 256, (L, pages, H, page, D // 2), generator=g, device=DEV, dtype=torch.uint8)
        # (scales of values around one: amounts up to 6 * 2^-2 or 6 * 2^-1, now and then more)
        scale = torch.randint(125, 127, (L, pages, H, page, D // 32), generator=g, device=DEV, dtype=torch.uint8)
        scale += 2 * (torch.rand(scale.shape, generator=g, device=DEV) < 0.02).to(torch.uint8)
        st[x + "_cache"], st[x + "_scale"] = codes.transpose(2, 3), scale.transpose(2, 3)
    return st


def _prepare_load(case, g, rng):
    T, H, D, page = case["tokens"], case["kv_heads"], case["D"], case["page"]
    pages = -(-T // page) + 2
    order = torch.randperm(pages, generator=g, device=DEV)[: -(-T // page)]
    st = {k: v[0] for k, v in _packed(g, 1, pages, H, page, D).items()}
    st["slot"] = (order[:, None] * page + torch.arange(page, device=DEV)).reshape(-1)[:T].to(torch.int32)
    st["k_out"], st["v_out"] = (torch.zeros((T, H, D), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    return st


def _prepare_attention(case, g, rng):
    dt, b, D, R, KH = torch.bfloat16, case["batch"], case["D"], _rows(case), case["kv_heads"]
    trees, ctx = _shape(case)
    rng.shuffle(trees)
    rng.shuffle(ctx)
    meta = _metadata(case, trees, 32000, rng)
    table, pool = _pages(ctx, case["page"], 8, g)
    st = {k: v[0] for k, v in _packed(g, 1, pool, KH, case["page"], D).items()}
    st |= {"k_new": _rand(g, b, R, KH, D, dtype=dt), "v_new": _rand(g, b, R, KH, D, dtype=dt), "q": _rand(g, b, R, case["q_heads"], D, dtype=dt) * 1.5,
           "table": table, "ctx": torch.tensor(ctx, **I32), "parent": meta["parent"], "count": meta["count"]}
    st["out"] = torch.zeros_like(st["q"])
    return st


def _prepare_sampled(case, g, rng):
    b, V, R, past, n = case["batch"], case["V"], _rows(case), case["past"], len(_stages(case))
    words = -(-V // 32)
    trees, _ = _shape(case)
    rng.shuffle(trees)
    meta = _metadata(case, trees, V, rng)

    def uniform(*shape):
        return torch.rand(shape, generator=g, device=DEV)

    # what was said so far: frequent tokens often, the first half of it the prompt
    said = (V * uniform(b, past) ** 3).long().clamp_(max=V - 1)
    counts = torch.zeros((b, V), **I32)
    counts.scatter_add_(1, said[:, past // 2:], torch.ones_like(said[:, past // 2:], dtype=torch.int32))
    seen = torch.zeros((b, 32 * words), dtype=torch.int64, device=DEV)
    seen.scatter_(1, said, 1)
    # the target gives a row's drafted tokens about 0.5, 0.2, 0.1 .. of its mass: the others' is V exp(2) where logits spread by 2
    logits = 2.0 * torch.randn((b, R, V), generator=g, device=DEV)
    if R > 1:
        row = (meta["parent"] + 1).long()
        share = math.log(V) + 2.5 - 0.9 * meta["rank"].float() + 0.5 * torch.randn(row.shape, generator=g, device=DEV)
        at = (row * V + meta["tok"].long().clamp(min=0))
        logits.view(b, -1).scatter_(1, torch.where(meta["tok"] >= 0, at, 0), torch.where(meta["tok"] >= 0, share, 0.0))
    # grammar masks for the rows of a fourth of the sequences; biases for as many others; an eighth without a temperature
    each = torch.arange(b, device=DEV)
    bound = each % 4 == 3
    rows_bound = max(1, b // 4) * R
    mask_row = torch.where(bound[:, None], (each // 4)[:, None] * R + torch.arange(R, device=DEV), -1)
    allowed = uniform(rows_bound, 32 * words) < 0.3
    n_bias = -(-b // 4)
    return {"logits": logits.to(_dtype(case)), "counts": counts, "seen": _bits(seen), "allowed": _bits(allowed.long()),
            "mask_row": mask_row.to(torch.int32).contiguous(),
            "bias": torch.where(uniform(n_bias, V) < 0.01, 4 * uniform(n_bias, V) - 2, 0.0),
            "bias_row": torch.where(each % 4 == 1, each // 4, -1).to(torch.int32),
            "repetition": 1.0 + 0.2 * uniform(b), "presence": 0.5 * uniform(b), "frequency": 0.2 * uniform(b), "meta": meta,
            "temperature": torch.where(each % 8 == 5, 0.0, 0.6 + 0.6 * uniform(b)), "uniform": uniform(b, n + 1),
            "outs": {"accept_len": torch.zeros((b,), **I32), "out_tokens": torch.zeros((b, n + 1), **I32), "n_out": torch.zeros((b,), **I32),
                     "path_row": torch.zeros((b, n + 1), **I32), "out_logp": torch.zeros((b, n + 1), device=DEV)}}


def _bits(bits):
    """Truth values [rows, 32 * words] as words of 32 bits, the lowest bit first."""
    x = (bits.view(bits.shape[0], -1, 32) << torch.arange(32, device=DEV)).sum(2)
    return torch.where(x >= 2 ** 31, x - 2 ** 32, x).to(torch.int32)


_PREPARE = {"rotate": _prepare_rotate, "append": _prepare_append, "pack": _prepare_append, "load": _prepare_load,
            "attention": _prepare_attention, "sampled": _prepare_sampled}


# ---- one pass ---------------------------------------------------------------------------------------------------

def run(st):
    return (_OWN if own else _PLAIN)[st["case"]["kind"]](st)


def _own_rotate(st):
    from paper_2404_19124_amd import binding as S
    S.spec_rotate_rows(st["q"], st["k"], st["q_out"], st["k_out"], st["cos"], st["sin"], pos=st.get("pos"), ctx_len=st.get("ctx"),
                       node_depth=st.get("depth"), n_nodes=st.get("count"), q_weight=st["q_weight"], k_weight=st["k_weight"], eps=EPS,
                       pairs=st["case"]["pairs"])
    return {"q": st["q_out"], "k": st["k_out"]}


def _own_append(st):
    from paper_2404_19124_amd import binding as S
    S.spec_cache_append(st["k_new"], st["v_new"], st["slot"], st["k_cache"], st["v_cache"], src_row=st["src"], pos=st["pos"],
                        cos=st["cos"], sin=st["sin"], k_weight=st["k_weight"], eps=EPS, pairs=st["case"]["pairs"])
    return {"k": st["k_cache"], "v": st["v_cache"]}


def _own_pack(st):
    from paper_2404_19124_amd import binding as S
    cache = (st["k_cache"], st["v_cache"], st["k_scale"], st["v_scale"])
    S.spec_packed_append(st["k_new"], st["v_new"], st["slot"], *cache, src_row=st["src"], pos=st["pos"], cos=st["cos"], sin=st["sin"],
                         k_weight=st["k_weight"], eps=EPS, pairs=st["case"]["pairs"])
    S.spec_packed_load(*cache, st["kept"], st["k_out"], st["v_out"])
    return {"k": st["k_out"], "v": st["v_out"]}


def _own_load(st):
    from paper_2404_19124_amd import binding as S
    S.spec_packed_load(st["k_cache"], st["v_cache"], st["k_scale"], st["v_scale"], st["slot"], st["k_out"], st["v_out"])
    return {"k": st["k_out"], "v": st["v_out"]}


def _own_attention(st):
    from paper_2404_19124_amd import binding as S
    c = st["case"]
    if "workspace" not in st:
        st["workspace"] = torch.empty(S.spec_packed_attention_workspace(c["batch"], _rows(c), c["q_heads"], c["kv_heads"], c["D"]),
                                      dtype=torch.uint8, device=DEV)
    S.spec_packed_attention(st["q"], st["k_new"], st["v_new"], st["k_cache"], st["v_cache"], st["k_scale"], st["v_scale"], st["table"],
                            st["ctx"], st["parent"], st["count"], st["out"], st["workspace"])
    return {"out": st["out"]}


_PENALTIES = ("counts", "seen", "repetition", "presence", "frequency", "bias", "bias_row", "allowed", "mask_row")


def _own_sampled(st):
    from paper_2404_19124_amd import binding as S
    m, o = st["meta"], st["outs"]
    if "workspace" not in st:
        st["workspace"] = torch.empty(S.spec_verify_sampled_workspace(*st["logits"].shape, st["logits"].dtype), dtype=torch.uint8, device=DEV)
    S.spec_verify_sampled(st["logits"], st["uniform"], m["count"], o["accept_len"], o["out_tokens"], o["n_out"], o["path_row"],
                          st["workspace"], out_logp=o["out_logp"], temperature=st["temperature"],
                          penalties={k: st[k] for k in _PENALTIES}, node_tok=m["tok"], node_parent=m["parent"], update=True)
    return {**o, "counts": st["counts"], "seen": st["seen"]}


_OWN = {"rotate": _own_rotate, "append": _own_append, "pack": _own_pack, "load": _own_load, "attention": _own_attention,
        "sampled": _own_sampled}


def _normed(x, weight):
    """float32 rows; with a weight over the root of their mean square, which is summed in 64 bits"""
    x = x.float()
    if weight is None:
        return x
    inv = 1 / torch.sqrt(x.double().square().mean(-1, keepdim=True) + EPS)
    return x * inv.float() * weight


def _turned(x, cos, sin, pairs):
    """The first 2 * cos.shape[-1] elements of float32 heads [.., heads, D] turned by the angles of their positions [.., half]."""
    half = cos.shape[-1]
    cos, sin = cos[..., None, :], sin[..., None, :]
    if pairs:
        a, b = x[..., 0:2 * half:2], x[..., 1:2 * half:2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    else:
        a, b = x[..., :half], x[..., half:2 * half]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    return torch.cat([turned, x[..., 2 * half:]], -1)


def _plain_rotate(st):
    if "pos" in st:
        pos = st["pos"]
        live = pos >= 0
    else:
        pos = st["ctx"][:, None] + torch.cat([torch.zeros_like(st["depth"][:, :1]) if st["depth"].shape[1] else st["ctx"][:, None] * 0, st["depth"]], 1)
        live = torch.arange(pos.shape[1], device=DEV) <= st["count"][:, None]
    cos, sin = st["cos"][pos.long()], st["sin"][pos.long()]
    for x in "qk":
        y = _turned(_normed(st[x], st[x + "_weight"]), cos, sin, st["case"]["pairs"]).to(st[x].dtype)
        st[x + "_out"] = torch.where(live[:, :, None, None], y, st[x + "_out"])
    return {"q": st["q_out"], "k": st["k_out"]}


def _new_rows(st):
    """The float32 keys and values of the entries with a slot, [layers, tokens, heads, D], and their slots."""
    T = st["case"]["tokens"]
    src = torch.arange(T, device=DEV) if st["src"] is None else st["src"][:T].long()
    weight = None if st["k_weight"] is None else st["k_weight"][:, None, None, :]
    k = _normed(st["k_new"][:, src], weight)
    if st["cos"] is not None:
        pos = st["pos"][:T].long()
        k = _turned(k, st["cos"][pos], st["sin"][pos], st["case"]["pairs"])
    return k, st["v_new"][:, src].float(), st["slot"][:T].long()


def _plain_append(st):
    k, v, slot = _new_rows(st)
    L, pages, page = st["k_cache"].shape[:3]
    for cache, new in ((st["k_cache"], k), (st["v_cache"], v)):
        cache.view(L, pages * page, *cache.shape[3:])[:, slot] = new.to(cache.dtype)
    return {"k": st["k_cache"], "v": st["v_cache"]}


def _to_four_bits(x):
    """Scales and codes of float32 [.., D]: the largest of a group of 32 is at most 7 times its scale."""
    y = x.unflatten(-1, (-1, 32))
    bits = y.abs().amax(-1).contiguous().view(torch.int32)
    e = ((bits >> 23) - 129 + (bits % (1 << 23) > 0x600000).int()).clamp(-125, 125)
    z = y.abs() * ((127 - e) << 23).view(torch.float32)[..., None]
    code = (z > 0.25).int() + (z >= 0.75) + (z > 1.25) + (z >= 1.75) + (z > 2.5) + (z >= 3.5) + (z > 5) + 8 * (y < 0)
    code = code.flatten(-2)
    return (e + 127).to(torch.uint8), (code[..., 0::2] + 16 * code[..., 1::2]).to(torch.uint8)


def _values(codes, scale):
    """The float32 values that codes [.., D / 2] and scales [.., D / 32] stand for."""
    amount = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], device=DEV)
    amount = torch.cat([amount, -amount])
    code = torch.stack([codes & 15, codes >> 4], -1).flatten(-2).long()
    return (amount[code].unflatten(-1, (-1, 32)) * (scale.int() << 23).view(torch.float32)[..., None]).flatten(-2)


def _plain_pack(st):
    k, v, slot = _new_rows(st)
    page = st["k_cache"].shape[2]
    out = {}
    for x, new in (("k", k), ("v", v)):
        codes, scale = st[x + "_cache"], st[x + "_scale"]
        scale[:, slot // page, slot % page], codes[:, slot // page, slot % page] = _to_four_bits(new)
        kept = st["kept"].long()
        out[x] = _values(codes[:, kept // page, kept % page], scale[:, kept // page, kept % page]).to(torch.bfloat16)
    return out


def _plain_load(st):
    slot, page = st["slot"].long(), st["k_cache"].shape[1]
    return {x: _values(st[x + "_cache"][slot // page, slot % page], st[x + "_scale"][slot // page, slot % page]).to(torch.bfloat16) for x in "kv"}


def _paths(parent):
    """[batch, R, R] float32: 1 where the second row is the first one itself, its ancestor or the root."""
    b, M = parent.shape
    rows = torch.arange(M + 1, device=DEV)
    up = torch.cat([torch.full((b, 1), -1, **I32), parent + 1], 1)
    m = ((up[:, :, None] == rows) | (rows[:, None] == rows)).float()
    m = m @ m
    m = m @ m
    m = m @ m
    return ((m @ m) > 0).float()


def _plain_attention(st):
    c, ctx = st["case"], st["ctx"]
    b, R, H, KH, D = c["batch"], _rows(c), c["q_heads"], c["kv_heads"], c["D"]
    pos = torch.arange(c["ctx"], device=DEV)
    block, slot = st["table"][:, pos // c["page"]].long().clamp(min=0), pos % c["page"]
    cached = pos < ctx[:, None]                                     # [b, L]

    def keys(x):
        old = _values(st[x + "_cache"][block, slot], st[x + "_scale"][block, slot])
        old = torch.where(cached[:, :, None, None], old, 0.0)
        return torch.cat([old, st[x + "_new"].float()], 1).permute(0, 2, 1, 3)  # [b, KH, L + R, D]

    q = st["q"].float().view(b, R, KH, H // KH, D).permute(0, 2, 1, 3, 4).reshape(b, KH, -1, D)
    s = q @ keys("k").transpose(2, 3) * D ** -0.5
    sees = torch.cat([cached[:, None, :].expand(b, R, -1), _paths(st["parent"]) > 0], 2)      # [b, R, L + R]
    s = s.view(b, KH, R, H // KH, -1).masked_fill_(~sees[:, None, :, None, :], -INF)
    s = torch.exp(s - s.amax(-1, keepdim=True))
    s = (s / s.sum(-1, keepdim=True)).view(b, KH, R * (H // KH), -1)
    out = (s @ keys("v")).view(b, KH, R, H // KH, D).permute(0, 2, 1, 3, 4).reshape(b, R, H, D)
    live = torch.arange(R, device=DEV) <= st["count"][:, None]
    st["out"] = torch.where(live[:, :, None, None], out.to(st["q"].dtype), st["out"])
    return {"out": st["out"]}


def _unpacked(words, V):
    return ((words[..., None] >> torch.arange(32, device=DEV)) & 1).flatten(-2)[..., :V] > 0


def _processed(st, row, said):
    """The processed logits of one row of every sequence in float32, [batch, V]; `said`: its path's tokens, -1 where there is none."""
    each = torch.arange(row.shape[0], device=DEV)
    x, V = st["logits"][each, row].float(), st["logits"].shape[2]
    c = st["counts"].scatter_add(1, said.clamp(min=0), (said >= 0).int())
    seen = _unpacked(st["seen"], V) | (c > 0)
    rep, pres, freq = (st[k][:, None] for k in ("repetition", "presence", "frequency"))
    x = torch.where(seen, torch.where(x > 0, x / rep, x * rep), x)
    x = x - freq * c.float()
    x = x - torch.where(c > 0, pres, 0.0)
    x = x + torch.where(st["bias_row"][:, None] >= 0, st["bias"][st["bias_row"].long().clamp(min=0)], 0.0)
    mask = st["mask_row"][each, row].long()
    return x.masked_fill_(~(_unpacked(st["allowed"][mask.clamp(min=0)], V) | (mask < 0)[:, None]), -INF)


def _plain_sampled(st):
    """From the root down, a level at a time: the drafted tokens of a row come first, in the order of their nodes, then all others
    by number; the one in whose share of the row's mass the random number falls is emitted."""
    m, b, n = st["meta"], st["logits"].shape[0], st["uniform"].shape[1] - 1
    each, M, V = torch.arange(b, device=DEV), m["tok"].shape[1], st["logits"].shape[2]
    row, on = torch.zeros((b,), dtype=torch.int64, device=DEV), torch.ones((b,), dtype=torch.bool, device=DEV)
    said = torch.full((b, n + 1), -1, dtype=torch.int64, device=DEV)
    path, logp = said.clone(), torch.zeros((b, n + 1), device=DEV)
    tok, exists = m["tok"].long().clamp(min=0), torch.arange(M, device=DEV) < m["count"][:, None]
    T = st["temperature"].double()[:, None]
    for level in range(n + 1):
        x = _processed(st, row, said)
        top = x.amax(1, keepdim=True)
        w = torch.where(T > 0, torch.exp((x.double() - top.double()) / T.clamp(min=1e-300)), (x == top).double())
        first = torch.where(x == top, torch.arange(V, device=DEV), V).amin(1)
        w = torch.where((T > 0) | (torch.arange(V, device=DEV) == first[:, None]), w, 0.0)
        total = w.sum(1, keepdim=True)
        at = st["uniform"][:, level:level + 1].double() * total
        child = exists & (m["parent"] + 1 == row[:, None]) & (level < n)
        wc = torch.where(child, w.gather(1, tok), 0.0)
        cum = wc.cumsum(1)
        hit = child & (wc > 0) & (at < cum)
        got = torch.where(hit, torch.arange(M, device=DEV), M).amin(1) if M else torch.zeros_like(row)
        down = (got < M) if M else torch.zeros_like(on)
        others = torch.where(torch.zeros_like(w).scatter_add(1, tok, child.double()) > 0, 0.0, w)
        rest = others.cumsum(1)
        pick = (rest <= at - (cum[:, -1:] if M else 0.0)).sum(1)
        pick = torch.minimum(pick, torch.where(others > 0, torch.arange(V, device=DEV), 0).amax(1))
        token = torch.where(down, tok.gather(1, got.clamp(max=max(M - 1, 0))[:, None])[:, 0], pick) if M else pick
        share = torch.log(w[each, token] / total[:, 0]).float()
        said[:, level] = torch.where(on, token, -1)
        path[:, level] = torch.where(on, row, -1)
        logp[:, level] = torch.where(on, share, 0.0)
        on = on & down
        row = torch.where(on, got + 1, 0)
    kept = said >= 0
    a = kept.sum(1) - 1
    st["counts"].scatter_add_(1, said.clamp(min=0), kept.int())
    bits = torch.zeros((b, 32 * st["seen"].shape[1]), dtype=torch.int64, device=DEV)
    bits.scatter_add_(1, said.clamp(min=0), kept.long())
    st["seen"].bitwise_or_(_bits((bits > 0).long()))
    got = {"accept_len": a, "out_tokens": said, "n_out": a + 1, "path_row": path}
    return {**{k: v.to(torch.int32) for k, v in got.items()}, "out_logp": logp, "counts": st["counts"], "seen": st["seen"]}


_PLAIN = {"rotate": _plain_rotate, "append": _plain_append, "pack": _plain_pack, "load": _plain_load, "attention": _plain_attention,
          "sampled": _plain_sampled}


# ---- what one pass cannot do without ----------------------------------------------------------------------------

def work(case):
    kind, size = case["kind"], 2 if case.get("dtype", "bf16") == "bf16" else 4
    if kind == "rotate":
        rows = sum(1 + len(_nodes(t)) for t in _shape(case)[0]) if case["batch"] else case["tokens"]
        return {"bytes": 2 * size * rows * (case["q_heads"] + case["kv_heads"]) * case["D"] + 4 * rows * (1 + case["rot"]), "flops": 0}
    if kind in ("append", "pack", "load"):
        values = 2 * case.get("layers", 1) * case["tokens"] * case["kv_heads"] * case["D"]
        table = case["tokens"] * (8 + 4 * case.get("rot", 0))
        four = 0.5 + 1 / 32
        # (pack: rows in, codes and scales out; and back)
        each = 2 * size if kind == "append" else 2 * (size + four) if kind == "pack" else size + four
        return {"bytes": values * each + table, "flops": 0}
    if kind == "attention":
        trees, ctx = _shape(case)
        nodes = [_nodes(t) for t in trees]
        rows = sum(1 + len(n) for n in nodes)
        # (trees and lengths are dealt out apart: the mean of all pairings)
        pairs = sum(ctx) / len(ctx) * rows + sum(1 + sum(1 + len(p) for p in n) for n in nodes)
        data = case["D"] * (2 * case["kv_heads"] * ((0.5 + 1 / 32) * sum(ctx) + 2 * rows) + 4 * case["q_heads"] * rows)
        data += 4 * sum(2 + -(-n // case["page"]) for n in ctx) + 4 * rows
        return {"bytes": data, "flops": 4 * case["D"] * case["q_heads"] * pairs}
    # the rows of the kept path: about 0.6 of the drafted tokens that come to it are kept
    b, V, n = case["batch"], case["V"], len(_stages(case))
    rows = b * sum(0.6 ** i for i in range(n + 1))
    return {"bytes": rows * (V * size + V / 8 + V / 32 + V) + 4 * rows * min(case["past"], V), "flops": 0}


# ---- the definitions in 64 bits ---------------------------------------------------------------------------------

def exact(case, seed):
    st = prepare(case, seed)
    return _EXACT[case["kind"]](st)


def _exact_heads(x, weight, cos, sin, pos, pairs):
    """Heads [rows, heads, D] normed and turned in 64 bits, pair by pair as complex numbers."""
    x = x.double()
    if weight is not None:
        x = x / torch.sqrt((x * x).sum(-1, keepdim=True) / x.shape[-1] + EPS) * weight.double()
    if cos is None:
        return x
    turn = torch.complex(cos[pos].double(), sin[pos].double())[:, None, :]
    half = turn.shape[-1]
    first = torch.arange(half, device=DEV) * (2 if pairs else 1)
    second = first + (1 if pairs else half)
    z = torch.complex(x.index_select(-1, first), x.index_select(-1, second)) * turn
    y = x.clone()
    y.index_copy_(-1, first, z.real.contiguous())
    y.index_copy_(-1, second, z.imag.contiguous())
    return y


def _exact_rotate(st):
    c, got = st["case"], {}
    for x in "qk":
        out = torch.zeros(st[x].shape, dtype=torch.float64, device=DEV)
        for b in range(out.shape[0]):
            if "pos" in st:
                pos = st["pos"][b].long()
            else:
                pos = torch.tensor([int(st["ctx"][b])] + [int(st["ctx"][b]) + d for d in st["depth"][b, :int(st["count"][b])].tolist()], device=DEV)
            out[b, :len(pos)] = _exact_heads(st[x][b, :len(pos)], st[x + "_weight"], st["cos"], st["sin"], pos, c["pairs"])
        got[x] = out
    return got


def _exact_rows(st, layer):
    T = st["case"]["tokens"]
    src = torch.arange(T, device=DEV) if st["src"] is None else st["src"][:T].long()
    weight = None if st["k_weight"] is None else st["k_weight"][layer]
    k = _exact_heads(st["k_new"][layer].index_select(0, src), weight, st["cos"], st["sin"], st["pos"][:T].long(), st["case"]["pairs"])
    return k, st["v_new"][layer].index_select(0, src).double()


def _exact_append(st):
    got = {"k": st["k_cache"].double(), "v": st["v_cache"].double()}
    for layer in range(st["case"]["layers"]):
        for x, new in zip("kv", _exact_rows(st, layer)):
            got[x][layer].flatten(0, 1).index_copy_(0, st["slot"][:st["case"]["tokens"]].long(), new)
    return got


def _exact_pack(st):
    """The nearest of the amounts that four bits can say, of two as near the one with the even code."""
    amounts, got = [0, 0.5, 1, 1.5, 2, 3, 4, 6], {"k": [], "v": []}
    for layer in range(st["case"]["layers"]):
        for x, new in zip("kv", _exact_rows(st, layer)):
            y = new.unflatten(-1, (-1, 32))
            most = y.abs().amax(-1, keepdim=True)
            mantissa, e = torch.frexp(most)                      # most = mantissa * 2^e, mantissa in [0.5, 1)
            e = torch.where(most > 0, e - 3 + (mantissa > 0.875).int(), -125).clamp(-125, 125)
            z = torch.ldexp(y.abs(), -e)
            value, error = torch.zeros_like(z), z.clone()
            for i, a in enumerate(amounts):
                off = (z - a).abs()
                nearer = (off < error) | ((off == error) & (i % 2 == 0))
                value, error = torch.where(nearer, float(a), value), torch.where(nearer, off, error)
            got[x].append((torch.ldexp(value, e) * torch.sign(y)).flatten(-2))
    return {x: torch.stack(v) for x, v in got.items()}


def _exact_values(codes, scale):
    """[tokens, heads, D] of codes and scales, element by element from the formats' definition."""
    D = 2 * codes.shape[-1]
    d = torch.arange(D, device=DEV)
    code = (codes.index_select(-1, d // 2).int() >> (d % 2 * 4)) & 15
    low = code & 1
    high = (code >> 1) & 3
    amount = torch.where(high == 0, 0.5 * low, torch.ldexp(1 + 0.5 * low.double(), high - 1))
    amount = torch.where(code >= 8, -amount, amount)
    return torch.ldexp(amount.double(), scale.index_select(-1, d // 32).int() - 127)


def _exact_load(st):
    flat = {k: st[k].flatten(0, 1).index_select(0, st["slot"].long()) for k in ("k_cache", "k_scale", "v_cache", "v_scale")}
    return {x: _exact_values(flat[x + "_cache"], flat[x + "_scale"]) for x in "kv"}


def _exact_path(parent, node):
    """Rows that node's row sees: itself, its ancestors, the root."""
    rows = [0]
    while node >= 0:
        rows.append(node + 1)
        node = parent[node]
    return rows


def _exact_attention(st):
    c, out = st["case"], torch.zeros(st["q"].shape, dtype=torch.float64, device=DEV)
    group = c["q_heads"] // c["kv_heads"]
    for b, (length, count, parent) in enumerate(zip(st["ctx"].tolist(), st["count"].tolist(), st["parent"].tolist())):
        t = torch.arange(length, device=DEV)
        block = st["table"][b][t // c["page"]].long()
        R = 1 + count
        see = torch.zeros((R, length + R), dtype=torch.bool)
        see[:, :length] = True
        for r in range(R):
            see[r, [length + x for x in _exact_path(parent, r - 1)]] = True
        see = see.to(DEV)
        k, v = (torch.cat([_exact_values(st[x + "_cache"][block, t % c["page"]], st[x + "_scale"][block, t % c["page"]]), st[x + "_new"][b, :R].double()])
                for x in "kv")
        for h in range(c["kv_heads"]):
            q = st["q"][b, :R, h * group:(h + 1) * group].double().transpose(0, 1).contiguous()       # [group, R, D]
            s = torch.matmul(q, k[:, h].t().contiguous()) / math.sqrt(c["D"])
            s[:, ~see] = -INF
            out[b, :R, h * group:(h + 1) * group] = torch.matmul(torch.softmax(s, -1), v[:, h].contiguous()).transpose(0, 1)
    return {"out": out}


def _exact_sampled(st):
    """Log-probabilities of the emitted tokens, sequence by sequence; everything else is whole numbers."""
    m, (b, R, V), n = st["meta"], st["logits"].shape, st["uniform"].shape[1] - 1
    logp, bits = torch.zeros((b, n + 1), dtype=torch.float64, device=DEV), torch.arange(V, device=DEV)
    for q in range(b):
        parent, tok, count = m["parent"][q].tolist(), m["tok"][q].tolist(), int(m["count"][q])
        rep, pres, freq, T = (float(st[k][q]) for k in ("repetition", "presence", "frequency", "temperature"))
        heard = (st["seen"][q][bits // 32] >> (bits % 32)) & 1
        c, row = st["counts"][q].double(), 0
        for level in range(n + 1):
            x = st["logits"][q, row].double()
            x = torch.where((heard > 0) | (c > 0), torch.where(x > 0, x / rep, x * rep), x) - freq * c - pres * (c > 0)
            if int(st["bias_row"][q]) >= 0:
                x = x + st["bias"][int(st["bias_row"][q])].double()
            mask = int(st["mask_row"][q, row])
            if mask >= 0:
                x[((st["allowed"][mask][bits // 32] >> (bits % 32)) & 1) == 0] = -INF
            if T > 0:
                p = torch.softmax(x / T, 0)
            else:
                p = (bits == int(torch.argmax(x))).double()
            drafted = [i for i in range(count) if parent[i] == row - 1] if level < n else []
            order = [tok[i] for i in drafted]
            u, end, next_row = float(st["uniform"][q, level]), 0.0, None
            for i, t in zip(drafted, order):
                end += float(p[t])
                if u < end and float(p[t]) > 0:
                    next_row, token = i + 1, t
                    break
            if next_row is None:
                left = p.clone()
                left[order] = 0
                token = min(int((torch.cumsum(left, 0) <= u - end).sum()), int((left > 0).nonzero().max()))
            logp[q, level] = torch.log(p[token])
            if next_row is None:
                break
            row = next_row
            c[token] += 1
    none = {k: None for k in ("accept_len", "out_tokens", "n_out", "path_row", "counts", "seen")}
    return {**none, "out_logp": logp}


_EXACT = {"rotate": _exact_rotate, "append": _exact_append, "pack": _exact_pack, "load": _exact_load, "attention": _exact_attention,
          "sampled": _exact_sampled}
