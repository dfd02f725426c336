"""The operators around the base model's forward over a candidate tree, as a serving program calls them in every step.

A case is a dict of plain values.  `kind` names the operator:

  attention  spec_tree_attention: the rows of a token tree attend to a paged key/value cache and to their own ancestors
  extend     spec_cache_extend: block tables and slot maps from the sequences' lengths
  store      spec_cache_store: keys and values of the kept rows of all layers into their slots
  penalize   spec_penalize: repetition, presence and frequency penalties, biases and grammar masks on logits
  verify     spec_verify_tree: the same on the fly, first maximum of every row, and the accepted path

Sequence q has `R` rows: row 0 is the token sampled last, row 1 + i is node i of its tree.  `tree` is the branching per
stage and `B` the candidates kept, whose distinct prefixes are the nodes; tree "" is plain decoding of one token.
Lengths follow from the case alone and are dealt out to the sequences by the seed.
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


def _attention(name, q_heads, kv_heads, D, tree, B, batch, ctx, page, dtype="bf16"):
    return {"name": name, "kind": "attention", "q_heads": q_heads, "kv_heads": kv_heads, "D": D, "tree": tree, "B": B,
            "batch": batch, "ctx": ctx, "page": page, "dtype": dtype}


def _extend(name, batch, what, most, page):
    return {"name": name, "kind": "extend", "batch": batch, "what": what, "most": most, "page": page}


def _store(name, layers, kv_heads, D, tokens, rows, page, dtype="bf16"):
    return {"name": name, "kind": "store", "layers": layers, "kv_heads": kv_heads, "D": D, "tokens": tokens, "rows": rows,
            "page": page, "dtype": dtype}


def _logits(name, kind, V, tree, B, batch, past, dtype):
    return {"name": name, "kind": kind, "V": V, "tree": tree, "B": B, "batch": batch, "past": past, "dtype": dtype}


def listed():
    return [
        # one user of a 7B model, a short conversation: latency
        _attention("attention_7b_b1", 32, 32, 128, "5,3,2", 16, 1, 600, 16),
        # a full batch of the largest model, grouped heads, a wide tree: the matrix cores' work
        _attention("attention_70b_b32", 64, 8, 128, "6,4,3,2", 16, 32, 4000, 64),
        # code model with one shared key/value head on a loaded server: single chains over long files, odd pages
        _attention("attention_20b_chain", 48, 1, 128, "1,1,1,1,1", 1, 24, 16000, 48),
        # float32 models: ragged batch, small heads
        _attention("attention_f32", 12, 4, 80, "4,3,2", 24, 7, 1500, 16, "f32"),
        # every decoding step: one to four tokens more per sequence, a few new blocks, rows picked along the kept paths
        _extend("extend_step_b64", 64, "step", 4, 16),
        # admission of prompts into an empty server, others end and give their blocks back
        _extend("extend_prompts_b48", 48, "prompts", 6000, 16),
        # the step's kept rows of one user, all layers at once
        _store("store_step_b1", 32, 32, 128, 3, 49, 16),
        # a chunk of prompts, packed
        _store("store_prompt", 8, 8, 128, 16000, 0, 64),
        # one user's tree before sampling
        _logits("penalize_7b_b1", "penalize", 32000, "5,3,2", 16, 1, 500, "f32"),
        # a batch of plain decoding with an odd vocabulary, bf16 logits
        _logits("penalize_odd_b64", "penalize", 32003, "", 1, 64, 3000, "bf16"),
        # one user's tree: the smallest verification
        _logits("verify_7b_b1", "verify", 32000, "5,3,2", 16, 1, 500, "f32"),
        # a full batch of the largest vocabulary
        _logits("verify_70b_b32", "verify", 128256, "6,4,3,2", 16, 32, 2000, "bf16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choices(["attention", "extend", "store", "penalize", "verify"], [40, 15, 15, 15, 15])[0]
    tree, B = rng.choice(TREES)
    if kind == "attention":
        dtype = "f32" if rng.random() < 0.2 else "bf16"
        q_heads, kv_heads = rng.choice(HEADS)
        D = rng.choice([128, 128, 64, 8 * rng.randint(4, 32)])
        c = _attention("", q_heads, kv_heads, D, tree, B, _log_int(rng, 1, 64), _log_int(rng, 1, 40000),
                       rng.choice([16, 32, 64, 128, 256, rng.randint(1, 200)]), dtype)
        # (no dearer than the largest listed one)
        part = 0.1 if dtype == "f32" else 1.0
        while c["batch"] * c["ctx"] * max(q_heads * _rows(c) / 4e10, kv_heads / 3e8) * D > part:
            c["ctx"], c["batch"] = max(1, c["ctx"] * 2 // 3), max(1, c["batch"] * 3 // 4)
    elif kind == "extend":
        what = rng.choice(["step", "prompts"])
        c = _extend("", _log_int(rng, 1, 300), what, rng.randint(2, 8) if what == "step" else _log_int(rng, 20, 8000),
                    rng.choice([16, 32, 64, 128, rng.randint(1, 100)]))
        while what == "prompts" and c["batch"] * c["most"] > 300000:
            c["batch"] = max(1, c["batch"] // 2)
    elif kind == "store":
        rows = rng.choice([0, 8, 49, 65])
        c = _store("", rng.randint(1, 40), rng.choice([1, 4, 8, 32, 40]), rng.choice([128, 64, 8 * rng.randint(4, 32)]),
                   _log_int(rng, 1, 16000) if rows == 0 else _log_int(rng, 1, 250), rows, rng.choice([16, 64, rng.randint(1, 100)]),
                   rng.choice(["bf16", "bf16", "f32"]))
        size = 2 if c["dtype"] == "bf16" else 4
        while c["layers"] * c["kv_heads"] * c["D"] * size * max(c["tokens"], 8 * rows) > 2.6e8:
            c["layers"], c["tokens"] = max(1, c["layers"] // 2), max(1, c["tokens"] // 2)
    else:
        c = _logits("", kind, rng.choice([32000, 32016, 49152, 128256, rng.randint(1000, 130000)]), tree, B,
                    _log_int(rng, 1, 64), _log_int(rng, 1, 8000), rng.choice(["f32", "bf16"]))
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
        leaves = list(leaves)
        leaves.sort()
        rng.shuffle(leaves)
        got.append(leaves)
    return got


def _shape(case):
    """The trees and cached lengths of a case: its lengths spread over a factor of eight and more, one of them whole, and
    one new sequence with nothing cached."""
    rng = random.Random(json_key(case))
    most = case.get("ctx", 1)
    ctx = [max(1, int(most * math.exp(-2.2 * rng.random() ** 2))) for _ in range(case["batch"])]
    ctx[0] = most
    if case["batch"] > 4:
        ctx[1] = 0
    return _trees(case, rng), ctx


def json_key(case):
    return ";".join("%s=%s" % (k, case[k]) for k in sorted(case) if k != "name")


def _nodes(leaves):
    """Distinct prefixes in order of first appearance: {prefix: number}."""
    node = {}
    for leaf in leaves:
        for p in range(len(leaf)):
            node.setdefault(leaf[:p + 1], len(node))
    return node


def _metadata(case, trees, V, rng):
    """Candidate tokens and the token tree's tables, as spec_tree_metadata writes them."""
    b, B, n = case["batch"], case["B"], len(_stages(case))
    M = B * n
    cand = torch.zeros((b, B, n), dtype=torch.int32)
    of_cand = torch.zeros((b, B, n), dtype=torch.int32)
    tok, parent = torch.full((b, M), -1, dtype=torch.int32), torch.full((b, M), -1, dtype=torch.int32)
    count = torch.zeros((b,), dtype=torch.int32)
    for q, leaves in enumerate(trees):
        node, token = _nodes(leaves), {}
        count[q] = len(node)
        for prefix, i in node.items():
            family = token.setdefault(prefix[:-1], rng.sample(range(V), 8))
            tok[q, i] = family[prefix[-1]]
            parent[q, i] = node.get(prefix[:-1], -1)
        for c, leaf in enumerate(leaves):
            for p in range(n):
                of_cand[q, c, p] = node[leaf[:p + 1]]
                cand[q, c, p] = tok[q, node[leaf[:p + 1]]]
    return {k: v.to(DEV) for k, v in dict(cand=cand, of_cand=of_cand, tok=tok, parent=parent, count=count).items()}


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


def _prepare_attention(case, g, rng):
    dt, b, D, R = _dtype(case), case["batch"], case["D"], _rows(case)
    trees, ctx = _shape(case)
    rng.shuffle(trees)
    rng.shuffle(ctx)
    meta = _metadata(case, trees, 32000, rng)
    table, pool = _pages(ctx, case["page"], 8, g)

    def rand(*shape):
        return torch.randn(shape, generator=g, device=DEV).to(dt)

    # (keys a little alike, so that the softmax neither spreads evenly nor picks one)
    st = {"k_cache": rand(pool, case["page"], case["kv_heads"], D), "v_cache": rand(pool, case["page"], case["kv_heads"], D),
          "k_new": rand(b, R, case["kv_heads"], D), "v_new": rand(b, R, case["kv_heads"], D),
          "q": rand(b, R, case["q_heads"], D) * 1.5, "table": table, "ctx": torch.tensor(ctx, **I32),
          "parent": meta["parent"], "count": meta["count"]}
    st["out"] = torch.zeros_like(st["q"])
    return st


def _prepare_extend(case, g, rng):
    b, page, most = case["batch"], case["page"], case["most"]
    plan = random.Random(json_key(case))
    if case["what"] == "step":
        # kept rows 1 .. most; a few sequences wait
        old = [plan.randint(1, 4000) for _ in range(b)]
        add = [plan.randint(0, most) if plan.random() < 0.9 else 0 for _ in range(b)]
    else:
        # two thirds start with a prompt, the others end
        start = [plan.random() < 0.67 or q == 0 for q in range(b)]
        old = [0 if s else plan.randint(1, most) for s in start]
        add = [max(1, int(most * math.exp(-2.0 * plan.random()))) if s else -n for s, n in zip(start, old)]
    both = list(zip(old, add))
    rng.shuffle(both)
    old, add = [n for n, _ in both], [a for _, a in both]
    width = max(1, -(-max(n + max(a, 0) for n, a in both) // page))
    held = [-(-n // page) for n in old]
    free = sum(max(0, -(-(n + a) // page) - h) for (n, a), h in zip(both, held)) + 5
    pool = sum(held) + free
    at = torch.randperm(pool, generator=g, device=DEV).to(torch.int32)
    table = torch.full((b, width), -1, **I32)
    first = 0
    for q, h in enumerate(held):
        table[q, :h] = at[first:first + h]
        first += h
    head = rng.randrange(pool)
    ring = torch.full((pool,), -1, **I32)
    ring[(head + torch.arange(free, device=DEV)) % pool] = at[first:]
    cap = sum(max(a, 0) for a in add) + 7
    st = {"old": torch.tensor(old, **I32), "add": torch.tensor(add, **I32), "table": table, "ring": ring,
          "state": torch.tensor([head, free], **I32), "new": torch.zeros((b,), **I32), "added": torch.zeros((b,), **I32),
          "state_new": torch.zeros((2,), **I32), "row_start": torch.zeros((b + 1,), **I32),
          "slot": torch.zeros((cap,), **I32), "pos": torch.zeros((cap,), **I32)}
    if case["what"] == "step":
        path = [[0] + sorted(rng.sample(range(1, 48), most - 1)) for _ in range(b)]
        st["path"], st["src"] = torch.tensor(path, **I32), torch.zeros((cap,), **I32)
    return st


def _prepare_store(case, g, rng):
    dt, L, H, D, T = _dtype(case), case["layers"], case["kv_heads"], case["D"], case["tokens"]
    shape = (H, D)
    # rows = 0: a packed prompt, every row is kept; otherwise kept rows of trees of so many rows, up to four of each
    rows = T if case["rows"] == 0 else case["rows"] * -(-T // 4)
    pages = -(-2 * T // case["page"]) + 2

    def rand(*s):
        return torch.randn(s, generator=g, device=DEV).to(dt)

    st = {"k_cache": rand(L, pages, case["page"], *shape), "v_cache": rand(L, pages, case["page"], *shape),
          "k_new": rand(L, rows, *shape), "v_new": rand(L, rows, *shape)}
    # consecutive slots within a page, pages in any order; two entries behind the last token
    order = torch.randperm(pages, generator=g, device=DEV)[: -(-T // case["page"])]
    slots = (order[:, None] * case["page"] + torch.arange(case["page"], device=DEV)).reshape(-1)[:T]
    st["slot"] = torch.cat([slots, torch.full((2,), -1, device=DEV)]).to(torch.int32)
    st["src"] = None
    if case["rows"]:
        src = torch.randperm(rows, generator=g, device=DEV)[:T].sort()[0]
        st["src"] = torch.cat([src, torch.zeros((2,), device=DEV, dtype=src.dtype)]).to(torch.int32)
    else:
        st["k_new"], st["v_new"] = (torch.cat([x, x[:, :2]], 1) for x in (st["k_new"], st["v_new"]))
    return st


def _prepare_logits(case, g, rng):
    b, V, R, past = case["batch"], case["V"], _rows(case), case["past"]
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
    logits = torch.randn((b, R, V), generator=g, device=DEV)
    if R > 1:
        # the base model agrees with one child of most nodes
        row = (meta["parent"] + 1).long()
        boost = torch.where((meta["tok"] >= 0) & (uniform(b, R - 1) < 0.5), 6.0, 0.0)
        logits.view(b, -1).scatter_add_(1, row * V + meta["tok"].long().clamp(min=0), boost)
    # grammar masks for the rows of a fourth of the sequences, each of its own rows; biases for as many others
    bound = torch.arange(b, device=DEV) % 4 == 0
    rows_bound = (-(-b // 4)) * R
    mask_row = torch.where(bound[:, None], (torch.arange(b, device=DEV) // 4)[:, None] * R + torch.arange(R, device=DEV), -1)
    allowed = uniform(rows_bound, 32 * words) < 0.3
    own_bias = torch.arange(b, device=DEV) % 4 == 1
    st = {"logits": logits.to(_dtype(case)), "counts": counts, "seen": _pack(seen), "allowed": _pack(allowed.long()),
          "mask_row": mask_row.to(torch.int32).contiguous(),
          "bias": torch.where(uniform(-(-b // 4), V) < 0.01, 4 * uniform(-(-b // 4), V) - 2, 0.0),
          "bias_row": torch.where(own_bias, torch.arange(b, device=DEV) // 4, -1).to(torch.int32),
          "repetition": 1.0 + 0.3 * uniform(b), "presence": 0.5 * uniform(b), "frequency": 0.2 * uniform(b), "meta": meta}
    if case["kind"] == "penalize":
        st["out"] = torch.zeros_like(st["logits"])
    else:
        n = len(_stages(case))
        st["outs"] = {"greedy": torch.zeros((b, R), **I32), "accept_len": torch.zeros((b,), **I32),
                      "best_cand": torch.zeros((b,), **I32), "out_tokens": torch.zeros((b, n + 1), **I32),
                      "n_out": torch.zeros((b,), **I32), "path_row": torch.zeros((b, n + 1), **I32)}
    return st


def _pack(bits):
    """Truth values [rows, 32 * words] as words of 32 bits, the lowest bit first."""
    x = (bits.view(bits.shape[0], -1, 32) << torch.arange(32, device=DEV)).sum(2)
    return torch.where(x >= 2 ** 31, x - 2 ** 32, x).to(torch.int32)


_PREPARE = {"attention": _prepare_attention, "extend": _prepare_extend, "store": _prepare_store,
            "penalize": _prepare_logits, "verify": _prepare_logits}


# ---- one pass ---------------------------------------------------------------------------------------------------

def run(st):
    return (_OWN if own else _PLAIN)[st["case"]["kind"]](st)


def _own_attention(st):
    from paper_2404_19124_amd import binding as S
    c = st["case"]
    if "workspace" not in st:
        st["workspace"] = torch.empty(S.spec_tree_attention_workspace(c["batch"], _rows(c), c["q_heads"], c["kv_heads"],
                                                                      c["D"], st["q"].dtype), dtype=torch.uint8, device=DEV)
    S.spec_tree_attention(st["q"], st["k_new"], st["v_new"], st["k_cache"], st["v_cache"], st["table"], st["ctx"],
                          st["parent"], st["count"], st["out"], st["workspace"])
    return {"out": st["out"]}


def _own_extend(st):
    from paper_2404_19124_amd import binding as S
    S.spec_cache_extend(st["old"], st["add"], st["new"], st["added"], st["table"], st["ring"], st["state"], st["state_new"],
                        st["case"]["page"], st["row_start"], st["slot"], st["pos"], path_row=st.get("path"),
                        seq_rows=48 if "path" in st else 0, src_row=st.get("src"))
    return {k: st[k] for k in ("new", "added", "table", "ring", "state_new", "row_start", "slot", "pos", "src") if k in st}


def _own_store(st):
    from paper_2404_19124_amd import binding as S
    S.spec_cache_store(st["k_new"], st["v_new"], st["slot"], st["k_cache"], st["v_cache"], src_row=st["src"])
    return {"k": st["k_cache"], "v": st["v_cache"]}


_PENALTIES = ("counts", "seen", "repetition", "presence", "frequency", "bias", "bias_row", "allowed", "mask_row")


def _own_penalize(st):
    from paper_2404_19124_amd import binding as S
    m = st["meta"]
    S.spec_penalize(st["logits"], st["out"], {k: st[k] for k in _PENALTIES}, m["tok"], m["parent"], m["count"])
    return {"out": st["out"]}


def _own_verify(st):
    from paper_2404_19124_amd import binding as S
    m, o = st["meta"], st["outs"]
    S.spec_verify_tree(st["logits"], m["cand"], m["of_cand"], m["count"], o["greedy"], o["accept_len"], o["best_cand"],
                       o["out_tokens"], o["n_out"], o["path_row"], penalties={k: st[k] for k in _PENALTIES},
                       node_tok=m["tok"], node_parent=m["parent"], update=True)
    return {**o, "counts": st["counts"], "seen": st["seen"]}


_OWN = {"attention": _own_attention, "extend": _own_extend, "store": _own_store, "penalize": _own_penalize,
        "verify": _own_verify}


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
    block = st["table"][:, pos // c["page"]].long().clamp(min=0)
    cached = pos < ctx[:, None]                                     # [b, L]

    def keys(cache, new):
        old = torch.where(cached[:, :, None, None], cache[block, pos % c["page"]].float(), 0.0)
        return torch.cat([old, new.float()], 1).permute(0, 2, 1, 3)  # [b, KH, L + R, D]

    q = st["q"].float().view(b, R, KH, H // KH, D).permute(0, 2, 1, 3, 4).reshape(b, KH, -1, D)
    s = q @ keys(st["k_cache"], st["k_new"]).transpose(2, 3) * D ** -0.5
    sees = torch.cat([cached[:, None, :].expand(b, R, -1), _paths(st["parent"]) > 0], 2)      # [b, R, L + R]
    s = s.view(b, KH, R, H // KH, -1).masked_fill_(~sees[:, None, :, None, :], -INF)
    s = torch.exp(s - s.amax(-1, keepdim=True))
    s = (s / s.sum(-1, keepdim=True)).view(b, KH, R * (H // KH), -1)
    out = (s @ keys(st["v_cache"], st["v_new"])).view(b, KH, R, H // KH, D).permute(0, 2, 1, 3, 4).reshape(b, R, H, D)
    live = torch.arange(R, device=DEV) <= st["count"][:, None]
    st["out"] = torch.where(live[:, :, None, None], out.to(st["q"].dtype), st["out"])
    return {"out": st["out"]}


def _plain_extend(st):
    page, old, add, cap = st["case"]["page"], st["old"].long(), st["add"].long(), st["slot"].shape[0]
    b, width = st["table"].shape
    pool, head, free = st["ring"].shape[0], st["state"][0].long(), st["state"][1].long()
    new = (old + add).clamp(min=0)
    have, want = (old + page - 1) // page, (new + page - 1) // page
    grow = (add > 0) & (new <= width * page)
    blocks, rows = torch.where(grow, want - have, 0), torch.where(grow, add, 0)
    served = grow & (blocks.cumsum(0) <= free) & (rows.cumsum(0) <= cap)
    blocks, rows = torch.where(served, blocks, 0), torch.where(served, rows, 0)
    back = torch.where(add < 0, have - want, 0)
    new = torch.where(served | (add < 0), new, old)
    # blocks out of the ring into the tables, and of what was cut off back behind the ring's end
    at = torch.arange(width, device=DEV)
    first = blocks.cumsum(0) - blocks
    fresh = (at >= have[:, None]) & (at < (have + blocks)[:, None])
    taken = st["ring"][(head + first[:, None] + at - have[:, None]) % pool]
    table = torch.where(fresh, taken, st["table"])
    ring = torch.cat([st["ring"], st["ring"][:1]])                  # (the last entry takes what is not given back)
    given = (at >= want[:, None]) & (at < (want + back)[:, None])
    to = (head + free + (back.cumsum(0) - back)[:, None] + at - want[:, None]) % pool
    ring[torch.where(given, to, pool)] = st["table"]
    state = torch.stack([(head + blocks.sum()) % pool, free - blocks.sum() + back.sum()])
    # tokens, packed
    row_start = torch.cat([torch.zeros_like(rows[:1]), rows.cumsum(0)])
    t = torch.arange(cap, device=DEV)
    seq = torch.searchsorted(row_start[1:], t, right=True).clamp(max=b - 1)
    j = t - row_start[seq]
    pos = old[seq] + j
    live = t < row_start[-1]
    slot = table[seq, (pos // page).clamp(max=width - 1)].long() * page + pos % page
    got = {"new": new, "added": new - old, "table": table, "ring": ring[:pool], "state_new": state, "row_start": row_start,
           "slot": torch.where(live, slot, -1), "pos": torch.where(live, pos, -1)}
    if "path" in st:
        row = st["path"][seq, j.clamp(min=0, max=st["path"].shape[1] - 1)].long()
        got["src"] = torch.where(live, seq * 48 + row, -1)
    return {k: v.to(torch.int32) for k, v in got.items()}


def _plain_store(st):
    slot = st["slot"].long()
    src = torch.arange(slot.shape[0], device=DEV) if st["src"] is None else st["src"].long()
    # (entries without a slot store the first token once more)
    src, to = torch.where(slot < 0, src[0], src), torch.where(slot < 0, slot[0], slot)
    L, pages, page = st["k_cache"].shape[:3]
    for cache, new in ((st["k_cache"], st["k_new"]), (st["v_cache"], st["v_new"])):
        cache.view(L, pages * page, *cache.shape[3:])[:, to] = new[:, src]
    return {"k": st["k_cache"], "v": st["v_cache"]}


def _unpack(words, V):
    return ((words[..., None] >> torch.arange(32, device=DEV)) & 1).flatten(-2)[..., :V] > 0


def _processed(st):
    """The processed logits of every row in float32, [batch, R, V]."""
    m, V = st["meta"], st["logits"].shape[2]
    b, R, _ = st["logits"].shape
    c = st["counts"][:, None, :].expand(b, R, V).clone()
    if R > 1:
        tok = m["tok"].long().clamp(min=0)[:, None, :].expand(b, R, R - 1)
        c.scatter_add_(2, tok, (_paths(m["parent"])[:, :, 1:].int() * (m["tok"] >= 0)[:, None, :].int()))
    x = st["logits"].float()
    seen = _unpack(st["seen"], V)[:, None, :] | (c > 0)
    rep, pres, freq = (st[k][:, None, None] for k in ("repetition", "presence", "frequency"))
    x = torch.where(seen, torch.where(x > 0, x / rep, x * rep), x)
    x = x - freq * c.float()
    x = x - torch.where(c > 0, pres, 0.0)
    x = x + torch.where(st["bias_row"][:, None] >= 0, st["bias"][st["bias_row"].long().clamp(min=0)], 0.0)[:, None, :]
    row = st["mask_row"].long()
    return x.masked_fill_(~(_unpack(st["allowed"][row.clamp(min=0)], V) | (row < 0)[:, :, None]), -INF)


def _live(st):
    return torch.arange(st["logits"].shape[1], device=DEV) <= st["meta"]["count"][:, None]


def _plain_penalize(st):
    st["out"] = torch.where(_live(st)[:, :, None], _processed(st).to(st["logits"].dtype), st["out"])
    return {"out": st["out"]}


def _plain_verify(st):
    m, x = st["meta"], _processed(st)
    b, R, V = x.shape
    best = torch.where(x == x.amax(-1, keepdim=True), torch.arange(V, device=DEV), V).amin(-1)
    greedy = torch.where(_live(st), best, -1)
    rows = torch.cat([m["of_cand"].new_zeros((b, m["of_cand"].shape[1], 1)), m["of_cand"] + 1], 2).long()   # [b, B, n + 1]
    said = greedy.gather(1, rows.flatten(1)).view_as(rows)
    n = rows.shape[2] - 1
    mine = torch.cat([m["cand"], torch.full_like(rows[:, :, :1], -2)], 2)      # (nothing is speculated behind the last one)
    length = (said == mine).long().cumprod(2).sum(2)
    a = length.amax(1)
    cand = torch.where(length == a[:, None], torch.arange(rows.shape[1], device=DEV), rows.shape[1]).amin(1)
    at, each = torch.arange(n + 1, device=DEV), torch.arange(b, device=DEV)
    path = rows[each, cand]
    bonus = said[each, cand].gather(1, a[:, None])
    out = torch.where(at < a[:, None], mine[each, cand], torch.where(at == a[:, None], bonus, -1))
    kept = at <= a[:, None]
    st["counts"].scatter_add_(1, out.long().clamp(min=0), kept.int())
    bits = torch.zeros((b, 32 * st["seen"].shape[1]), dtype=torch.int64, device=DEV)
    bits.scatter_add_(1, out.long().clamp(min=0), kept.long())
    st["seen"].bitwise_or_(_pack((bits > 0).long()))
    got = {"greedy": greedy, "accept_len": a, "best_cand": cand, "out_tokens": out, "n_out": a + 1,
           "path_row": torch.where(kept, path, -1)}
    return {**{k: v.to(torch.int32) for k, v in got.items()}, "counts": st["counts"], "seen": st["seen"]}


_PLAIN = {"attention": _plain_attention, "extend": _plain_extend, "store": _plain_store, "penalize": _plain_penalize,
          "verify": _plain_verify}


# ---- what one pass cannot do without ----------------------------------------------------------------------------

def work(case):
    size = 2 if case.get("dtype") == "bf16" else 4
    if case["kind"] == "attention":
        trees, ctx = _shape(case)
        nodes = [_nodes(t) for t in trees]
        rows = sum(1 + len(n) for n in nodes)
        # (trees and lengths are dealt out apart: the mean of all pairings)
        pairs = sum(ctx) / len(ctx) * rows + sum(1 + sum(1 + len(p) for p in n) for n in nodes)
        data = size * case["D"] * (2 * case["kv_heads"] * (sum(ctx) + rows) + 2 * case["q_heads"] * rows)
        data += 4 * sum(2 + -(-n // case["page"]) for n in ctx) + 4 * rows
        return {"bytes": data, "flops": 4 * case["D"] * case["q_heads"] * pairs}
    if case["kind"] == "extend":
        st = _counts_of_extend(case)
        return {"bytes": 4 * (4 * case["batch"] + 2 * st["blocks"] + (3 if case["what"] == "step" else 2) * st["tokens"]), "flops": 0}
    if case["kind"] == "store":
        return {"bytes": 2 * 2 * size * case["layers"] * case["tokens"] * case["kv_heads"] * case["D"] + 8 * case["tokens"], "flops": 0}
    rows = sum(1 + len(_nodes(t)) for t in _shape(case)[0])
    b, V = case["batch"], case["V"]
    data = rows * V * size * (2 if case["kind"] == "penalize" else 1) + b * V / 8 + rows / 4 * V / 8 + -(-b // 4) * V * 4
    # (counts of the tokens that were said)
    return {"bytes": data + 4 * b * min(case["past"], V), "flops": 0}


def _counts_of_extend(case):
    plan, page, b, most = random.Random(json_key(case)), case["page"], case["batch"], case["most"]
    if case["what"] == "step":
        old = [plan.randint(1, 4000) for _ in range(b)]
        add = [plan.randint(0, most) if plan.random() < 0.9 else 0 for _ in range(b)]
    else:
        start = [plan.random() < 0.67 or q == 0 for q in range(b)]
        old = [0 if s else plan.randint(1, most) for s in start]
        add = [max(1, int(most * math.exp(-2.0 * plan.random()))) if s else -n for s, n in zip(start, old)]
    return {"tokens": sum(max(a, 0) for a in add), "blocks": sum(abs(-(-(n + a) // page) - -(-n // page)) for n, a in zip(old, add))}


# ---- the definitions in 64 bits ---------------------------------------------------------------------------------

def exact(case, seed):
    st = prepare(case, seed)
    if case["kind"] == "attention":
        return {"out": _exact_attention(st)}
    if case["kind"] == "store":
        return {k: _exact_store(st, k) for k in ("k", "v")}
    if case["kind"] == "penalize":
        return {"out": _exact_penalize(st)}
    return None   # whole numbers only


def _path(parent, node):
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
            see[r, [length + x for x in _path(parent, r - 1)]] = True
        see = see.to(DEV)
        k, v = (torch.cat([x[block, t % c["page"]], y[b, :R]]).double() for x, y in
                ((st["k_cache"], st["k_new"]), (st["v_cache"], st["v_new"])))
        for h in range(c["kv_heads"]):
            q = st["q"][b, :R, h * group:(h + 1) * group].double().transpose(0, 1)       # [group, R, D]
            s = torch.matmul(q, k[:, h].t().contiguous()) / math.sqrt(c["D"])
            s[:, ~see] = -INF
            out[b, :R, h * group:(h + 1) * group] = torch.matmul(torch.softmax(s, -1), v[:, h].contiguous()).transpose(0, 1)
    return out


def _exact_store(st, which):
    cache, new = st[which + "_cache"].double(), st[which + "_new"]
    L, pages, page = cache.shape[:3]
    flat = cache.view(L, pages * page, *cache.shape[3:])
    n = st["case"]["tokens"]
    src = torch.arange(n, device=DEV) if st["src"] is None else st["src"][:n].long()
    flat.index_copy_(1, st["slot"][:n].long(), new.index_select(1, src).double())
    return cache


def _exact_penalize(st):
    m, out = st["meta"], torch.zeros(st["logits"].shape, dtype=torch.float64, device=DEV)
    V = out.shape[2]
    bits = torch.arange(V, device=DEV)
    params = [st[k].tolist() for k in ("repetition", "presence", "frequency", "bias_row", "mask_row")]
    for b, (count, parent, rep, pres, freq, bias, mask) in enumerate(zip(m["count"].tolist(), m["parent"].tolist(), *params)):
        said = (st["seen"][b][bits // 32] >> (bits % 32)) & 1
        for r in range(1 + count):
            c = st["counts"][b].double()
            for row in _path(parent, r - 1)[1:]:
                c[m["tok"][b, row - 1].long()] += 1
            x = st["logits"][b, r].double()
            x = torch.where((said > 0) | (c > 0), torch.where(x > 0, x / rep, x * rep), x) - freq * c - pres * (c > 0)
            if bias >= 0:
                x = x + st["bias"][bias].double()
            if mask[r] >= 0:
                x[((st["allowed"][mask[r]][bits // 32] >> (bits % 32)) & 1) == 0] = -INF
            out[b, r] = x
    return out
