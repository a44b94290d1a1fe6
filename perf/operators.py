"""Cases of the drafted-token operators: what they are given, what they compute, what that costs at least.

Three kinds of call that a decode loop with drafted tokens makes of the library, one after the other:

- ``tree``: the drafted tokens of every request attend over the cache and over their own ancestors, and
  their K / V rows are appended to the cache;
- ``verify``: the drafted tokens are accepted or rejected against the target's probabilities;
- ``compact`` / ``fork`` / ``reserve``: what then happens to the cache -- accepted rows move up, pages are
  shared, copied, taken from the pool and given back.

``run`` computes a case in plain torch operations, or, where ``own`` is true, by the library's calls.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


# ------------------------------------------------------------------------------------------------ the cases
def _tree(name, **kw):
    case = {"name": name, "op": "tree", "dtype": "bf16", "batch": 1, "hq": 32, "hkv": 8, "d": 128, "nodes": 8,
            "branch": 2, "ragged": False, "page": 16, "lo": 1, "hi": 1024, "prompt": 64, "window": 0, "sinks": 0}
    return {**case, **kw}


def _verify(name, **kw):
    case = {"name": name, "op": "verify", "dtype": "f32", "batch": 1, "nodes": 8, "branch": 2, "vocab": 16384,
            "mode": "sample"}
    return {**case, **kw}


def _compact(name, **kw):
    case = {"name": name, "op": "compact", "dtype": "bf16", "batch": 8, "hkv": 8, "d": 128, "layers": 8, "page": 16,
            "lo": 64, "hi": 1024, "span": 32, "ident": 1, "moved": 3, "after": True}
    return {**case, **kw}


def _fork(name, **kw):
    case = {"name": name, "op": "fork", "dtype": "bf16", "batch": 8, "hkv": 8, "d": 128, "layers": 8, "page": 16,
            "lo": 1, "hi": 1024}
    return {**case, **kw}


def listed():
    return [
        # a single user, four tokens drafted in a row: latency
        _tree("tree chain 1x4", batch=1, nodes=4, branch=0, lo=500, hi=700),
        # a small serving batch with grouped heads and long image sequences (90 x 91 tokens) in contiguous caches
        _tree("tree gqa 8x16 long", batch=8, nodes=16, page=0, lo=4096, hi=8190),
        # the paged batch of the library's benchmark (32 heads, 64 x 65 image tokens, 200 of prompt), ragged trees
        _tree("tree mha 32x32 paged", batch=32, hq=32, hkv=32, nodes=32, branch=4, ragged=True, lo=1, hi=4160, prompt=200),
        # the same heads with the sliding window and four first tokens that stay visible
        _tree("tree window 64x16", batch=64, hq=32, hkv=32, nodes=16, lo=1, hi=4160, prompt=200, window=512, sinks=4),
        # many drafted tokens under few kv heads: as much arithmetic as memory
        _tree("tree gqa8 16x64", batch=16, hq=64, hkv=8, nodes=64, branch=3, lo=2048, hi=4160),
        # single precision and narrow heads, for checking a model against its reference
        _tree("tree f32 d64 8x8", dtype="f32", batch=8, hq=20, hkv=20, d=64, nodes=8, page=0, lo=1, hi=1144, prompt=120),
        # one user, a chain of four drafted tokens over an image codebook
        _verify("verify chain 1x5", batch=1, nodes=5, branch=0, vocab=16384, dtype="bf16"),
        # a batch of trees over a text-and-image vocabulary, drafted by sampling
        _verify("verify tree 64x32", batch=64, nodes=32, branch=4, vocab=65536),
        # greedy decoding
        _verify("verify greedy 32x16", batch=32, nodes=16, vocab=65536, mode="greedy"),
        # after the verification: the accepted rows of every layer move up behind the cached ones
        _compact("compact accepted 64", batch=64, layers=16, lo=64, hi=1024, span=32, ident=1, moved=3),
        # a cache that is cut down to its prompt and the rows that a mask keeps
        _compact("compact evicted 16", batch=16, layers=4, hkv=32, lo=2048, hi=4160, span=2048, ident=200, moved=208,
                 after=False),
        # every request is continued by a second one: pages shared, the part-filled last page copied in all layers
        _fork("fork 32", batch=32, layers=16, lo=1, hi=1024),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng):
    op = rng.choice(["tree", "tree", "tree", "verify", "verify", "compact", "fork", "reserve"])
    if op == "tree":
        hkv = rng.choice([1, 2, 3, 8, 20, 32])
        group = rng.choice([1, 2, 4, 8]) if hkv <= 8 else 1
        c = {"op": op, "dtype": rng.choice(["bf16", "bf16", "bf16", "f32"]), "hkv": hkv, "hq": hkv * group,
             "d": rng.choice([64, 128]), "nodes": _log(rng, 1, 64), "branch": rng.choice([0, 1, 2, 4]),
             "ragged": rng.random() < 0.5, "page": rng.choice([0, 1, 5, 16, 24, 64, 128]), "lo": rng.choice([0, 1, 17]),
             "hi": _log(rng, 20, 8192), "prompt": _log(rng, 1, 600), "window": rng.choice([0, 0, 1, 64, 512, 1000]),
             "sinks": rng.choice([0, 4])}
        most = 8 * 8192 * 8 if c["dtype"] == "bf16" else 8 * 8192           # cached (token, kv head) pairs
        c["batch"] = _log(rng, 1, max(1, min(256, most // (c["hkv"] * (c["hi"] + c["nodes"])))))
        return c
    if op == "verify":
        c = {"op": op, "dtype": rng.choice(["f32", "bf16"]), "nodes": _log(rng, 1, 64), "branch": rng.choice([0, 1, 2, 4]),
             "vocab": _log(rng, 2, 131072), "mode": rng.choice(["sample", "sample", "point", "greedy"])}
        c["batch"] = _log(rng, 1, max(1, min(256, 64 * 32 * 65536 // (c["nodes"] * c["vocab"]))))
        return c
    c = {"op": op, "dtype": rng.choice(["bf16", "f32"]), "hkv": rng.choice([1, 3, 8, 32]), "d": rng.choice([64, 128]),
         "layers": rng.choice([1, 2, 5, 8]), "page": rng.choice([1, 5, 16, 24, 64]), "lo": 1, "hi": _log(rng, 200, 2048)}
    if op == "compact":
        c["after"] = rng.random() < 0.5
        c["ident"], c["moved"] = rng.choice([0, 1, 3]) if c["after"] else _log(rng, 1, 40), _log(rng, 1, 60)
        c["span"] = c["ident"] + 2 * c["moved"] + rng.randrange(1, 40)      # positions that the kept ones come from
        c["lo"] = max(c["lo"], c["span"])
        c["hi"] = max(c["hi"], c["lo"])
    if op == "reserve":
        c = {"op": op, "page": c["page"], "lo": 0, "hi": c["hi"], "extra": _log(rng, 1, 64), "batch": _log(rng, 1, 512)}
        return c
    row = c["hkv"] * c["d"] * c["layers"] * (2 if c["dtype"] == "bf16" else 4)
    c["batch"] = _log(rng, 1, max(1, min(128, (1 << 30) // (row * (c["hi"] + c["page"] + c.get("span", 0))))))
    return c


# ------------------------------------------------------------------------------------------------ inputs
def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _ints(g, lo, hi, shape):
    """Whole numbers of [lo, hi], 32 bits."""
    return torch.randint(lo, hi + 1, shape, generator=g, device="cuda", dtype=torch.int32)


def _normal(g, shape, dtype, scale=1.0):
    t = torch.empty(shape, dtype=dtype, device="cuda").normal_(generator=g)
    return t if scale == 1.0 else t.mul_(scale)


def _parents(g, batch, nodes, branch):
    """Parents of a drafted tree: node 0 is the root, parent[i] < i; branch 0: a chain."""
    i = torch.arange(nodes, device="cuda", dtype=torch.int32)[None, :].expand(batch, nodes)
    if branch == 0:
        return (i - 1).contiguous()
    back = (torch.rand((batch, nodes), generator=g, device="cuda") * (2 * branch)).to(torch.int32) + 1
    parent = (i - back).clamp_(min=0)
    parent[:, 0] = -1
    return parent.contiguous()


def _pages_for(g, batch, tokens, page, spare=0):
    """Block table of `batch` rows that hold `tokens` tokens each, in a shuffled pool, and the pool's size."""
    per = -(-tokens // page)
    n = batch * per + spare
    perm = torch.randperm(n, generator=g, device="cuda").to(torch.int32)
    return perm[:batch * per].view(batch, per).contiguous(), n


def _prepare_tree(c, seed):
    g, dt = _gen(seed), DTYPES[c["dtype"]]
    b, n, hq, hkv, d = c["batch"], c["nodes"], c["hq"], c["hkv"], c["d"]
    cap = c["hi"] + n
    s = {"case": c, "cap": cap, "seq_len": _ints(g, c["lo"], c["hi"], (b,))}
    s["prompt_len"] = torch.minimum(s["seq_len"], torch.full_like(s["seq_len"], c["prompt"]))
    if c["page"]:
        s["table"], blocks = _pages_for(g, b, cap, c["page"])
        shape = (blocks, c["page"], hkv, d)
    else:
        s["table"], shape = None, (b, cap, hkv, d)
    s["k"], s["v"] = _normal(g, shape, dt), _normal(g, shape, dt)
    s["q"] = _normal(g, (b, n, hq, d), dt)
    s["k_new"], s["v_new"] = _normal(g, (b, n, hkv, d), dt), _normal(g, (b, n, hkv, d), dt)
    s["parent"] = _parents(g, b, n, c["branch"])
    s["count"] = _ints(g, 0, n, (b,)) if c["ragged"] else torch.full((b,), n, dtype=torch.int32, device="cuda")
    return s


def _prepare_verify(c, seed):
    g, dt = _gen(seed), DTYPES[c["dtype"]]
    b, n, v = c["batch"], c["nodes"], c["vocab"]
    logits = _normal(g, (b, n, v), torch.float32, 2.5)
    s = {"case": c, "parent": _parents(g, b, n, c["branch"])}
    s["target"] = torch.softmax(logits, -1).to(dt)
    draft = torch.softmax(logits.add_(_normal(g, (b, n, v), torch.float32, 0.5)), -1)
    del logits
    # the r-th child of a node has the r-th token that the draft drew there (or the r-th likeliest one)
    most = min(8, v)
    if c["mode"] == "sample":
        drawn = torch.multinomial(draft.view(b * n, v), most, replacement=True, generator=g).view(b, n, most)
    else:
        drawn = draft.topk(most, -1).indices
    parent = s["parent"].long()
    earlier = torch.ones((n, n), device="cuda", dtype=torch.bool).tril(-1)
    rank = ((parent[:, :, None] == parent[:, None, :]) & earlier).sum(-1) % most
    s["tokens"] = drawn[torch.arange(b, device="cuda")[:, None], parent.clamp(min=0), rank].to(torch.int32).contiguous()
    s["draft"] = draft.to(dt) if c["mode"] == "sample" else None
    s["uniforms"] = None if c["mode"] == "greedy" else torch.rand((b, n), generator=g, device="cuda")
    return s


def _prepare_compact(c, seed):
    """Kept positions: `ident` that stay where they are, then `moved` that come from behind the kept region, so
    that moving them leaves their old places as they were and a second call does the same work again."""
    g, dt = _gen(seed), DTYPES[c["dtype"]]
    b, kept = c["batch"], c["ident"] + c["moved"]
    s = {"case": c, "seq_len": _ints(g, c["lo"], c["hi"], (b,))}
    s["prompt_len"] = torch.zeros_like(s["seq_len"])
    s["table"], blocks = _pages_for(g, b, c["hi"] + c["span"], c["page"])
    s["k"] = _normal(g, (c["layers"], blocks, c["page"], c["hkv"], c["d"]), dt)
    s["v"] = _normal(g, s["k"].shape, dt)
    room = c["span"] - kept
    from_behind = torch.rand((b, room), generator=g, device="cuda").argsort(-1)[:, :c["moved"]].sort(-1).values + kept
    ident = torch.arange(c["ident"], device="cuda")[None, :].expand(b, -1)
    s["keep"] = torch.cat([ident, from_behind], -1).to(torch.int32).contiguous()
    s["count"] = torch.full((b,), kept, dtype=torch.int32, device="cuda")
    s["base"] = s["seq_len"] if c["after"] else None
    s["len_out"] = torch.zeros((b,), dtype=torch.int32, device="cuda")
    return s


def _prepare_fork(c, seed):
    """`batch` requests with their pages in a pool, and as many empty rows that they are forked to."""
    g, dt = _gen(seed), DTYPES[c["dtype"]]
    b, page = c["batch"], c["page"]
    lens = _ints(g, c["lo"], c["hi"], (b,))
    zero = torch.zeros_like(lens)
    per = -(-c["hi"] // page) + 1
    rows, blocks = _pages_for(g, b, per * page, page, spare=b)
    held = torch.arange(per, device="cuda")[None, :] < ((lens + page - 1) // page)[:, None]
    s = {"case": c, "seq_len": torch.cat([lens, zero]), "prompt_len": torch.cat([lens.clamp(max=64), zero])}
    s["table"] = torch.cat([rows.masked_fill(~held, -1), torch.full_like(rows, -1)])
    s["refs"] = torch.zeros((blocks,), dtype=torch.int32, device="cuda")
    s["refs"][rows[held].long()] = 1
    s["k"] = _normal(g, (c["layers"], blocks, page, c["hkv"], c["d"]), dt)
    s["v"] = _normal(g, s["k"].shape, dt)
    s["src"] = torch.randperm(b, generator=g, device="cuda").to(torch.int32)
    s["dst"] = torch.arange(b, 2 * b, device="cuda", dtype=torch.int32)
    s["keep_tokens"] = torch.cat([torch.full_like(lens, -1), zero])          # -1: the row is left alone
    s["status"] = torch.zeros((b,), dtype=torch.int32, device="cuda")
    return s


def _prepare_reserve(c, seed):
    g = _gen(seed)
    b, page = c["batch"], c["page"]
    lens = _ints(g, c["lo"], c["hi"], (b,))
    per = -(-(c["hi"] + c["extra"]) // page)
    rows, blocks = _pages_for(g, b, per * page, page)
    held = torch.arange(per, device="cuda")[None, :] < ((lens + page - 1) // page)[:, None]
    s = {"case": c, "seq_len": lens, "table": rows.masked_fill(~held, -1)}
    s["refs"] = torch.zeros((blocks,), dtype=torch.int32, device="cuda")
    s["refs"][rows[held].long()] = 1
    s["status"] = torch.zeros((b,), dtype=torch.int32, device="cuda")
    return s


def _inputs(case, seed):
    return {"tree": _prepare_tree, "verify": _prepare_verify, "compact": _prepare_compact, "fork": _prepare_fork,
            "reserve": _prepare_reserve}[case["op"]](case, seed)


def _handles(s):
    """What a program keeps from call to call: the problem's description, output buffers, workspace."""
    from paper_2609_19702_b200 import binding as dsa
    c = s["case"]
    if c["op"] == "verify":
        s["tree"] = dsa.Tree(c["nodes"], parent=s["parent"] if c["branch"] else None)
        s["verify"] = dsa.Verify(s["tokens"], s["target"], s["draft"], s["uniforms"])
        s["outs"] = dsa.alloc_verify_outputs(s["verify"])
        return
    if c["op"] == "reserve":
        s["pool"] = dsa.PagePool(s["refs"], c["page"])
        return
    k, table = s["k"], s["table"]
    one_layer = k if c["op"] == "tree" else k[0]
    q = s["q"] if c["op"] == "tree" else torch.empty((len(s["seq_len"]), c["hkv"], c["d"]), dtype=k.dtype, device="cuda")
    s["problem"] = dsa.Problem(
        q=q, k_cache=k, v_cache=s["v"], strides=(one_layer.stride(0), one_layer.stride(1), c["d"]),
        seq_len=s["seq_len"], prompt_len=s["prompt_len"], num_kv_heads=c["hkv"],
        max_seq_len=s["cap"] if c["op"] == "tree" else table.shape[1] * c["page"], max_prompt_len=c.get("prompt", 0),
        block_table=table, block_size=c["page"], num_blocks=one_layer.shape[0] if table is not None else 0)
    if c["op"] == "tree":
        s["diag"] = dsa.Diag(dsa.DSA_MASK_WINDOW, c["window"], n_sink=c["sinks"]) if c["window"] else None
        s["tree"] = dsa.Tree(c["nodes"], parent=s["parent"] if c["branch"] else None, node_count=s["count"] if c["ragged"] else None)
        s["out"], s["lse"] = dsa.alloc_tree_outputs(s["problem"])
        s["ws"] = dsa.alloc_tree_workspace(s["problem"], s["diag"], s["tree"])
    if c["op"] == "fork":
        s["pool"] = dsa.PagePool(s["refs"], c["page"])
        s["ws"] = dsa.alloc_fork_workspace(s["src"])


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:
        _handles(s)
    return s


# ------------------------------------------------------------------------------------------------ plain forms
def _places(s, pos):
    """Where the tokens at logical positions pos [B, P] live: indices of the cache's first two dimensions."""
    page = s["case"]["page"]
    if not page:
        return torch.arange(pos.shape[0], device="cuda")[:, None].expand_as(pos), pos
    return s["table"].long().gather(1, (pos // page).clamp(max=s["table"].shape[1] - 1)), pos % page


def _family(parent):
    """Whether node j is node i or an ancestor of it [B, N, N], and the depths [B, N]."""
    b, n = parent.shape
    i = torch.arange(n, device="cuda")
    up = (parent[:, :, None] == i) & (i < i[:, None])
    own_line = torch.linalg.matrix_power(up.float() + torch.eye(n, device="cuda"), n) > 0
    return own_line, own_line.sum(-1) - 1


def _plain_tree(s):
    c = s["case"]
    b, n, hq, hkv, d = c["batch"], c["nodes"], c["hq"], c["hkv"], c["d"]
    g = hq // hkv
    seq, prompt = s["seq_len"].long()[:, None], s["prompt_len"].long()[:, None]
    i = torch.arange(n, device="cuda")
    live = i < s["count"].long()[:, None]
    family, depth = _family(s["parent"].long())
    # the new rows go behind the cached ones
    blk, off = _places(s, seq + i)
    for_live = live[:, :, None, None]
    s["k"][blk, off] = torch.where(for_live, s["k_new"], s["k"][blk, off])
    s["v"][blk, off] = torch.where(for_live, s["v_new"], s["v"][blk, off])
    # what node i sees: the cached tokens, and the drafted ones of its own line
    pos = torch.arange(c["hi"], device="cuda")[None, :].expand(b, -1)
    cached = (pos < seq)[:, None, :].expand(b, n, -1)
    drafted = family & live[:, None, :]
    if c["window"]:
        first = prompt + c["sinks"]
        at = seq + depth                                                     # the nodes' logical positions
        cached = cached & ((pos < first)[:, None, :] | (at[:, :, None] - pos[:, None, :] < c["window"]))
        drafted = drafted & ((at < first)[:, None, :] | (at[:, :, None] - at[:, None, :] < c["window"]))
    seen = torch.cat([cached, drafted], -1) & live[:, :, None]              # [B, N, P + N]
    blk, off = _places(s, pos)
    keys = torch.cat([s["k"][blk, off], s["k_new"]], 1).float().permute(0, 2, 3, 1)            # [B, Hkv, D, P + N]
    values = torch.cat([s["v"][blk, off], s["v_new"]], 1).float().permute(0, 2, 1, 3)
    q = s["q"].float().view(b, n, hkv, g, d).permute(0, 2, 1, 3, 4).reshape(b, hkv, n * g, d)
    x = (q @ keys) / math.sqrt(d)
    x = x.view(b, hkv, n, g, -1).masked_fill(~seen[:, None, :, None, :], -math.inf)
    top = x.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    e = torch.exp(x - top)
    total = e.sum(-1, keepdim=True)
    p = e / torch.where(total == 0, 1.0, total)
    out = (p.view(b, hkv, n * g, -1) @ values).view(b, hkv, n, g, d)
    lse = (top + torch.log(total))[..., 0]
    return (out.permute(0, 2, 1, 3, 4).reshape(b, n, hq, d).to(s["q"].dtype),
            lse.permute(0, 2, 1, 3).reshape(b, n, hq), s["k"], s["v"])


def _plain_verify(s):
    c = s["case"]
    b, n, v = c["batch"], c["nodes"], c["vocab"]
    rows, words = torch.arange(b, device="cuda"), torch.arange(v, device="cuda")
    parent, tokens = s["parent"].long(), s["tokens"].long()
    cur = torch.zeros(b, dtype=torch.long, device="cuda")
    path = torch.full((b, n), -1, dtype=torch.long, device="cuda")
    path[:, 0] = 0
    length = torch.ones(b, dtype=torch.long, device="cuda")
    if c["mode"] == "greedy":
        x = s["target"]
        best = torch.where(x == x.amax(-1, keepdim=True), words, v).amin(-1)                   # ties: the lowest
    else:
        left, weight = s["target"][:, 0].double(), torch.ones(b, dtype=torch.float64, device="cuda")
        u = s["uniforms"].double()
    for i in range(1, n):  # a node's test hangs on the outcomes of the ones before it
        tested = parent[:, i] == cur
        token = tokens[:, i]
        if c["mode"] == "greedy":
            taken = tested & (token == best[rows, cur])
        else:
            mine = left[rows, token]
            if c["mode"] == "sample":
                q = s["draft"][rows, cur].double()
                taken = tested & (u[:, i] * weight * q[rows, token] < mine)
                rest = (left - weight[:, None] * q).clamp(min=0)
                total = rest.sum(-1)
            else:
                taken = tested & (u[:, i] * weight < mine)
                rest = left.masked_fill(words == token[:, None], 0)
                total = weight - mine
            turned = tested & ~taken
            left = torch.where(turned[:, None], rest, torch.where(taken[:, None], s["target"][:, i].double(), left))
            weight = torch.where(turned, total, torch.where(taken, 1.0, weight))
        path[rows, torch.where(taken, length, 0)] = torch.where(taken, i, 0)
        length += taken
        cur = torch.where(taken, i, cur)
    if c["mode"] == "greedy":
        word = best[rows, cur]
    else:
        total = left.sum(-1, keepdim=True)
        left = torch.where(total > 0, left, s["target"][rows, cur].double())
        word = (left.cumsum(-1) <= u[:, :1] * left.sum(-1, keepdim=True)).sum(-1)
    return path.int(), length.int(), word.int()


def _plain_compact(s):
    i = torch.arange(s["keep"].shape[1], device="cuda")
    base = s["base"].long()[:, None] if s["base"] is not None else torch.zeros_like(s["count"]).long()[:, None]
    blk, off = _places(s, base + s["keep"].long())
    to_blk, to_off = _places(s, (base + i).expand_as(blk))
    s["k"][:, to_blk, to_off] = s["k"][:, blk, off]
    s["v"][:, to_blk, to_off] = s["v"][:, blk, off]
    s["len_out"] = (base[:, 0] + s["count"]).int()
    return s["len_out"], s["k"], s["v"]


def _plain_release(s, keep):
    """Gives back the pages behind the first `keep` tokens of each row (negative: none of them)."""
    page = s["case"]["page"]
    e = torch.arange(s["table"].shape[1], device="cuda")
    gone = (e >= ((keep + page - 1) // page)[:, None]) & (keep >= 0)[:, None] & (s["table"] >= 0)
    s["refs"].scatter_add_(0, s["table"].clamp(min=0).long().view(-1), -gone.view(-1).int())
    s["table"].masked_fill_(gone, -1)


def _plain_fork(s):
    page = s["case"]["page"]
    _plain_release(s, s["keep_tokens"])
    src, dst = s["src"].long(), s["dst"].long()
    lens = s["seq_len"][src]
    full, part = lens // page, lens % page
    need = part > 0
    free = torch.argsort((s["refs"] != 0).int(), stable=True)               # the free pages, the lowest first
    fresh = free[(need.cumsum(0) - 1).clamp(min=0)]
    old = s["table"][src]
    e = torch.arange(old.shape[1], device="cuda")[None, :]
    shared = e < full[:, None]
    last = (e == full[:, None]) & need[:, None]
    s["refs"].scatter_add_(0, old.clamp(min=0).long().view(-1), shared.reshape(-1).int())
    s["refs"].scatter_add_(0, fresh, need.int())
    s["table"][dst] = torch.where(shared, old, torch.where(last, fresh[:, None].int(), -1))
    s["seq_len"][dst] = lens
    s["prompt_len"][dst] = s["prompt_len"][src]
    from_page = torch.where(need, old.gather(1, full.clamp(max=old.shape[1] - 1).long()[:, None])[:, 0], old[:, 0]).long()
    tokens = torch.arange(page, device="cuda")[None, :].expand(len(src), -1)
    copied = (tokens < part[:, None])[None, :, :, None, None]
    to, at = torch.where(need, fresh, from_page)[:, None], tokens
    s["k"][:, to, at] = torch.where(copied, s["k"][:, from_page[:, None], at], s["k"][:, to, at])
    s["v"][:, to, at] = torch.where(copied, s["v"][:, from_page[:, None], at], s["v"][:, to, at])
    return s["table"], s["refs"], s["seq_len"], s["prompt_len"], torch.zeros_like(s["status"]), s["k"], s["v"]


def _plain_reserve(s):
    c = s["case"]
    _plain_release(s, s["seq_len"])
    e = torch.arange(s["table"].shape[1], device="cuda")
    wanted = (s["seq_len"] + c["extra"] + c["page"] - 1) // c["page"]
    missing = (e < wanted[:, None]) & (s["table"] < 0)
    free = torch.argsort((s["refs"] != 0).int(), stable=True)
    fresh = free[(missing.view(-1).cumsum(0) - 1).clamp(min=0)]
    s["refs"].scatter_add_(0, fresh, missing.view(-1).int())
    s["table"].copy_(torch.where(missing, fresh.view_as(missing).int(), s["table"]))
    return s["table"], s["refs"], torch.zeros_like(s["status"])


# ------------------------------------------------------------------------------------------------ one pass
def run(s):
    op = s["case"]["op"]
    if own:
        from paper_2609_19702_b200 import binding as dsa
        if op == "tree":
            dsa.dsa_tree_step(s["problem"], s["diag"], s["tree"], s["k_new"], s["v_new"], s["out"], s["lse"], s["ws"])
            return s["out"], s["lse"], s["k"], s["v"]
        if op == "verify":
            dsa.dsa_verify_tree(s["verify"], s["tree"], *s["outs"])
            return s["outs"]
        if op == "compact":
            dsa.dsa_compact_kv(s["problem"], s["keep"], s["count"], base=s["base"], len_out=s["len_out"],
                               num_layers=s["case"]["layers"], stride_layer=s["k"].stride(0))
            return s["len_out"], s["k"], s["v"]
        if op == "fork":  # the rows of the last branch are given up, then the requests branch again
            dsa.dsa_release_pages(s["pool"], s["table"], s["keep_tokens"])
            dsa.dsa_fork_pages(s["pool"], s["problem"], s["src"], s["dst"], s["status"], s["ws"],
                               num_layers=s["case"]["layers"], stride_layer=s["k"].stride(0))
            return s["table"], s["refs"], s["seq_len"], s["prompt_len"], s["status"], s["k"], s["v"]
        # what the last draft took is given back, then room is made for the next one
        dsa.dsa_release_pages(s["pool"], s["table"], s["seq_len"])
        dsa.dsa_reserve_pages(s["pool"], s["table"], s["seq_len"], s["case"]["extra"], s["status"])
        return s["table"], s["refs"], s["status"]
    return {"tree": _plain_tree, "verify": _plain_verify, "compact": _plain_compact, "fork": _plain_fork,
            "reserve": _plain_reserve}[op](s)


# ------------------------------------------------------------------------------------------------ what it costs at least
def work(case):
    c = case
    size = 2 if c.get("dtype") == "bf16" else 4
    if c["op"] == "tree":
        b, n = c["batch"], c["nodes"] * (0.5 if c["ragged"] else 1.0)
        length = (c["lo"] + c["hi"]) / 2
        if c["window"]:
            length = min(length, min(length, c["prompt"]) + c["sinks"] + c["window"])
        rows = b * length * c["hkv"] * c["d"] * 2 * size                    # the cached rows that some node sees
        new = b * n * c["hkv"] * c["d"] * 2 * size                          # read and appended
        qo = b * n * c["hq"] * c["d"] * 2 * size
        return {"bytes": rows + 2 * new + qo + 4 * b * n * c["hq"], "flops": 4 * b * n * c["hq"] * c["d"] * length}
    if c["op"] == "verify":  # the target's row where the walk ends, and the draft's
        rows = 2 if c["mode"] == "sample" else 1
        return {"bytes": c["batch"] * (rows * c["vocab"] * size + 16 * c["nodes"]), "flops": 0}
    if c["op"] == "compact":
        moved = c["batch"] * c["moved"] * c["layers"] * c["hkv"] * c["d"] * 2 * size
        return {"bytes": 2 * moved + 4 * c["batch"] * (c["moved"] + c["ident"]), "flops": 0}
    entries = c["batch"] * (-(-(c["lo"] + c["hi"]) // (2 * c["page"])) + 1) * 4
    if c["op"] == "fork":
        copied = c["batch"] * (c["page"] - 1) / 2 * c["layers"] * c["hkv"] * c["d"] * 2 * size
        return {"bytes": 2 * copied + 4 * entries, "flops": 0}
    return {"bytes": 3 * entries, "flops": 0}


# ------------------------------------------------------------------------------------------------ in 64 bits
def exact(case, seed):
    """The definition, request by request: softmax over the tokens that a node sees.  The other operators have
    whole numbers and copies of rows, which the plain form's own have to equal."""
    if case["op"] != "tree":
        return None
    c = case
    s = _inputs(case, seed)
    b, n, hq, hkv, d = c["batch"], c["nodes"], c["hq"], c["hkv"], c["d"]
    parent, counts = s["parent"].tolist(), s["count"].tolist()
    out = torch.zeros((b, n, hq, d), dtype=torch.float64, device="cuda")
    lse = torch.full((b, n, hq), -math.inf, dtype=torch.float64, device="cuda")
    for r in range(b):
        length, prompt = int(s["seq_len"][r]), int(s["prompt_len"][r])
        lines, depth = [], []
        for i in range(counts[r]):
            p = parent[r][i]
            lines.append((lines[p] if 0 <= p < i else []) + [i])
            depth.append(len(lines[-1]) - 1)
        if not lines:
            continue
        m = len(lines)
        if c["page"]:
            k = s["k"][s["table"][r].long()].reshape(-1, hkv, d)[:length]
            v = s["v"][s["table"][r].long()].reshape(-1, hkv, d)[:length]
        else:
            k, v = s["k"][r, :length], s["v"][r, :length]
        k = torch.cat([k, s["k_new"][r, :m]]).double()
        v = torch.cat([v, s["v_new"][r, :m]]).double()
        seen = torch.zeros((m, length + m), dtype=torch.bool, device="cuda")
        places = torch.arange(length, device="cuda")
        for i in range(m):
            at = length + depth[i]
            w = c["window"]
            seen[i, :length] = ((places < prompt + c["sinks"]) | (at - places < w)) if w else True
            mine = [j for j in lines[i] if not w or depth[i] - depth[j] < w or length + depth[j] < prompt + c["sinks"]]
            seen[i, [length + j for j in mine]] = True
        for h in range(hq):
            x = s["q"][r, :m, h].double() @ k[:, h // (hq // hkv)].T / math.sqrt(d)
            x.masked_fill_(~seen, -math.inf)
            lse[r, :m, h] = torch.logsumexp(x, -1)
            out[r, :m, h] = torch.softmax(x, -1) @ v[:, h // (hq // hkv)]
    return out, lse, None, None
