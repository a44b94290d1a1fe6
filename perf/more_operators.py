"""Cases of the latent-cache operators: what they are given, what they compute, what that costs at least.

A latent cache holds one row a token, shared by all heads: R numbers that keys and values are both made from, and
P more that carry the position.  Four kinds of call work on it:

- ``step``: the new tokens of every request attend over the cache and over one another, with queries that have
  taken the keys' expansion in (the absorbed form), and their rows are appended;
- ``prompt``: the tokens of a ragged batch of prompts attend with keys and values expanded per head;
- ``map``: which request, position and cache slot every token of a ragged batch has;
- ``rows``: rows of such a batch go to their slots (``store``), or come from them (``gather``).

``run`` computes a case in plain torch operations, or, where ``own`` is true, by the library's calls.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


# ------------------------------------------------------------------------------------------------ the cases
def _step(name, **kw):
    case = {"name": name, "op": "step", "dtype": "bf16", "batch": 1, "heads": 16, "latent": 512, "rope": 64, "new": 1,
            "ragged": False, "page": 16, "lo": 1, "hi": 1024}
    return {**case, **kw}


def _prompt(name, **kw):
    case = {"name": name, "op": "prompt", "dtype": "bf16", "batch": 1, "heads": 16, "nope": 128, "rope": 64, "value": 128,
            "lo": 1, "hi": 600, "before": 0}
    return {**case, **kw}


def _map(name, **kw):
    return {"name": name, "op": "map", "batch": 8, "page": 16, "lo": 0, "hi": 1024, "new": 1, **kw}


def _rows(name, **kw):
    case = {"name": name, "op": "rows", "way": "store", "dtype": "bf16", "batch": 8, "latent": 512, "rope": 64, "page": 16,
            "lo": 0, "hi": 1024, "new": 512}
    return {**case, **kw}


def listed():
    return [
        # a single user, one token, the heads of one rank of eight: latency
        _step("step 1x16", lo=500, hi=700),
        # a serving batch of such a rank over sequences of all lengths (90 x 91 image tokens): memory
        _step("step 64x16 paged", batch=64, page=64, lo=1, hi=8190),
        # all heads on one GPU: arithmetic and memory about even
        _step("step 32x128 paged", batch=32, heads=128, page=64, lo=1024, hi=8190),
        # the same with four drafted tokens a request, fewer for some: arithmetic
        _step("step 16x128 drafted", batch=16, heads=128, new=4, ragged=True, page=16, lo=2048, hi=4160),
        # single precision and narrow rows in a contiguous cache, for checking a model against its reference
        _step("step f32 r256", dtype="f32", batch=4, heads=20, latent=256, rope=32, new=3, page=0, lo=1, hi=1144),
        # one long sequence (64 x 65 tokens) scored in one pass: arithmetic
        _prompt("prompt 1x4160", lo=4160, hi=4160),
        # a ragged batch of prompts, each behind a cached prefix of its own
        _prompt("prompt ragged 24", batch=24, lo=1, hi=600, before=512),
        # single precision, narrow heads
        _prompt("prompt f32 d64", dtype="f32", batch=4, heads=8, nope=64, value=64, rope=32, lo=1, hi=300),
        # the next token of a small batch: latency
        _map("map 8x1"),
        # a large ragged batch of prompts
        _map("map 256x512", batch=256, hi=4096, new=512),
        # its latent rows go to the cache
        _rows("rows store 64x512", batch=64),
        # the cached prefixes of a few requests come back to be expanded
        _rows("rows gather 8x4096", way="gather", lo=0, hi=0, new=4096, page=64),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng):
    op = rng.choice(["step", "step", "step", "prompt", "prompt", "map", "rows"])
    if op == "step":
        bf = rng.random() < 0.75
        c = {"op": op, "dtype": "bf16" if bf else "f32", "heads": rng.choice([1, 3, 8, 16, 20, 32, 64, 96, 128] if bf else [1, 3, 8, 20]),
             "latent": rng.choice([256, 512]), "rope": rng.choice([16, 32, 64]), "new": _log(rng, 1, 8 if bf else 4),
             "ragged": rng.random() < 0.4, "page": rng.choice([0, 1, 5, 16, 24, 64, 128]), "lo": rng.choice([0, 1, 17]),
             "hi": _log(rng, 20, 8192 if bf else 1500)}
        rows = c["heads"] * c["new"]
        most = 32 * 8192 * 128 if bf else 4 * 1500 * 60                     # (token, query row) pairs
        c["batch"] = _log(rng, 1, max(1, min(64 if bf else 8, most // (c["hi"] * max(rows, 32 if bf else 1)))))
        return c
    if op == "prompt":
        bf = rng.random() < 0.75
        wide = rng.random() < 0.7
        c = {"op": op, "dtype": "bf16" if bf else "f32", "heads": rng.choice([1, 3, 8, 16, 20] if bf else [1, 3, 8]),
             "nope": 128 if wide else 64, "value": 128 if wide else 64, "rope": rng.choice([16, 32, 64]), "lo": rng.choice([0, 1, 17]),
             "hi": _log(rng, 20, 4160 if bf else 400), "before": rng.choice([0, 0, 100, 700])}
        most = 16 * 4160 * 4160 if bf else 4 * 8 * 400 * 400
        c["batch"] = _log(rng, 1, max(1, min(32, most // (c["heads"] * c["hi"] * (c["hi"] + c["before"])))))
        return c
    c = {"op": op, "page": rng.choice([0, 1, 5, 16, 24, 64]), "lo": 0, "hi": _log(rng, 1, 4096), "new": _log(rng, 1, 512)}
    if op == "map":
        c["batch"] = _log(rng, 1, 256)
        return c
    c.update({"way": rng.choice(["store", "gather"]), "dtype": rng.choice(["bf16", "f32"]), "latent": rng.choice([256, 512]),
              "rope": rng.choice([16, 32, 64]), "hi": _log(rng, 1, 1024)})
    c["batch"] = _log(rng, 1, max(1, min(128, 16384 // c["new"])))
    return c


# ------------------------------------------------------------------------------------------------ inputs
def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _ints(g, lo, hi, shape):
    """Whole numbers of [lo, hi], 32 bits."""
    return torch.randint(lo, hi + 1, shape, generator=g, device="cuda", dtype=torch.int32)


def _normal(g, shape, dtype):
    return torch.empty(shape, dtype=dtype, device="cuda").normal_(generator=g)


def _starts(lens):
    return torch.cat([torch.zeros_like(lens[:1]), lens.cumsum(0, dtype=torch.int32)])


def _pages_for(g, batch, tokens, page):
    """Block table of `batch` rows that hold `tokens` tokens each, in a shuffled pool, and the pool's size."""
    per = max(1, -(-tokens // page))
    n = batch * per
    return torch.randperm(n, generator=g, device="cuda").to(torch.int32).view(batch, per).contiguous(), n


def _cache(s, g, c, tokens):
    """A cache with room for `tokens` tokens a request: pages and their table, or one region a request."""
    width = c["latent"] + c["rope"]
    if c["page"]:
        s["table"], blocks = _pages_for(g, c["batch"], tokens, c["page"])
        s["cache"] = _normal(g, (blocks, c["page"], width), DTYPES[c["dtype"]])
    else:
        s["table"], s["cache"] = None, _normal(g, (c["batch"], tokens, width), DTYPES[c["dtype"]])
    s["room"] = tokens


def _prepare_step(c, seed):
    g, dt = _gen(seed), DTYPES[c["dtype"]]
    b, n, width = c["batch"], c["new"], c["latent"] + c["rope"]
    s = {"case": c, "seq_len": _ints(g, c["lo"], c["hi"], (b,))}
    _cache(s, g, c, c["hi"] + n)
    s["q"] = _normal(g, (b, n, c["heads"], width), dt)
    s["c_new"] = _normal(g, (b, n, width), dt)
    s["count"] = _ints(g, 0, n, (b,)) if c["ragged"] else None
    s["scale"] = 1.0 / math.sqrt(128 + c["rope"])                           # (of the heads before their keys were absorbed)
    return s


def _prepare_prompt(c, seed):
    g, dt = _gen(seed), DTYPES[c["dtype"]]
    b, h = c["batch"], c["heads"]
    lens = _ints(g, c["lo"], c["hi"], (b,))
    lens[:1].clamp_(min=1)
    before = _ints(g, 0, c["before"], (b,))
    s = {"case": c, "lens": lens, "before": before, "q_start": _starts(lens), "kv_start": _starts(lens + before)}
    # buffers for the longest batch that the program takes; what lies behind the last sequence is nobody's
    s["q"] = _normal(g, (b * c["hi"], h, c["nope"] + c["rope"]), dt)
    kv_tokens = b * (c["hi"] + c["before"])
    s["kv"] = _normal(g, (kv_tokens, h, c["nope"] + c["value"]), dt)        # as one product with the expansion leaves them
    s["k_rope"] = _normal(g, (kv_tokens, c["rope"]), dt)
    s["scale"] = 1.0 / math.sqrt(c["nope"] + c["rope"])
    return s


def _prepare_map(c, seed):
    g = _gen(seed)
    b = c["batch"]
    s = {"case": c, "base": _ints(g, c["lo"], c["hi"], (b,)), "count": _ints(g, 0 if c["new"] > 1 else 1, c["new"], (b,))}
    s["room"] = c["hi"] + c["new"]
    s["table"], s["blocks"] = _pages_for(g, b, s["room"], c["page"]) if c["page"] else (None, b)
    n = b * c["new"]                                                        # the padded batch
    s["start"] = torch.zeros((b + 1,), dtype=torch.int32, device="cuda")
    s["slot"] = torch.zeros((n,), dtype=torch.int64, device="cuda")
    s["position"] = torch.zeros((n,), dtype=torch.int32, device="cuda")
    s["request"] = torch.zeros((n,), dtype=torch.int32, device="cuda")
    return s


def _prepare_rows(c, seed):
    g, dt = _gen(seed), DTYPES[c["dtype"]]
    s = {"case": c, "seq_len": _ints(g, c["lo"], c["hi"], (c["batch"],)), "count": _ints(g, 1, c["new"], (c["batch"],))}
    _cache(s, g, c, c["hi"] + c["new"])
    n = c["batch"] * c["new"]
    request = torch.repeat_interleave(torch.arange(c["batch"], device="cuda"), s["count"].long())
    at = torch.arange(len(request), device="cuda") - _starts(s["count"]).long()[request] + s["seq_len"].long()[request]
    slot = request * s["room"] + at
    if c["page"]:
        slot = s["table"][request, at // c["page"]].long() * c["page"] + at % c["page"]
    s["slot"] = torch.full((n,), -1, dtype=torch.int64, device="cuda")      # behind the last token: nothing
    s["slot"][:len(slot)] = slot
    s["rows"] = _normal(g, (n, c["latent"] + c["rope"]), dt)
    return s


def _inputs(case, seed):
    return {"step": _prepare_step, "prompt": _prepare_prompt, "map": _prepare_map, "rows": _prepare_rows}[case["op"]](case, seed)


def _handles(s):
    """What a program keeps from call to call: descriptions, output buffers, workspace."""
    from paper_2609_19702_b200 import binding as dsa
    c = s["case"]
    if c["op"] == "prompt":
        k_nope, v = s["kv"][..., :c["nope"]], s["kv"][..., c["nope"]:]
        s["prompt"] = dsa.Prompt(s["q"], k_nope, s["k_rope"], v, s["q_start"], s["kv_start"], max_q_len=c["hi"], sm_scale=s["scale"])
        s["out"], s["lse"] = dsa.alloc_prompt_outputs(s["prompt"])
        s["out"].zero_(), s["lse"].zero_()                                  # (rows of nobody stay as they are)
        return
    if c["op"] == "map":
        return
    cache = s["cache"]
    s["latent"] = dsa.Latent(cache, strides=(cache.stride(0), cache.stride(1)), seq_len=s["seq_len"], latent_dim=c["latent"],
                             rope_dim=c["rope"], max_seq_len=s["room"], sm_scale=s.get("scale", 1.0), block_table=s["table"],
                             block_size=c["page"], num_blocks=cache.shape[0] if c["page"] else 0)
    if c["op"] == "step":
        s["out"], s["lse"] = dsa.alloc_latent_outputs(s["latent"], s["q"])
        s["ws"] = dsa.alloc_latent_workspace(s["latent"], s["q"])


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:
        _handles(s)
    return s


# ------------------------------------------------------------------------------------------------ plain forms
def _softmax(x, seen):
    """Weights and log-sums of the scores x where `seen`, over the last dimension; rows that see nothing: 0 and -inf."""
    x = x.masked_fill_(~seen, -math.inf)
    top = x.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    e = torch.exp(x - top)
    total = e.sum(-1, keepdim=True)
    return e / torch.where(total == 0, 1.0, total), (top + torch.log(total))[..., 0]


def _plain_step(s):
    c = s["case"]
    b, n, h, r = c["batch"], c["new"], c["heads"], c["latent"]
    seq = s["seq_len"].long()[:, None]
    i = torch.arange(n, device="cuda")
    live = i < s["count"].long()[:, None] if s["count"] is not None else torch.ones((b, n), dtype=torch.bool, device="cuda")
    pos = torch.arange(c["hi"], device="cuda")[None, :].expand(b, -1)

    def places(at):
        if c["page"]:
            return s["table"].long().gather(1, at // c["page"]), at % c["page"]
        return torch.arange(b, device="cuda")[:, None].expand_as(at), at

    blk, off = places(seq + i)
    s["cache"][blk, off] = torch.where(live[:, :, None], s["c_new"], s["cache"][blk, off])
    keys = torch.cat([s["cache"][places(pos)], s["c_new"]], 1).float()      # [B, P + N, R + P]
    cached = (pos < seq)[:, None, :].expand(b, n, -1)
    seen = torch.cat([cached, (i <= i[:, None])[None].expand(b, -1, -1)], -1) & live[:, :, None]
    x = (s["q"].float().view(b, n * h, -1) @ keys.transpose(1, 2)).mul_(s["scale"])
    p, lse = _softmax(x.view(b, n, h, -1), seen[:, :, None, :])
    out = p.view(b, n * h, -1) @ keys[..., :r]
    return out.view(b, n, h, r).to(s["q"].dtype), lse, s["cache"]


def _padded(rows, start, lens, most):
    """Ragged rows [T, ...] as [B, most, ...], the last row repeated behind a sequence's end."""
    at = start[:-1, None].long() + torch.arange(most, device="cuda")
    return rows[at.clamp(max=rows.shape[0] - 1)].float()


def _plain_prompt(s):
    c = s["case"]
    most_q, most_k = c["hi"], c["hi"] + c["before"]
    lens, both = s["lens"].long(), (s["lens"] + s["before"]).long()
    q = _padded(s["q"], s["q_start"], lens, most_q).transpose(1, 2)                         # [B, H, Q, D]
    kv = _padded(s["kv"], s["kv_start"], both, most_k).permute(0, 2, 1, 3)                  # [B, H, K, ...]
    rope = _padded(s["k_rope"], s["kv_start"], both, most_k)[:, None].expand(-1, c["heads"], -1, -1)
    k = torch.cat([kv[..., :c["nope"]], rope], -1)
    i, j = torch.arange(most_q, device="cuda"), torch.arange(most_k, device="cuda")
    seen = (j <= i[:, None] + s["before"].long()[:, None, None]) & (j < both[:, None, None])
    p, lse = _softmax((q @ k.transpose(2, 3)).mul_(s["scale"]), seen[:, None])
    out = p @ kv[..., c["nope"]:]
    # back to the ragged layout; rows behind the last sequence stay zeros
    t = torch.arange(s["q"].shape[0], device="cuda")
    request = (t[:, None] >= s["q_start"][None, 1:]).sum(-1)
    there = (request < c["batch"])[:, None]
    request = request.clamp(max=c["batch"] - 1)
    at = (t - s["q_start"].long()[request]).clamp(max=most_q - 1)
    out, lse = out.permute(0, 2, 1, 3)[request, at], lse.permute(0, 2, 1)[request, at]
    return torch.where(there[..., None], out, 0).to(s["q"].dtype), torch.where(there, lse, 0)


def _plain_map(s):
    c = s["case"]
    b, n = c["batch"], s["slot"].shape[0]
    start = _starts(s["count"])
    t = torch.arange(n, device="cuda", dtype=torch.int32)
    request = (t[:, None] >= start[None, 1:]).sum(-1)
    there = request < b
    r = request.clamp(max=b - 1)
    position = t - start[r] + s["base"][r]
    if c["page"]:
        at = position.clamp(max=s["room"] - 1).long()
        slot = s["table"][r, at // c["page"]].long() * c["page"] + at % c["page"]
    else:
        slot = r * s["room"] + position
    return (start, torch.where(there, slot, -1), torch.where(there, position, -1), torch.where(there, request, -1).int())


def _plain_rows(s):
    c = s["case"]
    width = c["latent"] + c["rope"]
    flat = s["cache"].view(-1, width)
    there = (s["slot"] >= 0)[:, None]
    at = s["slot"].clamp(min=0)
    if c["way"] == "gather":
        s["rows"].copy_(torch.where(there, flat[at], s["rows"]))
        return s["rows"]
    # rows without a slot go to one more row behind the cache, which is cut off again
    more = torch.cat([flat, flat[:1]])
    more[torch.where(there[:, 0], at, flat.shape[0])] = s["rows"]
    flat.copy_(more[:-1])
    return s["cache"]


# ------------------------------------------------------------------------------------------------ one pass
def run(s):
    op = s["case"]["op"]
    if own:
        from paper_2609_19702_b200 import binding as dsa
        if op == "step":
            dsa.dsa_latent_step(s["latent"], s["q"], s["c_new"], s["out"], s["lse"], s["ws"], new_count=s["count"])
            return s["out"], s["lse"], s["cache"]
        if op == "prompt":
            dsa.dsa_latent_prompt(s["prompt"], s["out"], s["lse"])
            return s["out"], s["lse"]
        if op == "map":
            dsa.dsa_map_tokens(s["count"], s["start"], s["slot"], s["position"], s["request"], base=s["base"], block_table=s["table"],
                               block_size=s["case"]["page"], num_blocks=s["blocks"], max_seq_len=s["room"])
            return s["start"], s["slot"], s["position"], s["request"]
        if s["case"]["way"] == "gather":
            dsa.dsa_gather_rows(s["latent"], s["slot"], s["rows"])
            return s["rows"]
        dsa.dsa_store_rows(s["latent"], s["slot"], s["rows"])
        return s["cache"]
    return {"step": _plain_step, "prompt": _plain_prompt, "map": _plain_map, "rows": _plain_rows}[op](s)


# ------------------------------------------------------------------------------------------------ what it costs at least
def work(case):
    c = case
    size = 2 if c.get("dtype") == "bf16" else 4
    if c["op"] == "step":
        b, n = c["batch"], c["new"] * (0.5 if c["ragged"] else 1.0)
        length = (c["lo"] + c["hi"]) / 2
        width = c["latent"] + c["rope"]
        rows = b * (length + 2 * n) * width * size                          # cached ones read, new ones read and appended
        qo = b * n * c["heads"] * ((width + c["latent"]) * size + 4)
        return {"bytes": rows + qo, "flops": 2 * b * n * c["heads"] * (length + (n + 1) / 2) * (width + c["latent"])}
    if c["op"] == "prompt":
        lens, before = (c["lo"] + c["hi"]) / 2, c["before"] / 2
        square = (c["lo"] ** 2 + c["lo"] * c["hi"] + c["hi"] ** 2) / 3      # the mean square of lengths spread evenly
        pairs = c["batch"] * c["heads"] * (square / 2 + lens * before)
        q, kv = c["nope"] + c["rope"], c["nope"] + c["value"]
        tokens = c["batch"] * ((lens * (q + c["value"]) + (lens + before) * kv) * c["heads"] + (lens + before) * c["rope"])
        return {"bytes": tokens * size, "flops": 2 * pairs * (q + c["value"])}
    if c["op"] == "map":
        tokens = c["batch"] * c["new"]
        return {"bytes": tokens * 16 + 12 * c["batch"] + (4 * tokens / c["page"] if c["page"] else 0), "flops": 0}
    tokens = c["batch"] * (c["new"] + 1) / 2
    return {"bytes": tokens * ((c["latent"] + c["rope"]) * size * 2 + 8), "flops": 0}


# ------------------------------------------------------------------------------------------------ in 64 bits
def _attend(q, k, v, seen, scale):
    """softmax(scale q k^T) v over the keys that are seen: [..., Q, D], [..., K, D], [..., K, E]; and the log-sums."""
    x = (q @ k.transpose(-1, -2) * scale).masked_fill(~seen, -math.inf)
    return torch.softmax(x, -1).nan_to_num(0.0) @ v, torch.logsumexp(x, -1)


def exact(case, seed):
    """The definitions, request by request.  The other operators have whole numbers and copies of rows, which the
    plain form's own have to equal."""
    if case["op"] not in ("step", "prompt"):
        return None
    c = case
    s = _inputs(case, seed)
    outs, lses = [], []
    if c["op"] == "prompt":
        q0, k0 = s["q_start"].tolist(), s["kv_start"].tolist()
        for r in range(c["batch"]):
            nq, nk = q0[r + 1] - q0[r], k0[r + 1] - k0[r]
            kv = s["kv"][k0[r]:k0[r + 1]].double().transpose(0, 1)
            rope = s["k_rope"][k0[r]:k0[r + 1]].double().expand(c["heads"], -1, -1)
            seen = torch.ones((nq, nk), dtype=torch.bool, device="cuda").tril(nk - nq)
            parts = [_attend(s["q"][q0[r]:q0[r + 1], h].double(), torch.cat([kv[h, :, :c["nope"]], rope[h]], -1),
                             kv[h, :, c["nope"]:], seen, s["scale"]) for h in range(c["heads"])]
            outs.append(torch.stack([p[0] for p in parts], 1))
            lses.append(torch.stack([p[1] for p in parts], 1))
        nobody = s["q"].shape[0] - q0[-1]
        outs.append(torch.zeros((nobody, c["heads"], c["value"]), dtype=torch.float64, device="cuda"))
        lses.append(torch.zeros((nobody, c["heads"]), dtype=torch.float64, device="cuda"))
        return torch.cat(outs), torch.cat(lses)
    b, n, h, r = c["batch"], c["new"], c["heads"], c["latent"]
    out = torch.zeros((b, n, h, r), dtype=torch.float64, device="cuda")
    lse = torch.full((b, n, h), -math.inf, dtype=torch.float64, device="cuda")
    lens = s["seq_len"].tolist()
    counts = s["count"].tolist() if s["count"] is not None else [n] * b
    for j in range(b):
        rows = s["cache"][s["table"][j].long()].flatten(0, 1) if c["page"] else s["cache"][j]
        for i in range(counts[j]):
            k = torch.cat([rows[:lens[j]], s["c_new"][j, :i + 1]]).double()
            seen = torch.ones((1, len(k)), dtype=torch.bool, device="cuda")
            out[j, i], lse[j, i] = _attend(s["q"][j, i].double(), k, k[:, :r], seen, s["scale"])
    return out, lse, None
