"""The operators around a hybrid batch's attention, as a serving loop calls them, and their plain forms.

Three operators, each with its own cases ("op" in a case):

* ``scores``: attention whose scores are capped by a tanh or get a bias that grows with distance, under sliding windows,
  document masks and prefix masks.  One pass is one ``HybridAttention.forward`` of a plan made with ``Scores``.
* ``append``: the projections of a batch's new tokens normalised for each head, rotated by their position and written: queries
  to the rows that the attention reads, keys and values into the cache.  One pass is one layer of one step.
* ``tables``: blocks for the new tokens taken from a free list, and the slot and position of every new row.  One pass is one step.

With ``own`` false everything is computed by elementary torch operations in 32 bits (angles in 64).
"""
import math
import random

import torch

own = False

_DTYPES = {"fp16": torch.float16, "bf16": torch.bfloat16}


# ---------------------------------------------------------------------------------------------
# Cases
# ---------------------------------------------------------------------------------------------
def _scores(name, *, heads, dtype="bf16", block=16, head_major=False, n_prefill=0, q=(1, 1), past=(0, 0), n_decode=0,
            ctx=(1, 1), cap=0.0, slopes=False, window=0, docs=(0, 0), prefix=(0, 0), spread=1.0, lens_seed=1):
    hq, hkv, d = heads
    return {"name": name, "op": "scores", "hq": hq, "hkv": hkv, "d": d, "dtype": dtype, "block": block,
            "head_major": head_major, "n_prefill": n_prefill, "q_lo": q[0], "q_hi": q[1], "past_lo": past[0],
            "past_hi": past[1], "n_decode": n_decode, "ctx_lo": ctx[0], "ctx_hi": ctx[1], "cap": cap, "slopes": slopes,
            "window": window, "doc_lo": docs[0], "doc_hi": docs[1], "prefix_lo": prefix[0], "prefix_hi": prefix[1],
            "spread": spread, "lens_seed": lens_seed}


def _append(name, *, heads, rows, padded=0, dtype="bf16", block=16, head_major=False, layout="half", rot=None, theta=10000.0,
            scaling="none", factor=1.0, trained=8192, norm=True, offset=0.0, pos=(0, 1), packed=True, lens_seed=1):
    hq, hkv, d = heads
    return {"name": name, "op": "append", "hq": hq, "hkv": hkv, "d": d, "rows": rows, "padded": padded, "dtype": dtype,
            "block": block, "head_major": head_major, "layout": layout, "rot": d if rot is None else rot, "theta": theta,
            "scaling": scaling, "factor": factor, "trained": trained, "norm": norm, "offset": offset, "pos_lo": pos[0],
            "pos_hi": pos[1], "packed": packed, "lens_seed": lens_seed}


def _tables(name, *, block=16, n_prefill=0, q=(1, 1), past=(0, 0), n_decode=0, ctx=(1, 1), padded=0, lens_seed=1):
    return {"name": name, "op": "tables", "block": block, "n_prefill": n_prefill, "q_lo": q[0], "q_hi": q[1],
            "past_lo": past[0], "past_hi": past[1], "n_decode": n_decode, "ctx_lo": ctx[0], "ctx_hi": ctx[1],
            "padded": padded, "lens_seed": lens_seed}


def listed():
    return [
        # The smallest attention call: eight short replies, four heads of 64 channels, contiguous cache, capped scores.
        _scores("capped_decode_small", heads=(4, 4, 64), dtype="fp16", block=0, n_decode=8, ctx=(64, 512), cap=30.0, spread=2.0),
        # A chunk beside 64 replies with capped scores and 256 channels per head: the ordinary hybrid batch of that form.
        _scores("capped_hybrid", heads=(16, 8, 256), n_prefill=1, q=(1024, 1024), past=(3000, 3000), n_decode=64,
                ctx=(2048, 8192), cap=50.0, spread=2.0),
        # The same models' other layers: every token sees a window of 4096, and conversations are longer than that.
        _scores("window_hybrid", heads=(32, 8, 128), n_prefill=1, q=(512, 512), past=(7680, 7680), n_decode=128,
                ctx=(2048, 16384), window=4096, cap=50.0),
        # Scores that fall with distance, a slope per head and one K/V head per query head: a prompt and a few replies.
        _scores("distance_prompt", heads=(32, 32, 128), dtype="fp16", block=0, n_prefill=1, q=(4096, 4096), n_decode=8,
                ctx=(512, 4096), slopes=True),
        # One row of packed documents of 100 to 2000 tokens that do not see each other, padding between some of them.
        _scores("documents_packed", heads=(32, 8, 128), n_prefill=1, q=(8192, 8192), docs=(100, 2000)),
        # Odd everything: head counts of a tensor-parallel shard, blocks of 24, prefixes seen both ways, slopes, a cap.
        _scores("prefix_odd", heads=(15, 5, 128), block=24, n_prefill=3, q=(150, 700), past=(0, 1300), n_decode=21,
                ctx=(33, 5000), prefix=(64, 600), slopes=True, cap=20.0, spread=2.0),
        # The largest: a chunk of a long document beside 32 replies at 32K, all scores capped.
        _scores("capped_long", heads=(32, 4, 128), n_prefill=1, q=(2048, 2048), past=(30720, 30720), n_decode=32,
                ctx=(32768, 32768), cap=50.0),
        # A step of 16 replies: one token each, at positions of a few thousand.  Latency is all it costs.
        _append("append_decode", heads=(32, 8, 128), rows=16, pos=(500, 16000), theta=500000.0, scaling="parts", factor=8.0),
        # A prompt of 8192 tokens, normalised and rotated whole.
        _append("append_prompt", heads=(32, 8, 128), rows=8192, theta=1000000.0),
        # Half of the channels rotated in neighbouring pairs, no norm, blocks of 24 in head-major order, separate
        # projections, the batch padded to a captured size.
        _append("append_odd", heads=(9, 3, 64), rows=777, padded=23, dtype="fp16", block=24, head_major=True,
                layout="interleaved", rot=32, norm=False, pos=(0, 200000), packed=False, scaling="linear", factor=4.0),
        # A step of 256 replies: one token each, a new block for about one in sixteen.
        _tables("tables_decode", n_decode=256, ctx=(2048, 16384)),
        # Chunks of six long prompts beside 500 replies, padded to a captured size.
        _tables("tables_hybrid", n_prefill=6, q=(1000, 8192), past=(0, 24000), n_decode=500, ctx=(1, 32768), padded=100),
    ]


# (query heads, K/V heads, channels)
_HEADS = [(32, 32, 128), (32, 8, 128), (32, 4, 128), (16, 8, 128), (10, 5, 128), (9, 3, 128), (8, 1, 128),
          (32, 8, 64), (16, 1, 64), (9, 3, 64), (4, 4, 64), (16, 8, 256), (8, 2, 256)]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of any of the operators, any size up to the largest listed one."""
    op = rng.choice(["scores", "scores", "append", "tables"])
    while True:
        if op == "scores":
            kind = rng.choice(["decode", "prefill", "hybrid", "hybrid"])
            n_prefill = n_decode = 0
            q, past, ctx, docs, prefix = (0, 0), (0, 0), (1, 1), (0, 0), (0, 0)
            if kind != "decode":
                n_prefill = rng.choice([1, 1, 2, 3, 6])
                q_hi = _log_int(rng, 17, 8192 // n_prefill)
                q = (max(1, q_hi // rng.choice([1, 2, 5])), q_hi)
                past_hi = rng.choice([0, _log_int(rng, 64, 30720)])
                past = (past_hi // rng.choice([1, 3]), past_hi)
            if kind != "prefill":
                n_decode = _log_int(rng, 1, 160)
                ctx_hi = _log_int(rng, 64, 32768)
                ctx = (max(1, ctx_hi // rng.choice([1, 4, 8])), ctx_hi)
            mask = rng.choice(["causal", "window", "documents", "prefix"])
            window = _log_int(rng, 16, 8192) if mask == "window" else 0
            if mask == "documents":
                doc_hi = _log_int(rng, 20, 4000)
                docs = (max(1, doc_hi // rng.choice([1, 4, 20])), doc_hi)
            if mask == "prefix":
                prefix_hi = _log_int(rng, 16, 2000)
                prefix = (prefix_hi // rng.choice([1, 2, 8]), prefix_hi)
            change = rng.choice(["cap", "cap", "slopes", "both"] + (["none"] if mask != "causal" else []))
            case = _scores("", heads=rng.choice(_HEADS), dtype=rng.choice(["fp16", "bf16"]),
                           block=rng.choice([0, 16, 16, 16, 64, 24]), head_major=rng.random() < 0.2, n_prefill=n_prefill,
                           q=q, past=past, n_decode=n_decode, ctx=ctx, window=window, docs=docs, prefix=prefix,
                           cap=rng.choice([5.0, 20.0, 30.0, 50.0]) if change in ("cap", "both") else 0.0,
                           slopes=change in ("slopes", "both"), spread=rng.choice([1.0, 1.0, 2.0, 4.0]),
                           lens_seed=rng.randrange(1, 1 << 30))
        elif op == "append":
            heads = rng.choice(_HEADS)
            d = heads[2]
            scaling = rng.choice(["none", "linear", "parts", "index"])
            pos_hi = _log_int(rng, 2, 1 << 20)
            case = _append("", heads=heads, rows=_log_int(rng, 1, 8192), padded=rng.choice([0, 0, _log_int(rng, 1, 200)]),
                           dtype=rng.choice(["fp16", "bf16"]), block=rng.choice([0, 16, 16, 64, 24]),
                           head_major=rng.random() < 0.2, layout=rng.choice(["half", "half", "interleaved"]),
                           rot=rng.choice([d, d, d // 2, 16]), theta=rng.choice([1e4, 5e5, 1e6]), scaling=scaling,
                           factor=1.0 if scaling == "none" else rng.choice([2.0, 8.0, 32.0]), norm=rng.random() < 0.6,
                           offset=rng.choice([0.0, 1.0]), pos=(pos_hi // rng.choice([2, 7]), pos_hi),
                           packed=rng.random() < 0.7, lens_seed=rng.randrange(1, 1 << 30))
        else:
            n_prefill = rng.choice([0, 1, 3, 6, 20])
            q_hi = _log_int(rng, 2, 8192)
            past_hi = _log_int(rng, 1, 30000)
            ctx_hi = _log_int(rng, 1, 32768)
            case = _tables("", block=rng.choice([16, 16, 64, 24, 1]), n_prefill=n_prefill, q=(max(1, q_hi // 3), q_hi),
                           past=(past_hi // 4, past_hi), n_decode=_log_int(rng, 1, 600), ctx=(max(1, ctx_hi // 6), ctx_hi),
                           padded=rng.choice([0, 37]), lens_seed=rng.randrange(1, 1 << 30))
        if _cost(case) <= _cost(next(c for c in listed() if c["name"] == "capped_long")):
            del case["name"]
            return case


def _lengths(case):
    """((new tokens, visible tokens) per chunk, context per decode)."""
    rng = random.Random(case["lens_seed"])
    prefill = []
    for _ in range(case["n_prefill"]):
        q = rng.randint(case["q_lo"], case["q_hi"])
        prefill.append((q, q + rng.randint(case["past_lo"], case["past_hi"])))
    return prefill, [rng.randint(case["ctx_lo"], case["ctx_hi"]) for _ in range(case["n_decode"])]


def _masks(case):
    """What the masks are made of: (first key of each row's document or None, prefix length of each request or None).

    A chunk's documents follow each other from its first new token on; the first one may have begun in the cached
    part.  About one document in eight is padding: its rows see nothing."""
    prefill, decode = _lengths(case)
    rng = random.Random(case["lens_seed"] + 1)
    docs = prefix = None
    if case["doc_hi"]:
        docs = []
        for q, kv in prefill:
            t = kv - q
            start = max(0, t - rng.randint(0, case["doc_hi"]))
            while t < kv:
                n = min(rng.randint(case["doc_lo"], case["doc_hi"]), kv - t)
                docs += [start] * n if rng.random() >= 0.125 else [kv] * n
                t += n
                start = t
        docs += [max(0, kv - rng.randint(1, case["doc_hi"])) for kv in decode]
    if case["prefix_hi"]:
        prefix = [min(kv, rng.randint(case["prefix_lo"], case["prefix_hi"])) for _, kv in prefill] + [0] * len(decode)
    return docs, prefix


def _intervals(case):
    """Per request: (first visible key, end, position) of each of its rows, as lists."""
    prefill, decode = _lengths(case)
    docs, prefix = _masks(case)
    out, row = [], 0
    for r, (q, kv) in enumerate(prefill + [(1, n) for n in decode]):
        first, end, at = [], [], []
        for i in range(q):
            pos = kv - q + i
            a = max(0, pos - case["window"] + 1) if case["window"] else 0
            if docs is not None:
                a = max(a, docs[row])
            first.append(a)
            end.append(max(pos + 1, prefix[r]) if prefix is not None else pos + 1)
            at.append(pos)
            row += 1
        out.append((first, end, at))
    return out


def work(case):
    """Each input read once, each output written once; 4*d operations per visible (row, key) pair and query head."""
    if case["op"] == "tables":
        prefill, decode = _lengths(case)
        bs = case["block"]
        rows = sum(q for q, _ in prefill) + len(decode) + case["padded"]
        new = sum(-(-kv // bs) - -(-(kv - q) // bs) for q, kv in prefill + [(1, n) for n in decode])
        return {"bytes": 16 * (len(prefill) + len(decode)) + 8 * rows + 8 * new, "flops": 0}
    row_bytes = 2 * case["d"]
    if case["op"] == "append":
        values = case["rows"] * (case["hq"] + 2 * case["hkv"]) * case["d"]
        rotated = case["rows"] * (case["hq"] + case["hkv"]) * case["rot"]
        normed = case["rows"] * (case["hq"] + case["hkv"]) * case["d"] if case["norm"] else 0
        return {"bytes": 4 * values + 8 * (case["rows"] + case["padded"]), "flops": 3 * rotated + 4 * normed}
    pairs = keys = rows = 0
    for first, end, _ in _intervals(case):
        seen = [(a, e) for a, e in zip(first, end) if a < e]
        pairs += sum(e - a for a, e in seen)
        rows += len(first)
        reach = 0                                    # keys that some row sees, each counted once (firsts do not fall)
        for a, e in sorted(seen):
            keys += max(0, e - max(a, reach))
            reach = max(reach, e)
    return {"bytes": row_bytes * (2 * rows * case["hq"] + 2 * keys * case["hkv"]),
            "flops": 4 * case["d"] * case["hq"] * pairs}


def _cost(case):
    w = work(case)
    return w["bytes"] / 6e12 + w["flops"] / 8e14


# ---------------------------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------------------------
def _randn(gen, dtype, *shape, scale=1.0):
    return (torch.randn(*shape, generator=gen, device="cuda:0") * scale).to(dtype)


def _slots(case, lens, gen):
    """A block table for sequences of these lengths: blocks in an order of their own, a few to spare."""
    bs = case["block"]
    per = [-(-n // bs) for n in lens]
    n_blocks = sum(per) + 3
    perm = torch.randperm(n_blocks, generator=gen, device="cuda:0").to(torch.int32)
    table = torch.full((len(lens), max(per)), -1, dtype=torch.int32, device="cuda:0")
    owner = torch.repeat_interleave(torch.arange(len(lens)), torch.tensor(per)).cuda()
    starts = torch.tensor(per).cumsum(0) - torch.tensor(per)
    index = torch.arange(sum(per), device="cuda:0") - starts.cuda()[owner]
    table[owner, index] = perm[:sum(per)]
    return table, n_blocks


def _scores_inputs(case, seed):
    gen = torch.Generator(device="cuda:0").manual_seed(seed)
    dt, hq, hkv, d, bs = _DTYPES[case["dtype"]], case["hq"], case["hkv"], case["d"], case["block"]
    prefill, decode = _lengths(case)
    lens = [kv for _, kv in prefill] + decode
    s = {"prefill_q": _randn(gen, dt, sum(q for q, _ in prefill), hq, d, scale=case["spread"]),
         "decode_q": _randn(gen, dt, len(decode), hq, d, scale=case["spread"]), "table": None, "n_blocks": 0}
    if bs:
        s["table"], s["n_blocks"] = _slots(case, lens, gen)
        shape = [s["n_blocks"], bs, hkv, d]
    else:
        shape = [len(lens), max(lens), hkv, d]
    if case["head_major"]:
        shape[1], shape[2] = shape[2], shape[1]
    s["k"], s["v"] = _randn(gen, dt, *shape), _randn(gen, dt, *shape)
    # slopes that fall by a constant factor from head to head, as trained models have them
    s["slopes"] = [2.0 ** (-8.0 * (h + 1) / hq) for h in range(hq)] if case["slopes"] else None
    s["out"] = torch.zeros(s["prefill_q"].shape[0] + len(decode), hq, d, dtype=dt, device="cuda:0")
    return s


def _append_inputs(case, seed):
    gen = torch.Generator(device="cuda:0").manual_seed(seed)
    rng = random.Random(case["lens_seed"])
    dt, hq, hkv, d, bs = _DTYPES[case["dtype"]], case["hq"], case["hkv"], case["d"], case["block"]
    rows, n = case["rows"], case["rows"] + case["padded"]
    # more than a few rows: chunks of prompts, whose positions follow each other; few: replies, each at its own
    pos, slot, at = [], [], 0
    step = bs if bs else 64
    order = list(range(n // step + 9 if rows > 64 else rows + 3))
    rng.shuffle(order)
    if rows > 64:
        t = rng.randint(case["pos_lo"], case["pos_hi"])
        for i in range(rows):
            if i and rng.random() < 1.0 / 1500:
                t = rng.randint(case["pos_lo"], case["pos_hi"])
            pos.append(t)
            slot.append(order[i // step] * step + i % step)
            t += 1
    else:
        for i in range(rows):
            t = rng.randint(case["pos_lo"], case["pos_hi"])
            pos.append(t)
            slot.append(order[i] * step + t % step)
    pos += [0] * case["padded"]
    slot += [-1] * case["padded"]
    blocks = len(order)
    shape = [blocks, step, hkv, d]
    if case["head_major"]:
        shape[1], shape[2] = shape[2], shape[1]
    s = {"k_cache": _randn(gen, dt, *shape), "v_cache": _randn(gen, dt, *shape), "step": step,
         "slots": torch.tensor(slot, dtype=torch.int32, device="cuda:0"),
         "positions": torch.tensor(pos, dtype=torch.int32, device="cuda:0"),
         "q_out": torch.zeros(n, hq, d, dtype=dt, device="cuda:0"), "q_weight": None, "k_weight": None}
    if case["packed"]:
        qkv = _randn(gen, dt, n, (hq + 2 * hkv) * d)
        s["q"], s["k"], s["v"] = qkv[:, :hq * d], qkv[:, hq * d:(hq + hkv) * d], qkv[:, (hq + hkv) * d:]
    else:
        s["q"], s["k"], s["v"] = (_randn(gen, dt, n, h * d) for h in (hq, hkv, hkv))
    if case["norm"]:
        for key in ("q_weight", "k_weight"):
            s[key] = (torch.rand(d, generator=gen, device="cuda:0") + 0.5 - case["offset"]).to(dt)
    return s


def _tables_inputs(case, seed):
    gen = torch.Generator(device="cuda:0").manual_seed(seed)
    prefill, decode = _lengths(case)
    bs, meta, at = case["block"], [], 0
    for r, (q, kv) in enumerate(prefill):
        meta.append((at, q, kv, r))
        at += q
    for i, kv in enumerate(decode):
        meta.append((i, 1, kv, len(prefill) + i))
    held = [-(-(kv - q) // bs) for _, q, kv, _ in meta]
    need = [-(-kv // bs) for _, _, kv, _ in meta]
    n_blocks = sum(need) + 50
    perm = torch.randperm(n_blocks, generator=gen, device="cuda:0").to(torch.int32)
    table = torch.full((len(meta), max(need)), -1, dtype=torch.int32, device="cuda:0")
    owner = torch.repeat_interleave(torch.arange(len(meta)), torch.tensor(held)).cuda()
    starts = (torch.tensor(held).cumsum(0) - torch.tensor(held)).cuda()
    index = torch.arange(sum(held), device="cuda:0") - starts[owner]
    table[owner, index] = perm[:sum(held)]
    n_rows = at + len(decode) + case["padded"]
    return {"meta": torch.tensor(meta, dtype=torch.int32, device="cuda:0"), "free": perm[sum(held):].clone(), "table": table,
            "n_blocks": n_blocks, "n_prefill": len(prefill), "n_decode": len(decode), "n_rows": n_rows}


def prepare(case, seed):
    make = {"scores": _scores_inputs, "append": _append_inputs, "tables": _tables_inputs}[case["op"]]
    s = make(case, seed)
    s["case"] = case
    if own:
        {"scores": _own_scores, "append": _own_append, "tables": _own_tables}[case["op"]](s)
    elif case["op"] == "scores":
        prefill, decode = _lengths(case)
        s["lens"] = [kv for _, kv in prefill] + decode
        s["intervals"] = [tuple(torch.tensor(x, device="cuda:0") for x in t) for t in _intervals(case)]
        if case["slopes"]:
            s["slopes"] = torch.tensor(s["slopes"], device="cuda:0")
    elif case["op"] == "append":
        s["real"] = (s["slots"] >= 0).nonzero()[:, 0]
    return s


# ---------------------------------------------------------------------------------------------
# The framework's operators
# ---------------------------------------------------------------------------------------------
def _own_scores(s):
    import numpy as np
    from paper_2410_18038_amd import pod
    from paper_2410_18038_amd import workloads as wl
    case = s["case"]
    prefill, decode = _lengths(case)
    docs, prefix = _masks(case)
    meta, at = [], 0
    for r, (q, kv) in enumerate(prefill):
        meta.append((at, q, kv, r))
        at += q
    meta += [(i, 1, kv, len(prefill) + i) for i, kv in enumerate(decode)]
    bs, table = case["block"], s["table"]
    max_len = s["k"].shape[2 if case["head_major"] else 1]
    s["batch"] = wl.HybridBatch(
        name="case", n_prefill=len(prefill), n_decode=len(decode), n_q_heads=case["hq"], n_kv_heads=case["hkv"],
        head_dim=case["d"], dtype={"fp16": wl.F16, "bf16": wl.BF16}[case["dtype"]], softmax_scale=case["d"] ** -0.5,
        block_size=bs, max_blocks_per_seq=table.shape[1] if bs else 0,
        kv_seq_stride=0 if bs else max_len * case["hkv"] * case["d"], n_cache_rows=len(meta), n_blocks=s["n_blocks"],
        max_len=table.shape[1] * bs if bs else max_len, seq_meta=np.array(meta, dtype=np.int32),
        prefill_q=s["prefill_q"], decode_q=s["decode_q"], k_cache=s["k"], v_cache=s["v"], block_table=table,
        head_major=case["head_major"])
    s["attn"] = pod.HybridAttention(s["batch"], scores=pod.Scores(logit_cap=case["cap"], window=case["window"],
                                                                  slopes=s["slopes"], doc_start=docs, prefix_len=prefix))


def _own_append(s):
    from paper_2410_18038_amd import pod
    case = s["case"]
    k = s["k_cache"]
    params = pod.make_params(n_prefill=0, n_decode=0, n_q_heads=case["hq"], n_kv_heads=case["hkv"], head_dim=case["d"],
                             dtype={"fp16": pod.F16, "bf16": pod.BF16}[case["dtype"]], softmax_scale=case["d"] ** -0.5,
                             block_size=case["block"], max_blocks_per_seq=1, n_cache_rows=k.shape[0], n_blocks=k.shape[0],
                             kv_seq_stride=0 if case["block"] else s["step"] * case["hkv"] * case["d"],
                             kv_order=pod.KV_HEAD_MAJOR if case["head_major"] else pod.KV_TOKEN_MAJOR)
    rope = pod.Rope(case["rot"], layout=case["layout"], theta=case["theta"], scaling=case["scaling"], factor=case["factor"],
                    trained_len=case["trained"], low=1.0, high=_HIGH[case["scaling"]], cos_sin_scale=_magnitude(case))
    norm = pod.HeadNorm(s["q_weight"], s["k_weight"], eps=1e-6, weight_offset=case["offset"]) if case["norm"] else None
    s["append"] = pod.TokenAppend(params, rope=rope, norm=norm, device="cuda:0")


def _own_tables(s):
    from paper_2410_18038_amd import pod
    case = s["case"]
    params = pod.make_params(n_prefill=s["n_prefill"], n_decode=s["n_decode"], n_q_heads=1, n_kv_heads=1, head_dim=128,
                             dtype=pod.BF16, softmax_scale=1.0, block_size=case["block"],
                             max_blocks_per_seq=s["table"].shape[1], n_cache_rows=s["table"].shape[0], n_blocks=s["n_blocks"])
    s["tables"] = pod.TokenTables(params, s["n_rows"], device="cuda:0")


def run(state):
    op = state["case"]["op"]
    if own:
        if op == "scores":
            return state["attn"].forward(state["batch"], out=state["out"])
        if op == "append":
            state["append"](state["q"], state["k"], state["v"], state["slots"], state["positions"], state["k_cache"],
                            state["v_cache"], q_out=state["q_out"])
            return state["q_out"], state["k_cache"], state["v_cache"]
        t = state["tables"].build(state["meta"], state["free"], state["table"])
        return t.slots, t.positions, t.report, state["table"]
    return {"scores": _plain_scores, "append": _plain_append, "tables": _plain_tables}[op](state)


# ---------------------------------------------------------------------------------------------
# Plain forms
# ---------------------------------------------------------------------------------------------
def _sequence(case, cache, table, r, n):
    """The first n cached tokens of sequence r as [n, Hkv, d]."""
    if case["block"]:
        x = cache[table[r, :-(-n // case["block"])].long()]
        if case["head_major"]:
            x = x.transpose(1, 2)
        return x.reshape(-1, case["hkv"], case["d"])[:n]
    return (cache[r].transpose(0, 1) if case["head_major"] else cache[r])[:n]


def _plain_scores(s):
    case = s["case"]
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    group, scale = hq // hkv, d ** -0.5
    rows_q = torch.cat([s["prefill_q"], s["decode_q"]])
    row = 0
    for r, (first, end, pos) in enumerate(s["intervals"]):
        n_rows, n = first.numel(), s["lens"][r]
        k = _sequence(case, s["k"], s["table"], r, n).float().permute(1, 2, 0).contiguous()    # [Hkv, d, n]
        v = _sequence(case, s["v"], s["table"], r, n).float().transpose(0, 1).contiguous()     # [Hkv, n, d]
        key = torch.arange(n, device="cuda:0")
        some = max(1, (1 << 30) // (hq * n))
        for a in range(0, n_rows, some):
            b = min(n_rows, a + some)
            q = rows_q[row + a:row + b].float().reshape(b - a, hkv, group, d).transpose(0, 1).reshape(hkv, -1, d)
            x = torch.matmul(q, k).mul_(scale).view(hkv, b - a, group, n)
            if case["cap"]:
                x = x.div_(case["cap"]).tanh_().mul_(case["cap"])
            if case["slopes"]:
                far = (key[None, :] - pos[a:b, None]).abs().float()
                x -= s["slopes"].view(hkv, 1, group, 1) * far[None, :, None, :]
            hidden = (key[None, :] < first[a:b, None]) | (key[None, :] >= end[a:b, None])
            x.masked_fill_(hidden[None, :, None, :], -math.inf)
            top = x.amax(-1, keepdim=True)
            x = x.sub_(torch.where(top == -math.inf, 0.0, top)).exp_()
            total = x.sum(-1, keepdim=True)
            y = torch.matmul(x.view(hkv, -1, n), v).view(hkv, b - a, group, d)
            y = torch.where(total == 0, 0.0, y / total)
            s["out"][row + a:row + b] = y.transpose(0, 1).reshape(b - a, hq, d).to(s["out"].dtype)
        row += n_rows
    return s["out"]


_HIGH = {"none": 4.0, "linear": 4.0, "parts": 4.0, "index": 32.0}


def _magnitude(case):
    """What cosine and sine are multiplied by: 1, or 0.1 ln(factor) + 1 where the context is stretched by index."""
    return 0.1 * math.log(case["factor"]) + 1.0 if case["scaling"] == "index" else 1.0


def _frequencies(case):
    """Radians per position of each rotated pair, in 64 bits."""
    rot, theta, factor, trained = case["rot"], case["theta"], case["factor"], case["trained"]
    i = torch.arange(rot // 2, dtype=torch.float64, device="cuda:0")
    f = theta ** (-2.0 * i / rot)
    low, high = 1.0, _HIGH[case["scaling"]]
    if case["scaling"] == "linear":
        return f / factor
    if case["scaling"] == "parts":        # kept above `high` turns over the trained length, stretched below `low`
        keep = ((trained * f / (2 * math.pi) - low) / (high - low)).clamp(0, 1)
        return f * keep + f / factor * (1 - keep)
    if case["scaling"] == "index":        # the same, linear in the pair's index between the two
        at = [rot * math.log(trained / (turns * 2 * math.pi)) / (2 * math.log(theta)) for turns in (high, low)]
        lo, hi = max(math.floor(at[0]), 0), min(math.ceil(at[1]), rot - 1)
        keep = 1 - ((i - lo) / max(hi - lo, 0.001)).clamp(0, 1)
        return f * keep + f / factor * (1 - keep)
    return f


def _plain_append(s):
    case = s["case"]
    hq, hkv, d, rot = case["hq"], case["hkv"], case["d"], case["rot"]
    real = s["real"]
    angle = s["positions"][real].double()[:, None, None] * _frequencies(case)
    scale = _magnitude(case)
    cos, sin = (angle.cos() * scale).float(), (angle.sin() * scale).float()

    def heads(x, n, weight):
        x = x[real].float().view(-1, n, d)
        if case["norm"] and weight is not None:
            x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6) * (weight.float() + case["offset"])
        if case["layout"] == "half":
            a, b = x[..., :rot // 2], x[..., rot // 2:rot]
            turned = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
        else:
            a, b = x[..., 0:rot:2], x[..., 1:rot:2]
            turned = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
        return torch.cat([turned, x[..., rot:]], -1).to(s["q_out"].dtype)

    s["q_out"][real] = heads(s["q"], hq, s["q_weight"])
    block, at = s["slots"][real].long() // s["step"], s["slots"][real].long() % s["step"]
    for cache, new in ((s["k_cache"], heads(s["k"], hkv, s["k_weight"])), (s["v_cache"], s["v"][real].view(-1, hkv, d))):
        if case["head_major"]:
            cache[block, :, at] = new
        else:
            cache[block, at] = new
    return s["q_out"], s["k_cache"], s["v_cache"]


def _plain_tables(s):
    case, meta, bs = s["case"], s["meta"].long(), s["case"]["block"]
    dev = meta.device
    start, q, kv, row = meta.unbind(1)
    held, need = (kv - q + bs - 1) // bs, (kv + bs - 1) // bs
    new = need - held
    total = new.sum()
    before = new.cumsum(0) - new
    table = s["table"]
    n_new = _new_blocks(case)
    owner = torch.repeat_interleave(torch.arange(len(meta), device=dev), new, output_size=n_new)
    k = torch.arange(n_new, device=dev) - before[owner]
    table[row[owner], held[owner] + k] = s["free"][before[owner] + k]
    n_prefill_rows = q[:s["n_prefill"]].sum()
    first = torch.where(torch.arange(len(meta), device=dev) < s["n_prefill"], start, start + n_prefill_rows)
    n_real = s["n_rows"] - case["padded"]
    owner = torch.repeat_interleave(torch.arange(len(meta), device=dev), q, output_size=n_real)
    i = torch.arange(n_real, device=dev) - (q.cumsum(0) - q)[owner]
    pos = (kv - q)[owner] + i
    slots = torch.full((s["n_rows"],), -1, dtype=torch.int32, device=dev)
    positions = torch.zeros(s["n_rows"], dtype=torch.int32, device=dev)
    slots[first[owner] + i] = (table[row[owner], pos // bs].long() * bs + pos % bs).int()
    positions[first[owner] + i] = pos.int()
    zero = torch.zeros_like(total)
    report = torch.stack([total, zero, zero, zero + n_real]).int()
    return slots, positions, report, table


def _new_blocks(case):
    prefill, decode = _lengths(case)
    bs = case["block"]
    return sum(-(-kv // bs) - -(-(kv - q) // bs) for q, kv in prefill + [(1, n) for n in decode])


# ---------------------------------------------------------------------------------------------
# The definitions in 64 bits
# ---------------------------------------------------------------------------------------------
def exact(case, seed):
    return {"scores": _exact_scores, "append": _exact_append, "tables": _exact_tables}[case["op"]](case, seed)


def _exact_scores(case, seed):
    """Softmax over each row's own visible keys, head by head."""
    s = _scores_inputs(case, seed)
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device="cuda:0")
    rows_q = torch.cat([s["prefill_q"], s["decode_q"]])
    prefill, decode = _lengths(case)
    lens = [kv for _, kv in prefill] + decode
    row = 0
    for r, (first, end, at) in enumerate(_intervals(case)):
        n_rows, n = len(first), lens[r]
        keys, values = (_sequence(case, s[x], s["table"], r, n).double() for x in ("k", "v"))
        first, end, at = (torch.tensor(x, device="cuda:0")[:, None] for x in (first, end, at))
        j = torch.arange(n, device="cuda:0")[None, :]
        step = max(1, (1 << 27) // n)
        for h in range(hq):
            k, v = keys[:, h * hkv // hq], values[:, h * hkv // hq]
            for a in range(0, n_rows, step):
                b = min(a + step, n_rows)
                z = rows_q[row + a:row + b, h].double() @ k.T / math.sqrt(d)
                if case["cap"]:
                    z = case["cap"] * torch.tanh(z / case["cap"])
                if case["slopes"]:
                    z = z - s["slopes"][h] * (at[a:b] - j).abs()
                seen = (j >= first[a:b]) & (j < end[a:b])
                w = torch.softmax(torch.where(seen, z, torch.full_like(z, -math.inf)), -1)
                out[row + a:row + b, h] = torch.where(seen.any(-1, keepdim=True), w @ v, torch.zeros_like(w @ v))
        row += n_rows
    return out


def _exact_append(case, seed):
    """Every pair of channels is a complex number, turned by its position times its frequency."""
    s = _append_inputs(case, seed)
    d, rot = case["d"], case["rot"]
    live = [i for i, x in enumerate(s["slots"].tolist()) if x >= 0]
    pos = torch.tensor(s["positions"].tolist(), dtype=torch.float64, device="cuda:0")[live]
    f = []
    low, high = 1.0, _HIGH[case["scaling"]]
    for i in range(rot // 2):
        w = math.pow(case["theta"], -2.0 * i / rot)
        if case["scaling"] == "linear":
            w /= case["factor"]
        elif case["scaling"] == "parts":
            g = (case["trained"] * w / (2 * math.pi) - low) / (high - low)
            g = min(1.0, max(0.0, g))
            w = (1 - g) * w / case["factor"] + g * w
        elif case["scaling"] == "index":
            def pair(turns):
                return rot * math.log(case["trained"] / (turns * 2 * math.pi)) / (2 * math.log(case["theta"]))
            lo, hi = max(math.floor(pair(high)), 0), min(math.ceil(pair(low)), rot - 1)
            g = min(1.0, max(0.0, (i - lo) / max(hi - lo, 0.001)))
            w = g * w / case["factor"] + (1 - g) * w
        f.append(w)
    turn = torch.polar(torch.full((len(live), rot // 2), _magnitude(case), dtype=torch.float64, device="cuda:0"),
                       pos[:, None] * torch.tensor(f, dtype=torch.float64, device="cuda:0"))[:, None, :]

    def heads(x, n, weight):
        x = x[live].double().reshape(len(live), n, d)
        if weight is not None:
            x = x / torch.sqrt(x.pow(2).sum(-1, keepdim=True) / d + 1e-6) * (weight.double() + case["offset"])
        y = x.clone()
        if case["layout"] == "half":
            z = torch.complex(x[..., :rot // 2].contiguous(), x[..., rot // 2:rot].contiguous()) * turn
            y[..., :rot // 2], y[..., rot // 2:rot] = z.real, z.imag
        else:
            z = torch.view_as_complex(x[..., :rot].reshape(len(live), n, rot // 2, 2).contiguous()) * turn
            y[..., :rot] = torch.view_as_real(z).flatten(-2)
        return y

    q_out = s["q_out"].double()
    q_out[live] = heads(s["q"], case["hq"], s["q_weight"])
    k_cache, v_cache = s["k_cache"].double(), s["v_cache"].double()
    keys, values = heads(s["k"], case["hkv"], s["k_weight"]), s["v"][live].double().reshape(len(live), case["hkv"], d)
    slot = s["slots"][live].long()
    block, at = slot // s["step"], slot % s["step"]
    for cache, new in ((k_cache, keys), (v_cache, values)):
        (cache.transpose(1, 2) if case["head_major"] else cache)[block, at] = new
    return q_out, k_cache, v_cache


def _exact_tables(case, seed):
    """Request by request, token by token."""
    s = _tables_inputs(case, seed)
    bs, free, table = case["block"], s["free"].tolist(), s["table"].tolist()
    meta = s["meta"].tolist()
    slots, positions = [-1] * s["n_rows"], [0] * s["n_rows"]
    n_prefill_rows, taken = sum(q for _, q, _, _ in meta[:s["n_prefill"]]), 0
    for r, (start, q, kv, row) in enumerate(meta):
        for i in range(q):
            pos = kv - q + i
            if pos % bs == 0:
                table[row][pos // bs] = free[taken]
                taken += 1
            at = start + i + (n_prefill_rows if r >= s["n_prefill"] else 0)
            slots[at], positions[at] = table[row][pos // bs] * bs + pos % bs, pos
    report = [taken, 0, 0, n_prefill_rows + s["n_decode"]]
    return tuple(torch.tensor(x, dtype=torch.int32, device="cuda:0") for x in (slots, positions, report, table))
