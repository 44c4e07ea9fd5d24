"""Attention with changed scores: capped, falling with distance, masked by windows, documents and prefixes.

The reference is numpy in 64 bits, straight from the definition in the header.  How far a result may be off follows from
what is rounded: weights to the 16-bit type before the second product (half a step each, in the sum and in what it is
divided by), the result (half a step), and scores in 32 bits (2^-19 of a dot product's magnitude, 2^-21 of the cap, or
2^-20 of the largest score where all are below half of it, and 2^-21 of the largest bias, as a relative error of the
weights); in fp16, weights below 2^-24 of the largest are lost (half of that each).
"""
import ctypes
import dataclasses

import numpy as np
import pytest
import torch

from paper_2410_18038_amd import pod
from paper_2410_18038_amd import workloads as wl

TDT = {wl.F16: torch.float16, wl.BF16: torch.bfloat16}


# -- reference ------------------------------------------------------------------------------------- #
def intervals(batch, scores):
    """(first, end, position) of every output row."""
    n = batch.n_rows
    first, end, at = np.zeros(n, np.int64), np.zeros(n, np.int64), np.zeros(n, np.int64)
    for r, (start, q_len, kv_len, _) in enumerate(batch.seq_meta.tolist()):
        row0 = start + (batch.n_prefill_rows if r >= batch.n_prefill else 0)
        for i in range(q_len):
            pos = kv_len - q_len + i
            a = max(0, pos - scores.window + 1) if scores.window else 0
            if scores.doc_start is not None:
                a = max(a, scores.doc_start[row0 + i])
            b = pos + 1
            if scores.prefix_len is not None:
                b = max(b, min(scores.prefix_len[r], kv_len))
            first[row0 + i], end[row0 + i], at[row0 + i] = a, b, pos
    return first, end, at


def logical(batch, cache, r):
    """[kv_len, Hkv, d] of one request, in float64."""
    _, _, kv_len, row = (int(x) for x in batch.seq_meta[r])
    c = cache.transpose(1, 2) if batch.head_major else cache
    if batch.block_size:
        t = np.arange(kv_len)
        blocks = batch.block_table[row].long()[torch.from_numpy(t // batch.block_size)].clamp(min=0)
        return wl.as_f64(c[blocks, torch.from_numpy(t % batch.block_size)])
    return wl.as_f64(c[row, :kv_len])


def reference(batch, scores):
    """(result, tolerance), float64 [rows, Hq, d], of a batch on the CPU."""
    hq, hkv, d = batch.n_q_heads, batch.n_kv_heads, batch.head_dim
    out, tol = np.zeros((batch.n_rows, hq, d)), np.zeros((batch.n_rows, hq, d))
    first, end, at = intervals(batch, scores)
    q_all = np.concatenate([wl.as_f64(batch.prefill_q), wl.as_f64(batch.decode_q)])
    half = torch.finfo(TDT[batch.dtype]).eps / 2
    for r, (start, q_len, kv_len, _) in enumerate(batch.seq_meta.tolist()):
        row0 = start + (batch.n_prefill_rows if r >= batch.n_prefill else 0)
        rows = slice(row0, row0 + q_len)
        key = np.arange(kv_len)
        seen = (key >= first[rows, None]) & (key < end[rows, None])
        k_all, v_all = logical(batch, batch.k_cache, r), logical(batch, batch.v_cache, r)
        with np.errstate(invalid="ignore"):
            raw = [np.nanmax(np.abs(q_all[rows, h] @ k_all[:, h * hkv // hq].T), initial=0) * batch.softmax_scale for h in range(hq)]
        for h in range(hq):
            k, v, q = k_all[:, h * hkv // hq], v_all[:, h * hkv // hq], q_all[rows, h]
            with np.errstate(invalid="ignore"):
                s = q @ k.T * batch.softmax_scale
                size = np.abs(q) @ np.abs(k).T * batch.softmax_scale
            delta = 2.0 ** -19 * np.where(seen, size, 0).max(-1)
            if scores.logit_cap:
                s = scores.logit_cap * np.tanh(s / scores.logit_cap)
                below = np.nanmax(raw) <= 0.45 * scores.logit_cap        # every score of the request: the polynomial's error is relative
                delta += 2.0 ** -20 * np.where(seen, np.abs(s), 0).max(-1) if below else 2.0 ** -21 * scores.logit_cap
            if scores.slopes is not None:
                far = np.abs(key - at[rows, None])
                s = s - scores.slopes[h] * far
                delta += 2.0 ** -21 * abs(scores.slopes[h]) * far.max()
            s = np.where(seen, s, -np.inf)
            top = s.max(-1, keepdims=True)
            w = np.exp(s - np.where(np.isinf(top), 0, top))
            total = w.sum(-1, keepdims=True)
            w = w / np.where(total == 0, 1, total)                       # (a score that is no number makes its row none)
            o, size_v = np.zeros((q_len, d)), np.zeros((q_len, d))
            for i in range(q_len):                                       # what a row does not see is not even multiplied by 0
                o[i], size_v[i] = w[i, seen[i]] @ v[seen[i]], w[i, seen[i]] @ np.abs(v[seen[i]])
            out[rows, h] = o
            lost = 2.0 ** -25 * kv_len * np.abs(np.where(np.isfinite(v), v, 0)).max() if batch.dtype == wl.F16 else 0.0
            tol[rows, h] = half * 1.01 * (2 * size_v + np.abs(o)) + size_v * (2 * delta[:, None] + 2.0 ** -18) + lost + 2.0 ** -24
    return out, tol


def poison_unseen(batch, scores, value=float("nan")):
    """The batch with every cached token that no row of its request sees overwritten, and blocks of such tokens alone
    replaced in the table by a block of them."""
    first, end, _ = intervals(batch, scores)
    k, v = batch.k_cache.clone(), batch.v_cache.clone()
    table = None if batch.block_table is None else batch.block_table.clone()
    bs = batch.block_size
    for r, (start, q_len, kv_len, row) in enumerate(batch.seq_meta.tolist()):
        row0 = start + (batch.n_prefill_rows if r >= batch.n_prefill else 0)
        seen = np.zeros(kv_len, bool)
        for i in range(row0, row0 + q_len):
            seen[first[i]:end[i]] = True
        for t in np.flatnonzero(~seen).tolist():
            at = (int(table[row, t // bs]), t % bs) if bs else (row, t)
            if batch.head_major:
                k[at[0], :, at[1]] = v[at[0], :, at[1]] = value
            else:
                k[at] = v[at] = value
        if bs:
            spare = next(b for b in range(batch.n_blocks) if not (batch.block_table == b).any())
            k[spare] = v[spare] = value
            for b in range(-(-kv_len // bs)):
                if not seen[b * bs:(b + 1) * bs].any():
                    table[row, b] = spare
    return dataclasses.replace(batch, k_cache=k, v_cache=v, block_table=table)


def run(batch, scores, mode="fused", **plan_kw):
    dev = batch.to("cuda:0")
    attn = pod.HybridAttention(dev, scores=scores, **plan_kw)
    out = torch.full((batch.n_rows, batch.n_q_heads, batch.head_dim), 7.0, dtype=batch.torch_dtype, device="cuda:0")
    attn.forward(dev, out=out, mode=pod.MODES[mode])
    torch.cuda.synchronize()
    info = attn.info
    attn.close()
    return out.cpu(), info


def check(batch, scores, mode="fused", want=None, **plan_kw):
    print(f"case {batch.name} {mode} {scores} {plan_kw}"[:300], flush=True)
    got, info = run(batch, scores, mode, **plan_kw)
    want = reference(batch, scores) if want is None else want
    got = wl.as_f64(got)
    assert np.isfinite(got).all(), "non-finite GPU output"
    over = (np.abs(got - want[0]) / want[1]).max()
    assert over <= 1.0, f"{over:.3f} of the tolerance ({batch.name}, {mode})"
    return info


def slopes(hq):
    return [2.0 ** (-8.0 * (h + 1) / hq) for h in range(hq)]


def documents(batch, lens, seed):
    """First keys for documents of lens[0]..lens[1] tokens that follow each other; some of them padding."""
    rng = np.random.default_rng(seed)
    out = np.zeros(batch.n_rows, np.int32)
    for r, (start, q_len, kv_len, _) in enumerate(batch.seq_meta.tolist()):
        row0 = start + (batch.n_prefill_rows if r >= batch.n_prefill else 0)
        t = kv_len - q_len
        begin = max(0, t - int(rng.integers(0, lens[1])))
        while t < kv_len:
            n = min(int(rng.integers(lens[0], lens[1] + 1)), kv_len - t)
            out[row0 + t - (kv_len - q_len):row0 + t + n - (kv_len - q_len)] = begin if rng.random() > 0.25 else kv_len
            t += n
            begin = t
    return out.tolist()


def variant(name, batch):
    hq, n_req = batch.n_q_heads, len(batch.seq_meta)
    return {"nothing": lambda: pod.Scores(), "cap": lambda: pod.Scores(logit_cap=3.0), "slopes": lambda: pod.Scores(slopes=slopes(hq)),
            "window": lambda: pod.Scores(window=37), "documents": lambda: pod.Scores(doc_start=documents(batch, (5, 150), 1), logit_cap=30.0),
            "prefix": lambda: pod.Scores(prefix_len=[(29 * (r + 1)) % 400 for r in range(n_req)], slopes=slopes(hq)),
            "all": lambda: pod.Scores(logit_cap=20.0, window=100, slopes=slopes(hq), doc_start=documents(batch, (20, 300), 2),
                                      prefix_len=[150] * n_req)}[name]()


VARIANTS = ["nothing", "cap", "slopes", "window", "documents", "prefix", "all"]


# -- refusals and plans (host) ----------------------------------------------------------------------- #
def plain_params(b, **kw):
    kw = {**dict(n_prefill=b.n_prefill, n_decode=b.n_decode, n_q_heads=b.n_q_heads, n_kv_heads=b.n_kv_heads, head_dim=b.head_dim,
                 dtype=b.dtype, softmax_scale=b.softmax_scale, block_size=b.block_size, max_blocks_per_seq=b.max_blocks_per_seq,
                 n_cache_rows=b.n_cache_rows, n_blocks=b.n_blocks, kv_seq_stride=b.kv_seq_stride, n_compute_units=256), **kw}
    return pod.make_params(**kw)


def test_score_arguments_are_checked():
    b = wl.config_batch(1)
    plan = lambda scores, **kw: pod.pod_attn_plan_create_scored(plain_params(b, **kw), scores, b.seq_meta)
    plan(pod.Scores()).close()
    n_req = len(b.seq_meta)
    bad_slope, bad_doc, bad_prefix = [0.5] * 4, [0] * b.n_rows, [0] * n_req
    bad_slope[2], bad_doc[-1], bad_prefix[0] = float("inf"), -1, -3
    for scores in [pod.Scores(logit_cap=-1.0), pod.Scores(logit_cap=float("nan")), pod.Scores(logit_cap=float("inf")), pod.Scores(window=-1),
                   pod.Scores(slopes=bad_slope), pod.Scores(doc_start=bad_doc), pod.Scores(prefix_len=bad_prefix)]:
        with pytest.raises(pod.PodError) as e:
            plan(scores)
        assert e.value.status == -1 and len(str(e.value)) > 15
    for scores in [pod.Scores(logit_cap=1e21), pod.Scores(logit_cap=1e-30), pod.Scores(slopes=[1e25] * 4), pod.Scores(slopes=[0.0, -1e20, 0.0, 0.0])]:
        with pytest.raises(pod.PodError) as e:
            plan(scores)
        assert e.value.status == -1 and "too" in str(e.value)
    for scores in [pod.Scores(slopes=[1.0]), pod.Scores(doc_start=[0]), pod.Scores(prefix_len=[0] * (n_req + 1))]:
        with pytest.raises(ValueError):
            plan(scores)
    with pytest.raises(pod.PodError) as e:
        plan(pod.Scores(), head_dim=96)
    assert e.value.status == -2
    for scores in [pod.Scores(window=2**32 + 1), pod.Scores(logit_cap=1e-60)]:           # values that change on their way to 32 bits
        with pytest.raises(ValueError):
            plan(scores)
    wide = wl.config_batch(1)
    wide = dataclasses.replace(wide, head_dim=128, softmax_scale=1.0, kv_seq_stride=2 * wide.kv_seq_stride)   # head_dim 128, contiguous: built for the configuration otherwise
    plan = pod.pod_attn_plan_create_scored(plain_params(wide), pod.Scores(logit_cap=5.0), wide.seq_meta)
    assert not plan.info().prefill_heavy_advised and not plan.info().prefill_heavy_chosen
    for mode in ("fused_heavy", "prefill_only_heavy", "decode_only_lite"):
        with pytest.raises(pod.PodError) as e:
            pod.pod_attn_forward(16, 16, 16, 16, 16, 0, 16, plan, 256, 1 << 40, pod.MODES[mode])
        assert e.value.status == -2 and "changed scores" in str(e.value)
    plan.close()


def test_struct_layout_of_the_scores_matches_the_header(tmp_path):
    import os
    import subprocess
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    src = tmp_path / "sizes.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "pod_attn.h"\nint main(void){printf("%zu %zu %zu\\n",'
                   ' sizeof(pod_attn_scores), offsetof(pod_attn_scores, slopes), offsetof(pod_attn_scores, prefix_len)); return 0;}\n')
    exe = tmp_path / "sizes"
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.join(root, "include"), str(src), "-o", str(exe)], check=True)
    got = [int(x) for x in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()]
    assert got == [ctypes.sizeof(pod.ScoresParams), pod.ScoresParams.slopes.offset, pod.ScoresParams.prefix_len.offset]


def test_a_plan_without_scores_is_the_plain_one():
    b = wl.config_batch(1)
    one, other = (make(plain_params(b)) for make in (lambda p: pod.pod_attn_plan_create(p, b.seq_meta),
                                                     lambda p: pod.pod_attn_plan_create_scored(p, None, b.seq_meta)))
    assert bytes(one.info()) == bytes(other.info())
    assert (one.prefill_items() == other.prefill_items()).all() and (one.decode_units() == other.decode_units()).all()


def plan_batch(prefill, decode, hq, hkv, d, block, seed=1):
    """Lengths only (no tensors)."""
    meta, at = [], 0
    for r, (q, kv) in enumerate(prefill):
        meta.append((at, q, kv, r))
        at += q
    meta += [(i, 1, kv, len(prefill) + i) for i, kv in enumerate(decode)]
    longest = max(m[2] for m in meta)
    return dataclasses.replace(
        wl.config_batch(1), name="plan", n_prefill=len(prefill), n_decode=len(decode), n_q_heads=hq, n_kv_heads=hkv, head_dim=d,
        block_size=block, max_blocks_per_seq=-(-longest // block) if block else 0, kv_seq_stride=0 if block else longest * hkv * d,
        n_cache_rows=len(meta), n_blocks=10 ** 5 if block else 0, seq_meta=np.array(meta, np.int32),
        prefill_q=torch.empty(at, 0, 0), decode_q=torch.empty(len(decode), 0, 0))


@pytest.mark.parametrize("name", VARIANTS)
@pytest.mark.parametrize("prefill,decode,hq,hkv,d,kw", [
    ([(300, 900), (1, 1), (64, 64)], [1, 15, 16, 17, 700, 5000], 8, 2, 128, {}),
    ([(700, 4000)], [9000] * 40, 32, 8, 128, dict(prefill_split_len=256, max_prefill_waves=64)),
    ([(500, 2000)], [3000] * 3, 15, 5, 64, dict(decode_chunk=256, prefill_split_len=64, max_prefill_waves=64)),
    ([(700, 700)], [], 4, 4, 256, {}), ([], [40, 4000, 1], 8, 1, 256, {})])
def test_plans_cover_what_each_row_sees(name, prefill, decode, hq, hkv, d, kw):
    """Every visible key of a row is in exactly one item (or unit) of its K/V head, and no key is read that no row sees."""
    b = plan_batch(prefill, decode, hq, hkv, d, 16)
    scores = variant(name, b)
    plan = pod.pod_attn_plan_create_scored(plain_params(b, **kw), scores, b.seq_meta)
    first, end, _ = intervals(b, scores)
    group, items = hq // hkv, plan.prefill_items().tolist()
    for r, (start, q_len, kv_len, _) in enumerate(b.seq_meta[:len(prefill)].tolist()):
        for kvh in range(hkv):
            count = np.zeros((q_len * group, kv_len), np.int8)
            for req, head, row0, n_rows, k0, k1, prow0, split in items:
                if req == r and head == kvh:
                    assert 0 <= k0 <= k1 <= kv_len and 0 <= row0 and row0 + n_rows <= q_len * group
                    count[row0:row0 + n_rows, k0:k1] += 1
                    rows = start + np.arange(row0, row0 + n_rows) // group
                    some = first[rows] < end[rows]
                    assert k0 == k1 if not some.any() else first[rows][some].min() <= k0 < k1 <= end[rows][some].max()
                    assert split == 0 or k0 % 16 == 0
            rows = start + np.arange(q_len * group) // group
            key = np.arange(kv_len)
            seen = (key >= first[rows, None]) & (key < end[rows, None])
            assert (count[seen] == 1).all() and (count <= 1).all()
    units = plan.decode_units().tolist()
    for i, (_, _, kv_len, _) in enumerate(b.seq_meta[len(prefill):].tolist()):
        row = b.n_prefill_rows + i
        for kvh in range(hkv):
            cuts = sorted((u[2], u[3]) for u in units if u[0] == len(prefill) + i and u[1] == kvh)
            if first[row] >= end[row]:
                assert cuts == []
                continue
            assert cuts[0][0] == first[row] and cuts[-1][1] == end[row] and all(a < b for a, b in cuts)
            assert all(x[1] == y[0] and y[0] % 16 == 0 for x, y in zip(cuts, cuts[1:]))
    plan.close()


@pytest.mark.parametrize("prefill,decode", [([(300, 900), (1, 1)], [1, 700, 5000]), ([], [40, 1]), ([(64, 64)], [])])
@pytest.mark.parametrize("kw", [{}, dict(decode_chunk=256, prefill_split_len=64, max_prefill_waves=64), dict(n_compute_units=3)])
def test_plans_of_batches_that_see_nothing_hold_no_keys(prefill, decode, kw):
    b = plan_batch(prefill, decode, 8, 2, 128, 16)
    plan = pod.pod_attn_plan_create_scored(plain_params(b, **kw), pod.Scores(doc_start=[1 << 30] * b.n_rows), b.seq_meta)
    assert plan.info().n_decode_units == 0 and plan.info().n_partial_rows == 0
    assert all(k0 == k1 == 0 for _, _, _, _, k0, k1, _, _ in plan.prefill_items().tolist())
    plan.close()


# -- parity (GPU) ------------------------------------------------------------------------------------- #
GRID = [   # query heads, K/V heads, channels, type, block, head-major
    (8, 2, 128, wl.BF16, 16, False), (4, 4, 128, wl.F16, 0, False), (9, 3, 64, wl.F16, 24, False), (16, 1, 64, wl.BF16, 64, True),
    (4, 2, 256, wl.F16, 16, False), (8, 1, 256, wl.BF16, 0, True), (5, 5, 128, wl.F16, 1, False), (10, 5, 64, wl.BF16, 0, False),
    (6, 3, 256, wl.BF16, 6, False), (15, 5, 128, wl.BF16, 24, True)]


def grid_batch(hq, hkv, d, dtype, block, head_major, *, prefill=((200, 333), (37, 37), (1, 90)), decode=(1, 31, 32, 33, 257, 700), seed=0):
    b = wl.make_batch(f"{hq}/{hkv}-d{d}-bs{block}", prefill=list(prefill), decode_kv_lens=list(decode), n_q_heads=hq, n_kv_heads=hkv,
                      head_dim=d, dtype=dtype, seed=5000 + hq + hkv + d + block + seed, block_size=block, poison=float("nan"))
    return wl.to_head_major(b) if head_major else b


@pytest.mark.gpu
@pytest.mark.parametrize("name", VARIANTS)
@pytest.mark.parametrize("shape", GRID, ids=lambda s: "-".join(str(x) for x in s))
def test_changed_scores_match_the_definition(shape, name):
    """All changes over all head layouts, types and caches; what no row sees is NaN."""
    batch = grid_batch(*shape)
    scores = variant(name, batch)
    check(poison_unseen(batch, scores), scores)


@pytest.mark.gpu
@pytest.mark.parametrize("mode", ["fused", "serial", "streams", "fused_cta"])
@pytest.mark.parametrize("d,block", [(128, 16), (64, 0), (256, 24)])
def test_split_work_merges_to_the_same_result_in_every_mode(mode, d, block):
    batch = wl.make_batch(f"split-{d}", prefill=[(96, 1500), (70, 800)], decode_kv_lens=[1200, 90, 2047, 640, 5], n_q_heads=8, n_kv_heads=2,
                          head_dim=d, dtype=wl.BF16, seed=61, block_size=block, poison=float("nan"))
    for name in ("cap", "all", "documents"):
        scores = variant(name, batch)
        hidden = poison_unseen(batch, scores)
        want = reference(hidden, scores)
        info = check(hidden, scores, mode, want=want, decode_chunk=256, prefill_split_len=128, max_prefill_waves=64)
        assert name != "cap" or (info.max_decode_splits > 1 and info.max_prefill_splits > 1)
        check(hidden, scores, mode, want=want)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [wl.F16, wl.BF16])
@pytest.mark.parametrize("cap,spread", [(0.5, 1.0), (5.0, 30.0), (50.0, 4.0), (1000.0, 20.0), (30.0, 0.02), (1e6, 1.0),
                                        (1e-6, 1.0), (1e-18, 1.0), (1e18, 1.0)])
def test_caps_from_far_below_the_scores_to_far_above(dtype, cap, spread):
    batch = grid_batch(8, 2, 128, dtype, 16, False, decode=(5, 300, 1000))
    batch = dataclasses.replace(batch, prefill_q=(batch.prefill_q.float() * spread).to(batch.torch_dtype),
                                decode_q=(batch.decode_q.float() * spread).to(batch.torch_dtype))
    batch.prefill_q[3] = 0                                               # scores of exactly 0
    batch.decode_q[0] = 0
    check(batch, pod.Scores(logit_cap=cap))


@pytest.mark.gpu
@pytest.mark.parametrize("slope", [8.0, 0.25, 0.001, 0.0, -0.02])
@pytest.mark.parametrize("shape", [GRID[0], GRID[2], GRID[4]], ids=["128", "64", "256"])
def test_slopes_from_steep_to_rising(shape, slope):
    batch = grid_batch(*shape, prefill=((150, 150), (40, 700)), decode=(1, 64, 1500))
    check(batch, pod.Scores(slopes=[slope * (1 + h / 7) for h in range(batch.n_q_heads)], prefix_len=[90, 100, 0, 0, 700]))


@pytest.mark.gpu
@pytest.mark.parametrize("window", [1, 2, 16, 63, 64, 65, 333, 5000])
def test_windows_around_the_edges_of_tiles_and_steps(window):
    for shape in (GRID[0], GRID[2], GRID[8]):
        batch = grid_batch(*shape, prefill=((129, 400), (1, 1)), decode=(1, 16, 17, 400, 601))
        scores = pod.Scores(window=window)
        check(poison_unseen(batch, scores), scores)


@pytest.mark.gpu
@pytest.mark.parametrize("shape", [(32, 8, 128, wl.BF16, 16, False), (8, 1, 64, wl.F16, 0, False), (6, 3, 128, wl.F16, 24, True)])
@pytest.mark.parametrize("prefill", [(), ((40, 300),)])
def test_units_of_one_round_merge_their_groups(shape, prefill):
    """Decodes cut into two to eight units each, with and without a chunk beside them, some seeing nothing; called again and
    again, since the units' counters have to be back at zero."""
    batch = grid_batch(*shape, prefill=prefill, decode=(400, 390, 1, 512, 300, 450), seed=9)
    far = 1 << 30
    for scores in (pod.Scores(logit_cap=4.0), pod.Scores(window=350, slopes=slopes(shape[0])),
                   pod.Scores(doc_start=[0] * (batch.n_rows - 6) + [far, 100, 0, 7, far, 33])):
        hidden = poison_unseen(batch, scores)
        want = reference(hidden, scores)
        info = check(hidden, scores, want=want)
        assert 2 <= info.max_decode_splits <= 8 and info.n_decode_units <= 1024
        dev = hidden.to("cuda:0")
        attn = pod.HybridAttention(dev, scores=scores)
        first = attn.forward(dev).clone()
        for mode in ("fused", "serial", "fused", "streams", "fused_cta", "fused"):
            again = attn.forward(dev, mode=pod.MODES[mode])
            torch.cuda.synchronize()
            assert torch.equal(again, first), mode
        attn.close()


@pytest.mark.gpu
def test_rows_that_see_nothing_are_zero():
    """Single rows, blocks of rows, whole requests, a whole batch; beside rows that see keys and alone."""
    for shape in (GRID[0], GRID[1], GRID[4]):
        batch = grid_batch(*shape, prefill=((300, 300), (40, 90)), decode=(1, 70, 300))
        far = 1 << 30
        docs = [0] * batch.n_rows
        docs[3] = docs[310] = far
        docs[64:270] = [far] * 206
        docs[-1] = docs[-3] = far
        for kw in ({}, dict(decode_chunk=64, prefill_split_len=64, max_prefill_waves=64)):
            for mode in ("fused", "serial", "streams"):
                check(batch, pod.Scores(doc_start=docs), mode, **kw)
        got, info = run(batch, pod.Scores(doc_start=[far] * batch.n_rows))
        assert (got == 0).all() and info.n_decode_units == 0
        got, _ = run(batch, pod.Scores(doc_start=docs), "decode_only")
        n = batch.n_prefill_rows
        assert (got[:n] == 7).all() and (got[n] == 0).all() and (got[n + 2] == 0).all() and not (got[n + 1] == 7).any()
        got, _ = run(batch, pod.Scores(doc_start=docs), "prefill_only")
        assert (got[n:] == 7).all() and (got[64:270] == 0).all() and (got[3] == 0).all()


@pytest.mark.gpu
@pytest.mark.parametrize("shape", [GRID[0], GRID[1], GRID[2], GRID[4], GRID[5]], ids=lambda s: "-".join(str(x) for x in s))
@pytest.mark.parametrize("value", [float("inf"), float("-inf"), float("nan")])
def test_values_that_are_no_numbers_reach_only_the_rows_that_see_them(shape, value):
    """In V and in K, at keys that some rows of a tile see and others do not: behind a row, ahead of its window, in another
    document.  Queries are small, so that every visible weight is a number of the 16-bit type above 0."""
    base = grid_batch(*shape, prefill=((200, 333), (90, 90)), decode=(31, 257, 300))
    base = dataclasses.replace(base, prefill_q=base.prefill_q * 0.1, decode_q=base.decode_q * 0.1)
    for scores in (pod.Scores(logit_cap=30.0), pod.Scores(window=40), variant("documents", base)):
        batch = poison_unseen(base, scores, value)
        for which in ("v_cache", "k_cache"):
            cache = getattr(batch, which).clone()
            for row, t in ((0, 333 - 60), (0, 333 - 171), (1, 45), (3, 250)):
                at = (int(batch.block_table[row, t // batch.block_size]), t % batch.block_size) if batch.block_size else (row, t)
                index = (at[0], 0, at[1]) if batch.head_major else (at[0], at[1], 0)
                cache[index][3:9] = value
            case = dataclasses.replace(batch, **{which: cache})
            with np.errstate(invalid="ignore", over="ignore"):
                want, tol = reference(case, scores)
            got = wl.as_f64(run(case, scores)[0])
            if which == "k_cache" and value != value or which == "v_cache":
                assert np.array_equal(np.isfinite(got), np.isfinite(want))
            sound = np.isfinite(want) & np.isfinite(tol)
            if which == "k_cache":                              # an infinite key gives scores of either sign: only untouched rows
                first, end, _ = intervals(case, scores)
                touched = np.zeros(case.n_rows, bool)
                for r, t in ((0, 333 - 60), (0, 333 - 171), (1, 45), (3, 250)):
                    start, q_len = case.seq_meta[r, 0], case.seq_meta[r, 1]
                    rows = np.arange(q_len) + start + (case.n_prefill_rows if r >= 2 else 0)
                    touched[rows] |= (first[rows] <= t) & (t < end[rows])
                sound &= ~touched[:, None, None]
            assert np.isfinite(got[sound]).all() and (np.abs(got[sound] - want[sound]) <= tol[sound]).all()


@pytest.mark.gpu
def test_sum_of_what_a_row_sees_keeps_its_sign_of_infinity():
    """In prompts, whose tiles hold the values next to rows that do not see them: +inf, -inf, and both together NaN."""
    batch = grid_batch(8, 2, 128, wl.BF16, 16, False, prefill=((90, 90),), decode=())
    batch = dataclasses.replace(batch, prefill_q=batch.prefill_q * 0.1, v_cache=batch.v_cache.clone())
    for t, channel, value in ((20, 0, np.inf), (20, 1, -np.inf), (20, 2, np.inf), (40, 2, -np.inf)):
        batch.v_cache[int(batch.block_table[0, t // 16]), t % 16, :, channel] = value
    got = run(batch, pod.Scores(window=30))[0].float()
    for i in range(90):
        sees = [max(0, i - 29) <= t <= i for t in (20, 40)]
        want = [np.inf if sees[0] else None, -np.inf if sees[0] else None,
                np.nan if all(sees) else np.inf if sees[0] else -np.inf if sees[1] else None]
        for c, w in enumerate(want):
            x = got[i, :, c]
            assert torch.isfinite(x).all() if w is None else torch.isnan(x).all() if w != w else (x == w).all(), (i, c)


@pytest.mark.gpu
def test_random_batches_with_changed_scores():
    rng = np.random.default_rng(20)
    for i in range(24):
        hq, hkv, d = [(8, 2, 128), (4, 4, 64), (9, 3, 128), (16, 1, 64), (8, 1, 256), (32, 8, 128)][int(rng.integers(6))]
        prefill = [(int(q), int(q) + int(rng.integers(0, 600))) for q in rng.integers(1, 300, int(rng.integers(0, 4)))]
        decode = rng.integers(1, 900, int(rng.integers(0 if prefill else 1, 12))).tolist()
        batch = wl.make_batch(f"random{i}", prefill=prefill, decode_kv_lens=decode, n_q_heads=hq, n_kv_heads=hkv, head_dim=d,
                              dtype=int(rng.integers(2)), seed=700 + i, block_size=int(rng.choice([0, 16, 16, 32, 24, 5])), poison=float("nan"))
        if rng.random() < 0.3:
            batch = wl.to_head_major(batch)
        scores = pod.Scores(logit_cap=float(rng.choice([0, 2.0, 40.0])), window=int(rng.choice([0, 0, 20, 150])),
                            slopes=slopes(hq) if rng.random() < 0.4 else None,
                            doc_start=documents(batch, (1, 200), i) if rng.random() < 0.4 else None,
                            prefix_len=rng.integers(0, 300, len(batch.seq_meta)).tolist() if rng.random() < 0.4 else None)
        kw = [{}, dict(decode_chunk=64), dict(prefill_split_len=64, max_prefill_waves=64), dict(n_compute_units=8)][int(rng.integers(4))]
        check(poison_unseen(batch, scores), scores, str(rng.choice(["fused", "serial", "fused_cta"])), **kw)


@pytest.mark.gpu
@pytest.mark.parametrize("block", [0, 16])
def test_long_contexts_and_offsets_beyond_32_bits(block):
    """128K keys under a window, a cap and slopes; cache offsets that pass 2^32 bytes."""
    lens = [131072] * 6 + [131071, 100000]
    batch = wl.make_batch("long", prefill=[(40, 131072)], decode_kv_lens=lens, n_q_heads=16, n_kv_heads=16, head_dim=128, dtype=wl.BF16,
                          seed=9, block_size=block, device="cuda:0")
    assert batch.k_cache.numel() * 2 > 2 ** 32
    for scores in (pod.Scores(window=3000, slopes=slopes(16)), pod.Scores(logit_cap=10.0)):
        attn = pod.HybridAttention(batch, scores=scores)
        out = attn.forward(batch)
        torch.cuda.synchronize()
        # the reference of one head and a few rows, on the host
        first, end, at = intervals(batch, scores)
        for r, row, q in ((0, 39, batch.prefill_q[39]), (8, 47, batch.decode_q[7]), (7, 46, batch.decode_q[6])):
            cache_row, n = int(batch.seq_meta[r, 3]), int(batch.seq_meta[r, 2])
            for h in (0, 15):
                if block:
                    blocks = batch.block_table[cache_row, :-(-n // 16)].long()
                    k, v = (c[blocks, :, h].reshape(-1, 128)[:n].double().cpu().numpy() for c in (batch.k_cache, batch.v_cache))
                else:
                    k, v = (c[cache_row, :n, h].double().cpu().numpy() for c in (batch.k_cache, batch.v_cache))
                s = k @ q[h].double().cpu().numpy() * batch.softmax_scale
                if scores.logit_cap:
                    s = scores.logit_cap * np.tanh(s / scores.logit_cap)
                if scores.slopes is not None:
                    s = s - scores.slopes[h] * np.abs(np.arange(n) - at[row])
                s, v = s[first[row]:end[row]], v[first[row]:end[row]]
                w = np.exp(s - s.max())
                w /= w.sum()
                size = w @ np.abs(v)
                err = np.abs(out[row, h].double().cpu().numpy() - w @ v)
                assert (err <= 2.0 ** -8 * 1.01 * (2 * size + np.abs(w @ v)) + size * 2.0 ** -12).all()
        attn.close()


@pytest.mark.gpu
def test_capture_static_scratch_and_repeated_calls_give_the_same_bits():
    batch = grid_batch(8, 2, 128, wl.BF16, 16, False, decode=(900, 31, 64, 257, 1200))
    scores = variant("all", batch)
    dev = batch.to("cuda:0")
    attn = pod.HybridAttention(dev, scores=scores, decode_chunk=128, prefill_split_len=64, max_prefill_waves=64)
    want = attn.forward(dev).clone()
    torch.cuda.synchronize()
    other = torch.cuda.Stream()
    with torch.cuda.stream(other):
        again = attn.forward(dev)
    torch.cuda.synchronize()
    assert torch.equal(again, want)
    out = torch.zeros_like(want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        attn.forward(dev, out=out)
    for _ in range(4):
        out.fill_(3.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
        assert torch.equal(attn.forward(dev), want)
    out.fill_(3.0)
    pod.pod_attn_forward_static(dev.prefill_q.data_ptr(), dev.decode_q.data_ptr(), dev.k_cache.data_ptr(), dev.v_cache.data_ptr(),
                                attn.seq_meta_dev.data_ptr(), dev.block_table.data_ptr(), out.data_ptr(), attn.plan, pod.MODE_FUSED,
                                torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    assert torch.equal(out, want)
    attn.close()


@pytest.mark.gpu
def test_plans_on_two_streams_at_once_give_the_bits_of_each_alone():
    """A plan bound by ticket whose groups a kernel of its own merges, and one of decodes that merge themselves; each has its
    own workspace, and what one call clears must be the next one's of the same plan only."""
    runs = []
    for decode, prefill, name, kw in [((900, 31, 64, 257, 1200), ((200, 333), (37, 37)), "all", dict(decode_chunk=128, prefill_split_len=64, max_prefill_waves=64)),
                                      ((1500, 700, 1), (), "cap", {})]:
        batch = grid_batch(8, 2, 128, wl.BF16, 16, False, prefill=prefill, decode=decode)
        dev = batch.to("cuda:0")
        attn = pod.HybridAttention(dev, scores=variant(name, batch), **kw)
        runs.append((dev, attn, attn.forward(dev).clone(), torch.cuda.Stream(), []))
    torch.cuda.synchronize()
    for _ in range(20):
        for dev, attn, _, stream, got in runs:
            with torch.cuda.stream(stream):
                got.append(attn.forward(dev))
    torch.cuda.synchronize()
    for _, attn, want, _, got in runs:
        assert all(torch.equal(g, want) for g in got)
        attn.close()


@pytest.mark.gpu
@pytest.mark.parametrize("config", [1, 3])
def test_benchmark_batches_with_nothing_changed_stay_within_the_bar_of_the_plain_plan(config):
    """A plan whose scores are changed by nothing, against the plain plan of the same batch: other kernels and cuts, one result."""
    batch = wl.config_batch(config, device="cuda:0")
    plain, scored = pod.HybridAttention(batch), pod.HybridAttention(batch, scores=pod.Scores())
    a, b = plain.forward(batch).double(), scored.forward(batch).double()
    bar = {wl.F16: 2e-3, wl.BF16: 1e-2}[batch.dtype]                   # of either from the exact result
    assert float((a - b).abs().max()) <= 2 * bar
    plain.close()
    scored.close()


@pytest.mark.gpu
def test_a_layer_with_a_window_from_its_projections():
    """Append and windowed attention together: a decode step whose oldest blocks have been given back."""
    batch = wl.make_batch("step", prefill=[(40, 140)], decode_kv_lens=[300, 49, 16], n_q_heads=4, n_kv_heads=2, head_dim=64, dtype=wl.F16,
                          seed=31, block_size=16)
    scores = pod.Scores(window=64, logit_cap=8.0)
    dev = poison_unseen(batch, scores).to("cuda:0")
    attn = pod.HybridAttention(dev, scores=scores)
    n = batch.n_rows
    tables = pod.TokenTables(attn.params, n)
    lacks = [(r, i) for r, (_, q, kv, _) in enumerate(batch.seq_meta.tolist()) for i in range(-(-(kv - q) // 16), -(-kv // 16))]
    free = torch.tensor([int(dev.block_table[r, i]) for r, i in lacks], dtype=torch.int32, device="cuda:0")
    tables.build(attn.seq_meta_dev, free, dev.block_table)
    append = pod.TokenAppend(attn.params, rope=pod.Rope(32, layout="interleaved"), norm=pod.HeadNorm())
    qkv = torch.randn(n, 8 * 64, generator=torch.Generator().manual_seed(1)).half().cuda()
    args = qkv[:, :256], qkv[:, 256:384], qkv[:, 384:]
    out = attn.forward_tokens(dev, append, tables, *args)
    rows = append(*args, tables.slots, tables.positions, dev.k_cache, dev.v_cache)
    seen = dataclasses.replace(dev, prefill_q=rows[:40], decode_q=rows[40:]).to("cpu")
    want, tol = reference(seen, scores)
    assert (np.abs(wl.as_f64(out) - want) <= tol).all()
    attn.close()


def test_masks_that_are_no_32_bit_integers_are_refused():
    """An array of 64-bit integers or of floats would be wrapped or cut off on its way to the plan, and mask something else."""
    b = wl.config_batch(1)
    plan = lambda **kw: pod.pod_attn_plan_create_scored(plain_params(b), pod.Scores(**kw), b.seq_meta)
    n_req = len(b.seq_meta)
    for name, size in (("doc_start", b.n_rows), ("prefix_len", n_req)):
        for bad in (2.0 ** 32, 2 ** 32 + 5, -2 ** 32, 0.5, float("nan"), float("inf"), 2 ** 31):
            values = np.zeros(size, np.int64 if isinstance(bad, int) else np.float64)
            values[-1] = bad
            with np.errstate(invalid="ignore"), pytest.raises((ValueError, OverflowError)):
                plan(**{name: values})
        for good in (np.full(size, 3, np.int64), np.full(size, 3.0), [3] * size, torch.full((size,), 3)):
            plan(**{name: good}).close()


@pytest.mark.gpu
@pytest.mark.parametrize("cap", [2000.0, 6e4, 7e5, 3e6])
def test_scores_well_below_a_cap_of_thousands_keep_their_digits(cap):
    """Dot products and their scale are exact here (whole numbers below 2^24 and a power of two), so that what is left of the
    tolerance is the cap's: 2^-20.7 of a score, doubled for the difference of two, and the softmax weights' and the result's
    halves of a step.  Each row sees two keys with values 1 and -1 whose scores are 2 to 4 in a hundred of the cap and at most 1 apart."""
    rng = np.random.default_rng(int(cap))
    n, d = 256, 128
    batch = wl.make_batch("pairs", prefill=[(n, n)], decode_kv_lens=[2] * 64, n_q_heads=2, n_kv_heads=2, head_dim=d, dtype=wl.F16, seed=3,
                          block_size=16, softmax_scale=1.0)
    scale = 2.0 ** -4
    batch = dataclasses.replace(batch, softmax_scale=scale, k_cache=torch.zeros_like(batch.k_cache), v_cache=torch.ones_like(batch.v_cache),
                                prefill_q=torch.zeros_like(batch.prefill_q), decode_q=torch.zeros_like(batch.decode_q))
    # keys: 1 in the first eight channels; the ninth is 1 for every second key, whose values are -1
    batch.k_cache[..., :8] = 1.0
    batch.k_cache[:, 1::2, :, 8] = 1.0
    batch.v_cache[:, 1::2] = -1.0
    q = np.zeros((n + 64, 2, d))
    q[..., :8] = rng.integers(int(0.02 * cap / scale / 8), int(0.04 * cap / scale / 8), (n + 64, 2, 1)).clip(1, 60000)
    q[..., 8] = rng.integers(-16, 17, (n + 64, 2))
    q = torch.from_numpy(q).half()
    batch.prefill_q.copy_(q[:n])
    batch.decode_q.copy_(q[n:])
    got = wl.as_f64(run(batch, pod.Scores(logit_cap=cap, window=2))[0])
    q = wl.as_f64(q)
    base, step = q[..., :8].sum(-1) * scale, q[..., 8] * scale
    assert (base <= 2 ** 24 * scale).all()
    even, odd = cap * np.tanh(base / cap), cap * np.tanh((base + step) / cap)
    w = 1 / (1 + np.exp(odd - even))                                     # of the key whose value is 1
    want = 2 * w - 1
    want[0] = 1.0                                                        # the prompt's first row sees one key
    delta = 2 * 2.0 ** -20.7 * np.abs(even) + 2.0 ** -23 * np.abs(even)
    tol = 2.0 ** -11 * 1.01 * (2 + np.abs(want)) + 2 * w * (1 - w) * delta + 2.0 ** -18
    err = np.abs(got - want[..., None]).max(-1)
    print("cap", cap, "of the tolerance", float((err / tol).max()), "error", float(err.max()), flush=True)
    assert (err <= tol).all()


@pytest.mark.gpu
@pytest.mark.parametrize("block", [16, 0])
@pytest.mark.parametrize("name", ["cap", "cap and slopes", "slopes"])
def test_plans_of_heavy_prompts_launch_a_workgroup_per_item(name, block):
    """512 items and more, as long as the decode stream: the launch that POD_MODE_FUSED takes by itself there, which kernel it
    is, rows of it against the definition, and the bits of the other launches (persistent ones with a trace or an event log)."""
    from torch.profiler import ProfilerActivity, profile
    n_kv, heads, kv_heads, d = 16384, 32, 4, 128
    batch = wl.make_batch("heavy", prefill=[(2048, n_kv)], decode_kv_lens=[n_kv - 5 * i for i in range(16)], n_q_heads=heads, n_kv_heads=kv_heads,
                          head_dim=d, dtype=wl.BF16, seed=51, block_size=block, device="cuda:0")
    scores = pod.Scores(logit_cap=20.0 if "cap" in name else 0.0, slopes=slopes(heads) if "slopes" in name else None)
    attn = pod.HybridAttention(batch, scores=scores)
    assert attn.info.n_prefill_items >= 2 * attn.info.n_compute_units and attn.info.fused_grid <= 2 * attn.info.n_compute_units
    torch.cuda.synchronize()

    def kernels(call):
        with profile(activities=[ProfilerActivity.CUDA]) as prof:
            result = call()
            torch.cuda.synchronize()
        return {k for e in prof.key_averages() for k in ("fused_cta_scored", "fused_scored", "prefill_scored", "decode_scored") if "pod::" + k in e.key}, result

    taken, out = kernels(lambda: attn.forward(batch))
    assert taken == {"fused_cta_scored"}
    for mode in ("serial", "streams", "fused_cta", "fused"):
        assert torch.equal(attn.forward(batch, mode=pod.MODES[mode]), out), mode
    for on, off in ((attn.enable_trace, attn.disable_trace), (attn.enable_event_log, attn.disable_event_log)):
        on()
        taken, again = kernels(lambda: attn.forward(batch))
        off()
        assert taken == {"fused_scored"} and torch.equal(again, out)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        again = attn.forward(batch)
    side.synchronize()
    assert torch.equal(again, out)
    for r, row, q in ((0, 0, batch.prefill_q[0]), (0, 777, batch.prefill_q[777]), (0, 2047, batch.prefill_q[2047]), (1, 2048, batch.decode_q[0]),
                      (16, 2063, batch.decode_q[15])):
        n = n_kv - 2048 + row + 1 if r == 0 else int(batch.seq_meta[r, 2])
        cache_row = int(batch.seq_meta[r, 3])
        for h in (0, 9, 31):
            kvh = h * kv_heads // heads
            if block:
                blocks = batch.block_table[cache_row, :-(-n // block)].long()
                k, v = (c[blocks, :, kvh].reshape(-1, d)[:n].double().cpu().numpy() for c in (batch.k_cache, batch.v_cache))
            else:
                k, v = (c[cache_row, :n, kvh].double().cpu().numpy() for c in (batch.k_cache, batch.v_cache))
            s = k @ q[h].double().cpu().numpy() * batch.softmax_scale
            if scores.logit_cap:
                s = scores.logit_cap * np.tanh(s / scores.logit_cap)
            if scores.slopes is not None:
                s = s - scores.slopes[h] * np.arange(n - 1, -1, -1)
            w = np.exp(s - s.max())
            w /= w.sum()
            size = w @ np.abs(v)
            err = np.abs(out[row, h].double().cpu().numpy() - w @ v)
            # half a step of the weights in the sum and in what it is divided by and of the result; scores in 32 bits
            assert (err <= 2.0 ** -8 * 1.01 * (2 * size + np.abs(w @ v)) + size * 2.0 ** -12).all(), (row, h)
    attn.close()


def test_slopes_beside_a_scale_that_has_no_reciprocal_are_refused():
    """1 / softmax_scale is infinite for a subnormal scale, and times a slope of 0 no number."""
    b = wl.config_batch(1)
    for scale, refused in ((1e-40, True), (1e-38, True), (9e-31, True), (2e-30, False), (1.0, False)):
        params = plain_params(b, softmax_scale=scale)
        pod.pod_attn_plan_create_scored(params, pod.Scores(window=5), b.seq_meta).close()
        if refused:
            with pytest.raises(pod.PodError, match="too small for slopes") as e:
                pod.pod_attn_plan_create_scored(params, pod.Scores(slopes=[0.0] * b.n_q_heads), b.seq_meta)
            assert e.value.status == -1
        else:
            pod.pod_attn_plan_create_scored(params, pod.Scores(slopes=[0.0] * b.n_q_heads), b.seq_meta).close()
