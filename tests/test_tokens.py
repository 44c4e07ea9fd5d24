"""A batch's new tokens: slots and blocks from the request lengths, and their projections normalised, rotated and written.

References are numpy in 64 bits.  An appended value may differ from the reference by the rounding to its type (half a step)
and by what 32-bit arithmetic loses: cosines and sines are within 2^-22 of a unit (sine unit, angle kept to 2^-25 of a turn),
products, sums of up to 256 squares and the reciprocal root within 2^-20 of their terms, together below 2^-19 times the sum
of a pair's magnitudes.
"""
import ctypes
import math

import numpy as np
import pytest
import torch

from paper_2410_18038_amd import pod
from paper_2410_18038_amd import workloads as wl
from tests.helpers import oracle_out

TDT = {wl.F16: torch.float16, wl.BF16: torch.bfloat16}


def make_params(*, hq=8, hkv=2, d=128, dtype=wl.BF16, block=16, n_blocks=64, rows=8, max_blocks=8, head_major=False, max_len=64,
                n_prefill=0, n_decode=0):
    return pod.make_params(n_prefill=n_prefill, n_decode=n_decode, n_q_heads=hq, n_kv_heads=hkv, head_dim=d, dtype=dtype,
                           softmax_scale=1.0, block_size=block, max_blocks_per_seq=max_blocks if block else 0,
                           n_cache_rows=rows, n_blocks=n_blocks if block else 0, kv_seq_stride=0 if block else max_len * hkv * d,
                           kv_order=pod.KV_HEAD_MAJOR if head_major else pod.KV_TOKEN_MAJOR, n_compute_units=256)


# -- frequencies (host) ------------------------------------------------------------------------- #
def frequencies(rot, theta, scaling, factor, trained, low, high):
    out = []
    for i in range(rot // 2):
        f = theta ** (-2.0 * i / rot)
        keep = 1.0
        if scaling == "linear":
            keep = 0.0
        elif scaling == "parts":
            keep = (trained * f / (2 * math.pi) - low) / (high - low)
        elif scaling == "index":
            at = [rot * math.log(trained / (2 * math.pi * t)) / (2 * math.log(theta)) for t in (high, low)]
            a, b = (min(max(x, 0), rot - 1) for x in (math.floor(at[0]), math.ceil(at[1])))
            keep = 1 - (i - a) / max(b - a, 0.001)
        keep = min(max(keep, 0.0), 1.0)
        out.append(keep * f + (1 - keep) * f / factor)
    return np.array(out)


@pytest.mark.parametrize("scaling", ["none", "linear", "parts", "index"])
@pytest.mark.parametrize("rot,theta,factor,trained", [(16, 1e4, 4.0, 2048), (128, 5e5, 8.0, 8192), (256, 1e6, 32.0, 4096), (64, 1.5, 0.5, 64)])
def test_rope_table_holds_the_frequencies(scaling, rot, theta, factor, trained):
    if scaling == "none":
        factor = 1.0
    rope = pod.Rope(rot, theta=theta, scaling=scaling, factor=factor, trained_len=trained, low=1.0, high=4.0)
    turns = frequencies(rot, theta, scaling, factor, trained, 1.0, 4.0) / (2 * math.pi)
    assert rope.table.shape == (rot // 2,)
    # a few roundings of 64-bit arithmetic
    assert np.abs(rope.table.astype(np.float64) / 2.0 ** 64 - turns % 1.0).max() <= 2.0 ** -48 * max(1.0, turns.max())


def test_rope_parameters_are_checked():
    good = dict(layout=0, scaling=0, rot_dim=64, cos_sin_scale=1.0, theta=1e4, factor=1.0, trained_len=1.0, low=1.0, high=2.0)
    order = [n for n, _ in pod.RopeParams._fields_]

    def table(**kw):
        return pod.pod_attn_rope_table(pod.RopeParams(*[{**good, **kw}[n] for n in order]))

    table()
    for status, kw in [(-1, dict(layout=2)), (-1, dict(scaling=4)), (-1, dict(rot_dim=0)), (-1, dict(rot_dim=272)),
                       (-2, dict(rot_dim=40)), (-1, dict(theta=1.0)), (-1, dict(theta=math.nan)), (-1, dict(cos_sin_scale=math.inf)),
                       (-1, dict(scaling=1, factor=0.0)), (-1, dict(scaling=2, high=1.0)), (-1, dict(scaling=3, low=0.0)),
                       (-1, dict(scaling=3, trained_len=math.nan))]:
        with pytest.raises(pod.PodError) as e:
            table(**kw)
        assert e.value.status == status, kw
    assert pod.lib().pod_attn_rope_table(None, None) == -1
    with pytest.raises(ValueError):
        pod.Rope(64, layout="pairs")
    with pytest.raises(ValueError):
        pod.Rope(64, scaling="more")


# -- refusals (host; nothing is launched) -------------------------------------------------------- #
def test_table_arguments_are_checked_before_anything_is_launched():
    prm = make_params(n_prefill=1, n_decode=2)
    good = dict(params=prm, seq_meta=16, free_blocks=16, n_free=4, block_table=16, n_rows=10, slots=16, positions=16, report=16)

    def refuse(status, **kw):
        with pytest.raises(pod.PodError) as e:
            pod.pod_attn_build_tables(**{**good, **kw})
        assert e.value.status == status and len(str(e.value)) > 20, kw

    refuse(-1, n_rows=1)
    refuse(-1, n_rows=-1)
    refuse(-1, n_free=-1)
    for name in ("seq_meta", "block_table", "slots", "positions", "report", "free_blocks"):
        refuse(-1, **{name: 0})
        refuse(-1, **{name: 18})
    refuse(-1, params=make_params(n_prefill=-1))
    refuse(-1, params=make_params(block=0, n_decode=2))                            # free blocks for a contiguous cache
    refuse(-2, params=make_params(n_decode=2, block=1 << 20, n_blocks=1 << 12))    # 2^32 slots
    refuse(-1, params=make_params(n_decode=2, block=0, max_len=64, hkv=0), n_free=0)


def test_append_arguments_are_checked_before_anything_is_launched():
    prm = make_params()
    rope = pod.Rope(128).params
    good = dict(params=prm, rope=rope, rope_table=16, norm=None, q=16, q_stride=1024, k=16, k_stride=256, v=16, v_stride=256,
                slots=16, positions=16, n_rows=4, q_out=32, k_cache=16, v_cache=16)

    def refuse(status, **kw):
        with pytest.raises(pod.PodError) as e:
            pod.pod_attn_append(**{**good, **kw})
        assert e.value.status == status and len(str(e.value)) > 15, kw

    for name in ("q", "k", "v", "q_out", "k_cache", "v_cache"):
        refuse(-1, **{name: 0})
        refuse(-1, **{name: 24})
    for name in ("slots", "positions"):
        refuse(-1, **{name: 0})
        refuse(-1, **{name: 18})
    refuse(-1, rope_table=0)
    refuse(-1, rope_table=8)
    refuse(-1, n_rows=-1)
    refuse(-1, q_stride=1016)
    refuse(-1, k_stride=248)
    refuse(-1, v_stride=260)
    refuse(-1, q_out=16, q_stride=1032)                                  # in place, but rows apart
    refuse(-1, rope=pod.Rope(256).params)                                # more than head_dim
    refuse(-1, norm=pod.HeadNormParams(None, None, -1.0, 0.0, 1, 1))
    refuse(-1, norm=pod.HeadNormParams(None, None, math.nan, 0.0, 1, 0))
    refuse(-1, norm=pod.HeadNormParams(8, None, 1e-6, 0.0, 1, 1))
    refuse(-2, params=make_params(d=96))
    refuse(-2, params=make_params(block=1 << 20, n_blocks=1 << 12))
    pod.pod_attn_append(**{**good, "n_rows": 0})                         # nothing to do
    assert pod.lib().pod_attn_append(None, None, 0, None, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0) == -1


def test_struct_layouts_of_the_token_calls_match_the_header(tmp_path):
    import os
    import subprocess
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    src = tmp_path / "sizes.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "pod_attn.h"\nint main(void){printf("%zu %zu %zu %zu\\n",'
                   ' sizeof(pod_rope_params), offsetof(pod_rope_params, theta), sizeof(pod_head_norm),'
                   ' offsetof(pod_head_norm, normalise_k)); return 0;}\n')
    exe = tmp_path / "sizes"
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.join(root, "include"), str(src), "-o", str(exe)], check=True)
    got = [int(x) for x in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()]
    assert got == [ctypes.sizeof(pod.RopeParams), pod.RopeParams.theta.offset, ctypes.sizeof(pod.HeadNormParams),
                   pod.HeadNormParams.normalise_k.offset]


# -- append --------------------------------------------------------------------------------------- #
def append_reference(q, k, v, slots, positions, k_cache, v_cache, q_out, *, d, layout, f, scale, norm, head_major, per_block):
    """float64 (q_out, k_cache, v_cache, tolerance of q_out, of k_cache before rounding)."""
    q_out, k_cache, v_cache = (wl.as_f64(t) for t in (q_out, k_cache, v_cache))
    q_tol, k_tol = np.zeros_like(q_out), np.zeros_like(k_cache)
    half = len(f)
    for i, (slot, pos) in enumerate(zip(slots, positions)):
        if slot < 0 or slot >= k_cache.shape[0] * per_block:
            continue
        at = (slot // per_block, slice(None), slot % per_block) if head_major else (slot // per_block, slot % per_block)
        for what, x in (("q", wl.as_f64(q[i]).reshape(-1, d)), ("k", wl.as_f64(k[i]).reshape(-1, d))):
            if norm is not None and norm[what][0]:
                w = norm[what][1]
                weight = 1.0 if w is None else wl.as_f64(w) + norm["offset"]
                x = x / np.sqrt((x * x).mean(-1, keepdims=True) + norm["eps"]) * weight
            y, size = x.copy(), np.abs(x)
            angle = (int(pos) * f) if half else np.zeros(0)
            for j in range(half):
                a, b = (j, j + half) if layout == "half" else (2 * j, 2 * j + 1)
                c, s = math.cos(angle[j]) * scale, math.sin(angle[j]) * scale
                y[:, a], y[:, b] = x[:, a] * c - x[:, b] * s, x[:, b] * c + x[:, a] * s
                size[:, a] = size[:, b] = (np.abs(x[:, a]) + np.abs(x[:, b])) * abs(scale)
            if what == "q":
                q_out[i], q_tol[i] = y, size * 2.0 ** -19
            else:
                k_cache[at], k_tol[at] = y, size * 2.0 ** -19
        v_cache[at] = wl.as_f64(v[i]).reshape(-1, d)
    return q_out, k_cache, v_cache, q_tol, k_tol


def close(got, want, tol, dtype):
    """Within half a step of the type and the tolerance given."""
    step = torch.finfo(TDT[dtype]).eps / 2
    tiny = 2.0 ** -25 if dtype == wl.F16 else 0.0                        # half a step of the smallest fp16 numbers
    err = np.abs(wl.as_f64(got) - want)
    assert (err <= np.abs(want) * step * (1 + 2.0 ** -7) + tol * (1 + step) + tiny).all(), float(err.max())


APPENDS = [   # heads, channels, type, block, head-major, rows, layout, rotated, norm, offset, scaling, in one projection
    ((8, 2), 128, wl.BF16, 16, False, 37, "half", 128, "both", 0.0, "none", True),
    ((8, 2), 128, wl.F16, 16, True, 1, "half", 64, None, 0.0, "linear", True),
    ((9, 3), 64, wl.F16, 24, False, 130, "interleaved", 32, "both", 1.0, "parts", True),
    ((4, 4), 64, wl.BF16, 0, False, 65, "half", 16, "q", 0.0, "index", False),
    ((8, 2), 256, wl.BF16, 16, False, 21, "interleaved", 256, "k", 1.0, "parts", False),
    ((5, 5), 256, wl.F16, 1, False, 19, "half", 64, "plain", 0.0, "none", True),
    ((15, 5), 128, wl.BF16, 0, True, 50, "interleaved", 16, None, 0.0, "none", False),
    ((1, 1), 64, wl.BF16, 64, False, 300, "half", 64, "both", 0.0, "index", True),
    ((16, 1), 64, wl.F16, 8, True, 3, None, 0, "both", 0.0, "none", True),
    ((32, 32), 128, wl.F16, 16, False, 9, None, 0, None, 0.0, "none", True),
]


def make_append(heads, d, dtype, block, head_major, rows, layout, rot, norm, offset, scaling, packed, *, seed, pad=0, far=False):
    hq, hkv = heads
    rng = np.random.default_rng(seed)
    per = block or 40
    n_blocks = rows // per + 5
    prm = make_params(hq=hq, hkv=hkv, d=d, dtype=dtype, block=block, n_blocks=n_blocks, rows=n_blocks, head_major=head_major, max_len=per)
    tdt, n = TDT[dtype], rows + pad
    gen = torch.Generator().manual_seed(seed)
    randn = lambda *shape: torch.randn(*shape, generator=gen).to(tdt)
    if packed:
        qkv = randn(n, (hq + 2 * hkv) * d + 8)
        q, k, v = qkv[:, :hq * d], qkv[:, hq * d:(hq + hkv) * d], qkv[:, (hq + hkv) * d:(hq + 2 * hkv) * d]
    else:
        q, k, v = randn(n, hq * d), randn(n, hkv * d), randn(n, hkv * d)
    slots = rng.permutation(n_blocks * per)[:rows].astype(np.int32)
    positions = rng.integers(0, 1 << (31 if far else 17), rows).astype(np.int32)
    slots = np.concatenate([slots, np.full(pad, -1, np.int32)])
    positions = np.concatenate([positions, np.zeros(pad, np.int32)])
    shape = (n_blocks, hkv, per, d) if head_major else (n_blocks, per, hkv, d)
    k_cache, v_cache = torch.full(shape, float("nan"), dtype=tdt), torch.full(shape, float("nan"), dtype=tdt)
    q_out = torch.full((n, hq, d), float("nan"), dtype=tdt)
    weight = lambda: (torch.rand(d, generator=gen) + 0.5 - offset).to(tdt)
    hn, want_norm = None, None
    if norm is not None:
        use = {"q": norm in ("q", "both", "plain"), "k": norm in ("k", "both", "plain")}
        w = {x: None if norm == "plain" else weight() for x in "qk"}
        want_norm = {"q": (use["q"], w["q"]), "k": (use["k"], w["k"]), "offset": offset, "eps": 1e-5}
        hn = dict(q_weight=w["q"], k_weight=w["k"], eps=1e-5, weight_offset=offset, q=use["q"], k=use["k"])
    factor, scale = (1.0 if scaling == "none" else 8.0), (1.2 if scaling == "index" else 1.0)
    rope, f = None, np.zeros(0)
    if rot:
        rope = pod.Rope(rot, layout=layout, theta=5e5, scaling=scaling, factor=factor, trained_len=4096, low=1.0, high=4.0, cos_sin_scale=scale)
        f = frequencies(rot, 5e5, scaling, factor, 4096, 1.0, 4.0)
    want = append_reference(q, k, v, slots, positions, k_cache, v_cache, q_out, d=d, layout=layout, f=f,
                            scale=float(np.float32(scale)), norm=want_norm, head_major=head_major, per_block=per)
    cuda = lambda t: t.cuda()
    if packed:
        dev = qkv.cuda()
        qd, kd, vd = dev[:, :hq * d], dev[:, hq * d:(hq + hkv) * d], dev[:, (hq + hkv) * d:(hq + 2 * hkv) * d]
    else:
        qd, kd, vd = (t.cuda() for t in (q, k, v))
    if hn is not None:
        hn = pod.HeadNorm(**{x: (cuda(y) if torch.is_tensor(y) else y) for x, y in hn.items()})
    app = pod.TokenAppend(prm, rope=rope, norm=hn)
    return app, (qd, kd, vd, torch.from_numpy(slots).cuda(), torch.from_numpy(positions).cuda(), k_cache.cuda(), v_cache.cuda()), q_out.cuda(), want


def check_append(got, want, dtype):
    (q_out, k_cache, v_cache), (wq, wk, wv, q_tol, k_tol) = got, want
    for name, g, w, tol in (("q", q_out, wq, q_tol), ("k", k_cache, wk, k_tol), ("v", v_cache, wv, np.zeros_like(wv))):
        assert np.array_equal(np.isnan(wl.as_f64(g)), np.isnan(w)), name            # what is no token's is left as it was
        seen = ~np.isnan(w)
        close(g.cpu()[torch.from_numpy(seen)], w[seen], tol[seen], dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("case", APPENDS, ids=lambda c: "-".join(str(x) for x in c[:3]))
def test_append_matches_the_definition(case):
    app, args, q_out, want = make_append(*case, seed=5, pad=7)
    print("case", case, flush=True)
    app(*args, q_out=q_out)
    check_append((q_out, args[5], args[6]), want, case[2])


@pytest.mark.gpu
@pytest.mark.parametrize("case", [APPENDS[0], APPENDS[2]], ids=["half", "interleaved"])
def test_append_at_positions_up_to_two_to_the_31(case):
    """The reference's angle is a 64-bit product, off by 2^31 * 2^-53 turns and less: far below the tolerance."""
    app, args, q_out, want = make_append(*case, seed=6, far=True)
    app(*args, q_out=q_out)
    check_append((q_out, args[5], args[6]), want, case[2])


@pytest.mark.gpu
def test_append_in_place_skips_rows_whose_slot_is_no_slot():
    case = ((4, 4), 64, wl.F16, 16, False, 11, "half", 64, "both", 0.0, "none", False)
    app, args, q_out, want = make_append(*case, seed=8)
    q = args[0]
    before = q.clone()
    slots = args[3].clone()
    slots[3], slots[7] = -5, args[5].shape[0] * 16                       # before and behind the cache
    app(q, args[1], args[2], slots, args[4], args[5], args[6], q_out=q.view(11, 4, 64))
    wq = want[0]
    kept = [i for i in range(11) if i not in (3, 7)]
    close(q.view(11, 4, 64)[kept], wq[kept], want[3][kept], wl.F16)
    assert torch.equal(q[[3, 7]], before[[3, 7]])
    k = args[5].view(-1, 4, 64)
    assert torch.isnan(k[args[3][[3, 7]].long()]).all()                  # their own places were not written


@pytest.mark.gpu
def test_unrotated_channels_of_unnormalised_heads_are_copied_bit_by_bit():
    case = ((4, 2), 128, wl.BF16, 16, False, 33, "half", 32, None, 0.0, "none", True)
    app, args, q_out, _ = make_append(*case, seed=9)
    args[0][:, 32:128] = float("inf")
    args[0][5, 40] = float("nan")
    args[2][3] = float("-inf")
    app(*args, q_out=q_out)
    rows = args[0].reshape(33, 4, 128)
    assert torch.equal(q_out[..., 32:].view(torch.int16), rows[..., 32:].contiguous().view(torch.int16))
    assert torch.isfinite(q_out[:, 0, :32].float()).all()
    assert torch.equal(args[6].view(-1, 256)[args[3].long()].view(torch.int16), args[2].contiguous().view(torch.int16))


# -- tables --------------------------------------------------------------------------------------- #
def tables_reference(meta, n_prefill, n_decode, block, n_free, free, table, n_rows, per_row, n_cache_rows, n_blocks):
    table = table.copy() if table is not None else None
    slots, positions = np.full(n_rows, -1, np.int64), np.zeros(n_rows, np.int64)
    prows = sum(max(int(m[1]), 0) for m in meta[:n_prefill])
    ok = []
    for r, (start, q, kv, row) in enumerate(meta.tolist()):
        fits = q >= 1 and kv >= q and start >= 0 and 0 <= row < n_cache_rows and kv <= per_row
        ok.append(fits and (start + q <= n_rows if r < n_prefill else q == 1 and start < n_decode))
    blocks = lambda n: -(-n // block)
    need = [blocks(m[2]) - blocks(m[2] - m[1]) if good and block else 0 for good, m in zip(ok, meta.tolist())]
    enough, taken = sum(need) <= n_free, 0
    for r, (start, q, kv, row) in enumerate(meta.tolist()):
        for i in range(q):
            at = start + i + (prows if r >= n_prefill else 0)
            if not 0 <= at < n_rows or start < 0 or (r >= n_prefill and start >= n_decode):
                continue
            if not ok[r]:
                slots[at], positions[at] = -1, 0
                continue
            pos = kv - q + i
            positions[at] = pos
            if not block:
                slots[at] = row * per_row + pos
            elif enough:
                if pos % block == 0:
                    table[row, pos // block] = free[taken]
                    taken += 1
                b = table[row, pos // block]
                slots[at] = b * block + pos % block if 0 <= b < n_blocks else -1
    report = [taken, 0 if enough else sum(need) - n_free, len(ok) - sum(ok), prows + n_decode]
    return slots, positions, report, table


def make_tables(prefill, decode, block, *, seed, spare=3, pad=0, missing=0):
    """(meta, table with the blocks of the cached tokens entered, free list, blocks in all)."""
    rng = np.random.default_rng(seed)
    meta, at = [], 0
    for r, (q, kv) in enumerate(prefill):
        meta.append((at, q, kv, r))
        at += q
    order = rng.permutation(len(decode))
    meta += [(int(order[i]), 1, kv, len(prefill) + i) for i, kv in enumerate(decode)]
    meta = np.array(meta, np.int32).reshape(-1, 4)
    n_rows = at + len(decode) + pad
    if not block:
        return meta, None, None, 0, n_rows
    blocks = lambda n: -(-n // block)
    held, need = blocks(meta[:, 2] - meta[:, 1]), blocks(meta[:, 2])
    n_blocks = int(need.sum()) + spare
    perm = rng.permutation(n_blocks).astype(np.int32)
    table = np.full((len(meta), int(need.max()) + 1), -1, np.int32)
    used = 0
    for r in range(len(meta)):
        table[r, :held[r]] = perm[used:used + held[r]]
        used += held[r]
    free = perm[used:]
    if missing:
        free = free[:int((need - held).sum()) - missing]
    return meta, table, free, n_blocks, n_rows


def run_tables(meta, n_prefill, n_decode, block, table, free, n_blocks, n_rows, per_row=64):
    n_cache_rows = len(meta)
    prm = make_params(n_prefill=n_prefill, n_decode=n_decode, block=block, n_blocks=n_blocks, rows=max(n_cache_rows, 1),
                      max_blocks=table.shape[1] if block else 0, max_len=per_row)
    cuda = lambda a: None if a is None else torch.from_numpy(a).cuda()
    tables = pod.TokenTables(prm, n_rows)
    dev_table = cuda(table)
    tables.build(cuda(meta), cuda(free), dev_table)
    want = tables_reference(meta, n_prefill, n_decode, block, 0 if free is None else len(free), free, table, n_rows,
                            table.shape[1] * block if block else per_row, max(n_cache_rows, 1), n_blocks)
    assert tables.report.tolist() == want[2]
    assert tables.slots.tolist() == want[0].tolist()
    assert tables.positions.tolist() == want[1].tolist()
    if block:
        assert dev_table.tolist() == want[3].tolist()
    return tables


@pytest.mark.gpu
@pytest.mark.parametrize("block", [1, 16, 24, 64])
@pytest.mark.parametrize("prefill,decode,pad", [
    ([], [1], 0), ([(1, 1)], [], 3), ([(700, 700)], [1, 16, 17, 33], 5), ([(5, 900), (1, 17), (300, 301)], [48] * 5, 0),
    ([(16, 32), (17, 17), (15, 16)], list(range(1, 700)), 300), ([(3000, 5000)] + [(1, n) for n in range(1, 70)], [7], 1)])
def test_tables_follow_the_request_lengths(block, prefill, decode, pad):
    meta, table, free, n_blocks, n_rows = make_tables(prefill, decode, block, seed=11, pad=pad)
    run_tables(meta, len(prefill), len(decode), block, table, free, n_blocks, n_rows)


@pytest.mark.gpu
def test_tables_of_a_contiguous_cache_and_of_an_empty_batch():
    meta, _, _, _, n_rows = make_tables([(33, 64), (7, 9)], [64, 1, 20], 0, seed=12, pad=4)
    run_tables(meta, 2, 3, 0, None, None, 0, n_rows, per_row=64)
    run_tables(np.zeros((0, 4), np.int32), 0, 0, 16, np.full((1, 3), -1, np.int32), np.arange(4, dtype=np.int32), 4, 700)


@pytest.mark.gpu
@pytest.mark.parametrize("missing", [1, 40])
def test_nothing_is_taken_where_the_free_list_is_too_short(missing):
    meta, table, free, n_blocks, n_rows = make_tables([(700, 900), (40, 41)], [16, 17, 1, 33], 16, seed=13, pad=2, missing=missing)
    t = run_tables(meta, 2, 4, 16, table, free, n_blocks, n_rows)
    assert t.report.tolist()[:2] == [0, missing] and (t.slots == -1).all()


@pytest.mark.gpu
def test_requests_that_cannot_be_are_refused_and_the_others_served():
    """One fault each; the reference says what every row gets."""
    faults = [(0, 1, 0), (0, 1, -3), (0, 2, 5), (1, 3, 99), (1, 3, -1), (1, 2, 1 << 30), (3, 1, 2), (3, 0, 9), (4, 0, -1), (0, 0, -7),
              (0, 1, 1 << 30), (2, 2, -(1 << 31))]
    for request, column, value in faults:
        meta, table, free, n_blocks, n_rows = make_tables([(40, 50), (20, 20), (33, 90)], [17, 1, 32], 16, seed=14, pad=3)
        print("fault", request, column, value, flush=True)
        meta[request, column] = value
        tables = run_refused(meta, 3, 3, 16, table, free, n_blocks, n_rows, len(meta))
        assert tables.report.tolist()[2] == 1


@pytest.mark.gpu
@pytest.mark.parametrize("column,value", [(0, 5000), (1, 0), (1, -40)])
def test_rows_behind_a_gap_are_no_padding(column, value):
    """The second request begins behind as many rows as the batch has: they are its rows, and those around them padding."""
    meta, table, free, n_blocks, n_rows = make_tables([(3000, 3000), (2500, 2600)], [17], 16, seed=16, pad=6000)
    meta[1 if column == 0 else 0, column] = value
    for _ in range(5):
        tables = run_refused(meta, 2, 1, 16, table, free, n_blocks, n_rows, len(meta))
        placed, last = (5500, 7500) if column == 0 else (2501, 5500)      # (with a gap the decode row is one of the second request's)
        assert int((tables.slots >= 0).sum()) == placed and bool((tables.slots[last:] == -1).all())


def run_refused(meta, n_prefill, n_decode, block, table, free, n_blocks, n_rows, n_cache_rows):
    """Like run_tables, but only the rows that exactly one request names are compared."""
    prm = make_params(n_prefill=n_prefill, n_decode=n_decode, block=block, n_blocks=n_blocks, rows=n_cache_rows, max_blocks=table.shape[1])
    tables = pod.TokenTables(prm, n_rows)
    tables.slots.fill_(-9)
    dev_table = torch.from_numpy(table).cuda()
    tables.build(torch.from_numpy(meta).cuda(), torch.from_numpy(free).cuda(), dev_table)
    small = meta.copy()
    small[:, 1] = np.minimum(small[:, 1], 1 << 12)                       # (the reference walks over every row)
    want = tables_reference(small, n_prefill, n_decode, block, len(free), free, table, n_rows, table.shape[1] * block, n_cache_rows, n_blocks)
    assert dev_table.tolist() == want[3].tolist()
    named = np.zeros(n_rows, int)
    prows = sum(max(int(m[1]), 0) for m in meta[:n_prefill].tolist())
    for r, (start, q, kv, row) in enumerate(meta.tolist()):
        if start < 0 or (r >= n_prefill and start >= n_decode):
            continue
        at = start + (prows if r >= n_prefill else 0)
        if at < n_rows:
            named[at:min(n_rows, at + max(q, 0) if r < n_prefill else at + 1)] += 1
    once = named == 1
    assert tables.slots.cpu().numpy()[once].tolist() == want[0][once].tolist()
    return tables


@pytest.mark.gpu
def test_a_table_entry_that_names_no_block_gives_no_slot():
    meta, table, free, n_blocks, n_rows = make_tables([(40, 50)], [17, 20, 5], 16, seed=15)
    table[2, 1] = n_blocks
    table[3, 0] = -1
    t = run_tables(meta, 1, 3, 16, table, free, n_blocks, n_rows)
    assert (t.slots == -1).sum() == 2


# -- together ------------------------------------------------------------------------------------- #
def test_a_layer_refuses_calls_made_for_another_shape():
    """Rows of other heads, another type or another cache would be read as if they were the plan's."""
    mine = make_params()
    attn = pod.HybridAttention.__new__(pod.HybridAttention)
    attn.params = mine
    batch = wl.make_batch("other", prefill=[], decode_kv_lens=[5], n_q_heads=8, n_kv_heads=2, head_dim=128, dtype=wl.BF16, seed=1)
    q = k = v = torch.zeros(1, 8)
    for other in [dict(hq=4), dict(hkv=1), dict(d=64), dict(dtype=wl.F16), dict(block=0), dict(head_major=True)]:
        theirs = make_params(**other)
        for a, t in [(theirs, mine), (mine, theirs)]:
            with pytest.raises(ValueError, match="in the plan"):
                attn.forward_tokens(batch, pod.TokenAppend(a, device="cpu"), pod.TokenTables(t, 4, device="cpu"), q, k, v)


@pytest.mark.gpu
def test_token_calls_follow_the_current_stream():
    """Inputs that a stream is still writing, read by calls on it: only calls on another stream could see them too early."""
    batch = wl.make_batch("side", prefill=[(50, 333)], decode_kv_lens=[700, 31, 257], n_q_heads=4, n_kv_heads=4, head_dim=64,
                          dtype=wl.F16, seed=42, block_size=0, max_len=704).to("cuda:0")
    attn = pod.HybridAttention(batch)
    tables, append = pod.TokenTables(attn.params, batch.n_rows), pod.TokenAppend(attn.params, rope=pod.Rope(64))
    qkv = torch.randn(batch.n_rows, 12 * 64, device="cuda:0").half()
    layer = lambda meta, x: attn.forward_tokens(batch, append, tables.build(meta), x[:, :256], x[:, 256:512], x[:, 512:])
    want = layer(attn.seq_meta_dev, qkv).clone()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        meta, late = torch.zeros_like(attn.seq_meta_dev), torch.zeros_like(qkv)
        tables.slots.fill_(-1)
        busy = torch.randn(4096, 4096, device="cuda:0")
        for _ in range(4):
            busy = (busy @ busy).tanh()
        meta.copy_(attn.seq_meta_dev)
        late.copy_(qkv)
        got = layer(meta, late)
    torch.cuda.synchronize()
    assert torch.equal(got, want)
    attn.close()


@pytest.mark.gpu
@pytest.mark.parametrize("block,head_major", [(16, False), (24, False), (0, False), (64, True)])
def test_a_layer_from_its_projections(block, head_major):
    """Tables, append and attention of one batch, twice with a step of decoding between, against the oracle on the caches and
    queries that the append left (which the tests above compare with their definition)."""
    prefill, decode = [(150, 401), (64, 64)], [1, 47, 48, 49, 300, 1111]
    batch = wl.make_batch(f"layer-bs{block}", prefill=prefill, decode_kv_lens=decode, n_q_heads=8, n_kv_heads=2, head_dim=128,
                          dtype=wl.F16, seed=77, block_size=block, max_len=1200)
    if head_major:
        batch = wl.to_head_major(batch)
    dev = batch.to("cuda:0")
    attn = pod.HybridAttention(dev)
    n, gen = batch.n_rows, torch.Generator().manual_seed(3)
    tables = pod.TokenTables(attn.params, n + 9)
    free = None
    if block:
        # the new blocks of every request are taken out of the table, in the order in which they come back
        lacks = [(r, i) for r, (_, q, kv, row) in enumerate(batch.seq_meta.tolist()) for i in range(-(-(kv - q) // block), -(-kv // block))]
        free = torch.tensor([int(batch.block_table[r, i]) for r, i in lacks], dtype=torch.int32, device="cuda:0")
        whole = dev.block_table.clone()
        for r, i in lacks:
            dev.block_table[r, i] = -1
    tables.build(attn.seq_meta_dev, free, dev.block_table)
    if block:
        assert torch.equal(dev.block_table, whole)
    assert tables.report.tolist()[1:] == [0, 0, n]
    append = pod.TokenAppend(attn.params, rope=pod.Rope(128, theta=5e5), norm=pod.HeadNorm(eps=1e-6))
    qkv = torch.randn(n + 9, 12 * 128, generator=gen).half().cuda()
    q, k, v = qkv[:, :1024], qkv[:, 1024:1280], qkv[:, 1280:]
    out = attn.forward_tokens(dev, append, tables, q, k, v)
    rows = append(q, k, v, tables.slots, tables.positions, dev.k_cache, dev.v_cache)
    import dataclasses
    seen = dataclasses.replace(dev, prefill_q=rows[:214], decode_q=rows[214:n])
    want = oracle_out(seen.to("cpu"))
    assert np.abs(out.double().cpu().numpy() - want).max() <= 2e-3
    # every new key is where its token belongs
    flat = dev.k_cache.transpose(1, 2) if head_major else dev.k_cache
    flat = flat.reshape(-1, 2, 128)
    per_row = flat.shape[0] // (1 if block else len(batch.seq_meta))
    for r, (start, q_len, kv, row) in enumerate(batch.seq_meta.tolist()):
        at = start + (0 if r < 2 else 214)
        for i in range(q_len):
            t = kv - q_len + i
            slot = int(whole[row, t // block]) * block + t % block if block else row * per_row + t
            assert int(tables.slots[at + i]) == slot and int(tables.positions[at + i]) == t
    attn.close()


@pytest.mark.gpu
def test_tables_append_and_attention_in_one_graph():
    """Captured once and replayed with the program's own work between the replays; each replay against eager calls."""
    batch = wl.make_batch("graph", prefill=[(50, 333)], decode_kv_lens=[700, 31, 257], n_q_heads=4, n_kv_heads=4, head_dim=64,
                          dtype=wl.F16, seed=41, block_size=16).to("cuda:0")
    attn = pod.HybridAttention(batch)
    tables = pod.TokenTables(attn.params, batch.n_rows + 5)
    append = pod.TokenAppend(attn.params, rope=pod.Rope(64))
    qkv = torch.randn(batch.n_rows + 5, 12 * 64, device="cuda:0").half()
    out = torch.zeros(batch.n_rows, 4, 64, dtype=torch.float16, device="cuda:0")
    free = torch.zeros(64, dtype=torch.int32, device="cuda:0")
    lacks = [(r, i) for r, (_, q, kv, _) in enumerate(attn.batch_meta.tolist()) for i in range(-(-(kv - q) // 16), -(-kv // 16))]
    free[:len(lacks)] = torch.stack([batch.block_table[r, i] for r, i in lacks])

    def step():
        tables.build(attn.seq_meta_dev, free, batch.block_table)
        attn.forward_tokens(batch, append, tables, qkv[:, :256], qkv[:, 256:512], qkv[:, 512:], out=out)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(4):
        qkv.copy_(torch.randn(*qkv.shape, generator=torch.Generator().manual_seed(i)).half())
        out.zero_()
        tables.slots.fill_(-7)
        graph.replay()
        torch.cuda.synchronize()
        got, slots = out.clone(), tables.slots.clone()
        step()
        torch.cuda.synchronize()
        assert torch.equal(got, out) and torch.equal(slots, tables.slots) and bool(out.abs().sum() > 0)
    attn.close()


@pytest.mark.gpu
def test_tensors_that_do_not_fit_are_refused():
    app, args, q_out, _ = make_append(*APPENDS[0], seed=5)
    q, k, v, slots, positions, k_cache, v_cache = args
    for bad in [(q.float(), k, v, slots, positions, k_cache, v_cache), (q[:-1], k, v, slots, positions, k_cache, v_cache),
                (q, k.t().contiguous().t(), v, slots, positions, k_cache, v_cache), (q, k, v, slots.long(), positions, k_cache, v_cache),
                (q, k, v, slots.cpu(), positions, k_cache, v_cache), (q, k, v, slots, positions[:-1], k_cache, v_cache),
                (q, k, v, slots, positions, k_cache[:-1], v_cache), (q, k, v, slots, positions, k_cache, v_cache.transpose(1, 2))]:
        with pytest.raises(ValueError):
            app(*bad)
    with pytest.raises(ValueError):
        app(*args, q_out=q_out[:-1])
    with pytest.raises(ValueError):
        pod.TokenAppend(app.params, rope=pod.Rope(256))
    with pytest.raises(ValueError):
        pod.TokenAppend(app.params, norm=pod.HeadNorm(torch.ones(128, device="cuda:0")))
    tables = pod.TokenTables(make_params(n_decode=2), 4)
    meta, free, table = (torch.zeros(*s, dtype=torch.int32, device="cuda:0") for s in ((2, 4), (3,), (8, 8)))
    for bad in [(meta[:1], free, table), (meta.long(), free, table), (meta, free, table[:, :4]), (meta.cpu(), free, table)]:
        with pytest.raises(ValueError):
            tables.build(*bad)


# -- contiguous caches whose rows lie further apart than their tokens --------------------------------- #
def gapped_params(rows=5, tokens=40, gap=72, hq=4, hkv=2, d=64, dtype=wl.F16):
    """Rows of 40 tokens and 72 elements, which are no whole token."""
    return pod.make_params(n_prefill=0, n_decode=rows, n_q_heads=hq, n_kv_heads=hkv, head_dim=d, dtype=dtype, softmax_scale=1.0,
                           n_cache_rows=rows, kv_seq_stride=tokens * hkv * d + gap, n_compute_units=256)


def gapped_cache(rows=5, tokens=40, gap=72, hkv=2, d=64, **kw):
    whole = torch.full((rows, tokens * hkv * d + gap), float("nan"), dtype=torch.float16, **kw)
    return whole, whole[:, :tokens * hkv * d].view(rows, tokens, hkv, d)


def test_caches_whose_rows_lie_apart_are_taken_as_such_and_no_others(monkeypatch):
    """A dense tensor of a cache's shape ends before the last rows that kv_seq_stride names: written as one, the memory behind it."""
    calls = []
    monkeypatch.setattr(pod, "_call", lambda device, function, *args: calls.append(args))
    monkeypatch.setattr(pod, "_stream_of", lambda device: 0)
    i32 = lambda n: torch.zeros(n, dtype=torch.int32)
    for rows in (5, 1):
        append = pod.TokenAppend(gapped_params(rows=rows), device="cpu")
        q, k, v = torch.zeros(3, 256).half(), torch.zeros(3, 128).half(), torch.zeros(3, 128).half()
        whole, apart = gapped_cache(rows=rows)
        dense = apart.contiguous()
        append(q, k, v, i32(3), i32(3), apart, apart)
        assert calls.pop()[14:16] == (whole.data_ptr(), whole.data_ptr())
        for caches in ((dense, apart), (apart, dense), (dense, dense)):
            if rows == 1:                                                # the only row has none behind it
                append(q, k, v, i32(3), i32(3), *caches)
                calls.pop()
                continue
            with pytest.raises(ValueError, match="strides"):
                append(q, k, v, i32(3), i32(3), *caches)
    packed = pod.TokenAppend(make_params(hq=4, d=64, dtype=wl.F16, block=0, rows=5, max_len=40), device="cpu")
    with pytest.raises(ValueError, match="one piece"):
        packed(torch.zeros(3, 256).half(), torch.zeros(3, 128).half(), torch.zeros(3, 128).half(), i32(3), i32(3), gapped_cache()[1], gapped_cache()[1])
    assert calls == []


@pytest.mark.gpu
def test_append_to_a_cache_whose_rows_lie_apart():
    """Every token where its slot names it, nothing between the rows, and the attention reads the same places."""
    prm = gapped_params()
    whole, k_cache = gapped_cache(device="cuda:0")
    whole_v, v_cache = gapped_cache(device="cuda:0")
    append = pod.TokenAppend(prm)
    gen = torch.Generator().manual_seed(2)
    slots = torch.randperm(200, generator=gen)[:90].to(torch.int32)
    q, k, v = (torch.randn(90, n, generator=gen).half().cuda() for n in (256, 128, 128))
    q_out = append(q, k, v, slots.cuda(), torch.zeros(90, dtype=torch.int32, device="cuda:0"), k_cache, v_cache)
    assert torch.equal(q_out.view(90, 256), q)
    for cache, new, memory in ((k_cache, k, whole), (v_cache, v, whole_v)):
        want = torch.full((200, 128), float("nan"), dtype=torch.float16)
        want[slots.long()] = new.cpu()
        got = cache.reshape(200, 128).cpu()
        assert torch.equal(got.view(torch.int16), want.view(torch.int16))
        assert torch.isnan(memory[:, 5120:]).all()


@pytest.mark.gpu
def test_a_layer_over_a_cache_whose_rows_lie_apart():
    """The same batch and projections over a cache in one piece and over one with gaps: the same bits."""
    import dataclasses
    batch = wl.make_batch("apart", prefill=[(50, 333)], decode_kv_lens=[700, 31, 257], n_q_heads=4, n_kv_heads=2, head_dim=64,
                          dtype=wl.F16, seed=43, block_size=0, max_len=704).to("cuda:0")
    stride = batch.kv_seq_stride + 40
    qkv = torch.randn(batch.n_rows, 8 * 64, generator=torch.Generator().manual_seed(4)).half().cuda()

    def layer(b):
        attn = pod.HybridAttention(b)
        tables, append = pod.TokenTables(attn.params, b.n_rows).build(attn.seq_meta_dev), pod.TokenAppend(attn.params, rope=pod.Rope(64))
        out = attn.forward_tokens(b, append, tables, qkv[:, :256], qkv[:, 256:384], qkv[:, 384:])
        torch.cuda.synchronize()
        attn.close()
        return out

    def spread(cache):
        whole = torch.full((4, stride), float("nan"), dtype=torch.float16, device="cuda:0")
        whole[:, :batch.kv_seq_stride] = cache.reshape(4, -1)
        return whole[:, :batch.kv_seq_stride].view(cache.shape)

    other = dataclasses.replace(batch, kv_seq_stride=stride, k_cache=spread(batch.k_cache), v_cache=spread(batch.v_cache))
    want = layer(batch)
    got = layer(other)
    assert torch.equal(got, want) and torch.equal(other.k_cache, batch.k_cache) and torch.equal(other.v_cache, batch.v_cache)


# -- rows that no request owns ------------------------------------------------------------------------- #
def owned_rows_reference(meta, n_prefill, n_decode, block, n_free, free, table, n_rows, n_cache_rows, n_blocks):
    """(slots, positions, how many accepted requests own the row, table): a row without an owner has slot -1 and position 0."""
    per_row, table = table.shape[1] * block, table.copy()
    slots, positions, owners = np.full(n_rows, -1, np.int64), np.zeros(n_rows, np.int64), np.zeros(n_rows, np.int64)
    prows = sum(max(int(m[1]), 0) for m in meta[:n_prefill])
    blocks = lambda n: -(-n // block)
    accepted = []
    for r, (start, q, kv, row) in enumerate(meta.tolist()):
        at = start + (prows if r >= n_prefill else 0)
        if (q >= 1 and kv >= q and start >= 0 and 0 <= row < n_cache_rows and kv <= per_row and
                (start + q <= n_rows if r < n_prefill else q == 1 and start < n_decode)):
            accepted.append((at, q, kv, row))
    enough, taken = sum(blocks(kv) - blocks(kv - q) for _, q, kv, _ in accepted) <= n_free, 0
    for at, q, kv, row in accepted:
        held, need = blocks(kv - q), blocks(kv)
        if enough:
            table[row, held:need] = free[taken:taken + need - held]
            taken += need - held
        inside = max(0, min(q, n_rows - at))                             # (only decode rows can lie behind the last one)
        pos = np.arange(kv - q, kv)[:inside]
        entry = table[row, pos // block]
        owners[at:at + inside] += 1
        positions[at:at + inside] = pos
        slots[at:at + inside] = np.where(enough & (entry >= 0) & (entry < n_blocks), entry * block + pos % block, -1)
    return slots, positions, owners, table


ORDERS = {   # what becomes of (q_start, q_len, kv_len, cache_row) of three prompts, 40, 20 and 33 tokens, and four decodes
    "as they come": {}, "another order": {(0, 0): 53, (1, 0): 33, (2, 0): 0}, "a gap": {(2, 0): 63}, "a gap at the front": {(0, 0): 100},
    "over each other": {(1, 0): 39, (2, 0): 65}, "as far as without a gap": {(1, 0): 0},
    "begins before the rows": {(0, 0): -7}, "ends behind them": {(2, 0): 90}, "no tokens": {(1, 1): 0}, "fewer than none": {(0, 1): -3},
    "more than its context": {(0, 2): 39}, "no such cache row": {(2, 3): 99}, "longer than its cache row": {(1, 2): 1 << 30},
    "a decode before the rows": {(4, 0): -1}, "a decode behind them": {(3, 0): 9}, "the same row twice": {(5, 0): 1}, "none left": {(3, 0): 9, (4, 0): -2, (5, 0): 9, (6, 1): 2},
    "a refused prompt over one that is not": {(1, 0): 0, (1, 2): 5}, "a refused decode's row": {(3, 3): 99}, "a decode of two tokens": {(6, 1): 2}}


@pytest.mark.gpu
@pytest.mark.parametrize("name", ORDERS)
@pytest.mark.parametrize("short", [False, True])
def test_rows_that_no_request_owns_get_no_slot(name, short):
    """A slot left by the batch before would have the append write over a token that is still in use."""
    meta, table, free, n_blocks, n_rows = make_tables([(40, 50), (20, 20), (33, 90)], [17, 1, 32, 48], 16, seed=17, pad=20, missing=1 if short else 0)
    meta[3:, 0] = [0, 2, 1, 3]
    for (request, column), value in ORDERS[name].items():
        meta[request, column] = value
    prm = make_params(n_prefill=3, n_decode=4, block=16, n_blocks=n_blocks, rows=len(meta), max_blocks=table.shape[1])
    tables = pod.TokenTables(prm, n_rows)
    tables.slots.fill_(5)
    tables.positions.fill_(77)
    dev_table = torch.from_numpy(table).cuda()
    tables.build(torch.from_numpy(meta).cuda(), torch.from_numpy(free).cuda(), dev_table)
    slots, positions, owners, want_table = owned_rows_reference(meta, 3, 4, 16, len(free), free, table, n_rows, len(meta), n_blocks)
    once = owners <= 1
    assert tables.slots.cpu().numpy()[once].tolist() == slots[once].tolist()
    assert tables.positions.cpu().numpy()[once].tolist() == positions[once].tolist()
    assert dev_table.tolist() == want_table.tolist()


@pytest.mark.gpu
@pytest.mark.parametrize("prefill", [[], [(70, 70)], [(30000, 30000), (1, 5), (6000, 6000)]])
def test_rows_that_no_request_owns_among_many(prefill):
    """More decode rows than one workgroup looks after, and more rows than are marked at a time; some decodes twice or refused."""
    n = len(prefill)
    rng = np.random.default_rng(18)
    meta, table, free, n_blocks, n_rows = make_tables(prefill, [1 + int(x) for x in rng.integers(0, 40, 20000)], 16, seed=18, pad=9000)
    # (the decode with the most new blocks keeps them: what is changed has none)
    for r in np.flatnonzero((meta[:, 2] - 1) % 16 != 0)[:4000].tolist():
        if r < n:
            continue
        meta[r, 0] = int(rng.choice([-1, 20000, meta[r, 0], int(rng.integers(0, 20000))]))
    for gap in ([0] if n < 2 else [0, 2500]):
        if gap:
            meta[n - 1, 0] += gap
        prm = make_params(n_prefill=n, n_decode=20000, block=16, n_blocks=n_blocks, rows=len(meta), max_blocks=table.shape[1])
        tables = pod.TokenTables(prm, n_rows)
        tables.slots.fill_(5)
        dev_table = torch.from_numpy(table).cuda()
        tables.build(torch.from_numpy(meta).cuda(), torch.from_numpy(free).cuda(), dev_table)
        slots, positions, owners, want_table = owned_rows_reference(meta, n, 20000, 16, len(free), free, table, n_rows, len(meta), n_blocks)
        once = owners <= 1
        assert (owners == 0).sum() > 9000
        assert np.array_equal(tables.slots.cpu().numpy()[once], slots[once])
        assert np.array_equal(tables.positions.cpu().numpy()[once], positions[once])
        assert np.array_equal(dev_table.cpu().numpy(), want_table)


@pytest.mark.gpu
@pytest.mark.parametrize("name,n_rows,changes", [
    ("two rows short", 95, {}), ("no decode row", 93, {}), ("a refused prompt of many tokens", 105, {(1, 1): 1 << 30}),
    ("a refused prompt of more than there are rows for", 105, {(1, 1): 28, (1, 2): 27}), ("a row short, the free list as well", 96, {})])
def test_decodes_behind_the_last_row_take_no_blocks(name, n_rows, changes):
    """What the report says was taken is what the table's rows have got: a block taken for a row that is not there would be lost."""
    meta, table, free, n_blocks, _ = make_tables([(40, 50), (20, 20), (33, 90)], [17, 1, 33, 49], 16, seed=19, missing=1 if "free" in name else 0)
    meta[3:, 0] = [0, 2, 1, 3]
    for (request, column), value in changes.items():
        meta[request, column] = value
    prm = make_params(n_prefill=3, n_decode=4, block=16, n_blocks=n_blocks, rows=len(meta), max_blocks=table.shape[1])
    tables = pod.TokenTables(prm, n_rows)
    tables.slots.fill_(5)
    dev_table = torch.from_numpy(table).cuda()
    tables.build(torch.from_numpy(meta).cuda(), torch.from_numpy(free).cuda(), dev_table)
    prows = int(meta[:3, 1].sum())
    served = [r for r in range(7) if (r != 1 or not changes) and (r < 3 or prows + meta[r, 0] < n_rows)]
    need = [-(-int(meta[r, 2]) // 16) - -(-int(meta[r, 2] - meta[r, 1]) // 16) for r in served]
    # ("the free list as well": a block short for the whole batch, exactly enough without the decode left out)
    assert sum(need) <= len(free) and ("free" not in name or sum(need) == len(free))
    want = table.copy()
    taken = 0
    slots = np.full(n_rows, -1)
    for r, n in zip(served, need):
        start, q, kv, row = meta[r].tolist()
        held = -(-(kv - q) // 16)
        want[row, held:held + n] = free[taken:taken + n]
        taken += n
        at = start + (prows if r >= 3 else 0)
        slots[at:at + q] = [want[row, t // 16] * 16 + t % 16 for t in range(kv - q, kv)]
    assert dev_table.tolist() == want.tolist()
    assert tables.report.tolist() == [taken, 0, 1 if changes else 0, prows + 4]
    assert tables.slots.tolist() == slots.tolist()


def test_a_layer_refuses_slots_of_another_cache_and_rows_of_another_batch():
    """A slot of a contiguous cache is row * length + token: read with another length it is another request's token."""
    batch = wl.make_batch("other", prefill=[], decode_kv_lens=[5], n_q_heads=8, n_kv_heads=2, head_dim=128, dtype=wl.BF16, seed=1)
    q = k = v = torch.zeros(1, 8)
    for mine, others in [(dict(block=0), [dict(max_len=48), dict(max_len=65), dict(rows=9)]), (dict(), [dict(n_blocks=63)])]:
        for other in others:
            ours, theirs = make_params(**mine), make_params(**{**mine, **other})
            attn = pod.HybridAttention.__new__(pod.HybridAttention)
            attn.params = ours
            for a, t in [(theirs, ours), (ours, theirs), (theirs, theirs)]:
                with pytest.raises(ValueError, match="in the plan"):
                    attn.forward_tokens(batch, pod.TokenAppend(a, device="cpu"), pod.TokenTables(t, 4, device="cpu"), q, k, v)
    attn = pod.HybridAttention.__new__(pod.HybridAttention)
    attn.params = make_params(n_prefill=1, n_decode=3)
    for counts in [(0, 3), (1, 2), (2, 3), (3, 1)]:
        theirs = make_params(n_prefill=counts[0], n_decode=counts[1])
        with pytest.raises(ValueError, match="beside a plan for"):
            attn.forward_tokens(batch, pod.TokenAppend(theirs, device="cpu"), pod.TokenTables(theirs, 4, device="cpu"), q, k, v)
    # the length of a paged cache's rows and the table's width name no place
    attn = pod.HybridAttention.__new__(pod.HybridAttention)
    attn.params, attn.info = make_params(n_decode=1), pod.PlanInfo()
    theirs = make_params(n_decode=1, rows=3, max_blocks=5)
    theirs.kv_seq_stride = 640
    with pytest.raises(ValueError, match="slots must|q must"):
        attn.forward_tokens(batch, pod.TokenAppend(theirs, device="cpu"), pod.TokenTables(theirs, 1, device="cpu"), q, k, v)


def test_a_layer_refuses_a_batch_of_other_rows_than_the_plan():
    """The attention writes the plan's rows: those of a batch with fewer would end before it does."""
    attn = pod.HybridAttention.__new__(pod.HybridAttention)
    attn.params, attn.info = make_params(n_prefill=1, n_decode=2), pod.PlanInfo(n_prefill_rows=7)
    append, tables = pod.TokenAppend(attn.params, device="cpu"), pod.TokenTables(attn.params, 40, device="cpu")
    x = torch.zeros(40, 8)
    for prefill, decode in [([(6, 6)], [5, 9]), ([(8, 8)], [5, 9]), ([(7, 9)], [5]), ([(7, 9)], [5, 5, 5]), ([], [5, 9])]:
        batch = wl.make_batch("other", prefill=prefill, decode_kv_lens=decode, n_q_heads=8, n_kv_heads=2, head_dim=128, dtype=wl.BF16, seed=1)
        with pytest.raises(ValueError, match="rows beside a plan for"):
            attn.forward_tokens(batch, append, tables, x, x, x)
    batch = wl.make_batch("mine", prefill=[(7, 9)], decode_kv_lens=[5, 9], n_q_heads=8, n_kv_heads=2, head_dim=128, dtype=wl.BF16, seed=1)
    with pytest.raises(ValueError, match="q must"):
        attn.forward_tokens(batch, append, tables, x, x, x)
