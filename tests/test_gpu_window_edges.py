"""Windowed prefill where the cache holds numbers that are not finite, through each of the kernels that a run can be served by.

Which kernel that was is read from the device's own record of its launches, so that a changed rule on sizes cannot leave one of them
untested.  Tolerances are those of the windowed calls on finite caches (tests/test_gpu_window.py); a row that is worked out by itself
has fewer roundings than the others.
"""
import json
import re
import warnings

import numpy as np
import pytest
import torch
from torch.profiler import ProfilerActivity, profile

from oracle import attention, e5m2
from paper_2602_09323_b200 import binding
from tests import helpers
from tests.test_gpu_window import check, make, prefill

pytestmark = pytest.mark.gpu

# name: (lens, q_lens, kv heads, group, window, sinks).  More than 512 query tokens are never rows of the decode kernel; tiles
# that leave the device's SMs room are one to a CTA, and where a window has several tiles of keys those are shared by a cluster.
RUNS = {
    "rows": ([403, 64, 9, 700], [4, 3, 9, 5], 2, 5, 200, 3),
    "one tile": ([900, 700, 40], [300, 250, 40], 2, 4, 60, 3),
    "cluster": ([1900, 700, 40], [300, 250, 40], 2, 4, 1000, 3),
    "two tiles": ([900, 420, 300, 77] * 4, [300, 20, 300, 40] * 4, 4, 4, 150, 3),
    "small": ([400, 33, 90] * 14, [25, 33, 17] * 14, 8, 3, 120, 3),
}
KERNELS = {"rows": (64, 128), "one tile": (64, 128), "cluster": (64, 128), "two tiles": (64, 128), "small": (64,)}
ROUTES = [(name, dim) for name, dims in KERNELS.items() for dim in dims]


def served_by(call, tmp_path):
    """The result of a call, and its attention kernels: names and numbers of CTAs.  None where the device's record is not to be
    had (another profiler holds it): what was computed is tested all the same."""
    with profile(activities=[ProfilerActivity.CUDA], acc_events=True) as prof:
        result = call()
        torch.cuda.synchronize()
    path = str(tmp_path / "launches.json")
    prof.export_chrome_trace(path)
    with open(path) as f:
        seen = [(e["name"], e["args"]["grid"][0]) for e in json.load(f)["traceEvents"] if e.get("cat") == "kernel"]
    if not seen:
        warnings.warn("no record of launches: which kernel served a call is not checked")
        return result, None
    return result, [x for x in seen if "paged_" in x[0]]


def check_route(launches, w, route):
    assert launches is None or route_of(launches, w) == route


def route_of(launches, w):
    (name, grid), = launches
    if "paged_decode_kernel" in name:
        assert re.search(r"true>", name), name             # rows that are query tokens
        return "rows"
    turns, window, small = re.search(r"paged_prefill_kernel<\d+, \w+, (\w+), (\w+), (\w+)>", name).groups()
    assert window == "true", name
    if small == "true":
        return "small"
    if turns == "true":
        return "two tiles"
    tile = 128 // (w.num_q_heads // w.num_kv_heads)
    pieces = (w.q.shape[0] // tile + w.batch) * w.num_kv_heads
    assert grid % pieces == 0
    return "one tile" if grid == pieces else "cluster"


def runs(name, dim, fmt, seed):
    lens, q_lens, hkv, group, window, sinks = RUNS[name]
    w, cache, kv, table = make(lens, q_lens, group * hkv, hkv, dim, fmt, window, sinks, seed=seed)
    ref, spread = attention.window_attention(w.q.float().numpy(), kv, w.block_table.numpy(), lens, window, sinks, w.cu_q_lens.numpy())
    return w, cache, table, ref, spread


def granules(w, cache):
    return cache.data.view(w.num_blocks, w.num_kv_heads, cache.granule_bytes), torch.from_numpy(helpers.granule_index_map(cache))


def positions(name, w):
    """Of every query row: its sequence and its position."""
    lens, q_lens = RUNS[name][:2]
    of = np.repeat(np.arange(len(lens)), q_lens)
    at = np.concatenate([L - n + np.arange(n) for L, n in zip(lens, q_lens)])
    return of, at


def some_tokens(name):
    """Per sequence, tokens that some queries of a run see and others do not: one at the window's lower edge, one in the run."""
    lens, q_lens, _, _, window, _ = RUNS[name]
    picked = []
    for L, n in zip(lens, q_lens):
        edge = L - n - window + 1 + n // 2                 # seen by the first half of the run
        picked.append(sorted({p for p in (edge, L - n + n // 3) if 3 <= p < L}))
    return picked


@pytest.mark.parametrize("fmt,code", [("e4m3", 0x7F), ("e5m2", 0x7C), ("e5m2", 0xFE)])
@pytest.mark.parametrize("name,dim", ROUTES)
def test_a_value_that_is_not_finite_reaches_those_who_see_it_and_no_one_else(name, dim, fmt, code, tmp_path):
    w, cache, table, ref, spread = runs(name, dim, fmt, seed=301)
    window, sinks, group = RUNS[name][4], RUNS[name][5], RUNS[name][3]
    raw, idx = granules(w, cache)
    of, at = positions(name, w)
    sees = np.zeros(len(of), dtype=bool)
    for b, picked in enumerate(some_tokens(name)):
        for pos in picked:
            raw[int(table[b, pos // 16]), 1, int(idx[1, pos % 16, 5])] = code      # dim 5 of its value, kv head 1
            sees |= (of == b) & (at >= pos) & ((at - window < pos) | (pos < sinks))
    assert 0 < sees.sum() < len(sees)
    out, launches = served_by(lambda: prefill(w, cache, table, window, sinks, extra_rows=2), tmp_path)
    check_route(launches, w, name)
    spoilt = out[torch.from_numpy(sees)][:, group:2 * group, 5].float()
    assert not torch.isfinite(spoilt).any()
    out = out.clone()
    hit = np.zeros(ref.shape, dtype=bool)
    hit[sees, group:2 * group, 5] = True
    out[torch.from_numpy(hit)] = torch.from_numpy(ref[hit]).to(torch.bfloat16).cuda()
    check(out, ref, spread, fmt, prefill=True, vmax=6.0, what=name)


@pytest.mark.parametrize("name,dim", ROUTES)
def test_a_value_scale_that_is_infinite_reaches_those_who_see_its_block(name, dim, tmp_path):
    """What a token with an infinite value leaves: codes of zero under a scale that is infinite."""
    w, cache, table, ref, spread = runs(name, dim, "e4m3", seed=303)
    lens, q_lens, _, group, window, sinks = RUNS[name]
    raw, idx = granules(w, cache)
    of, at = positions(name, w)
    sees = np.zeros(len(of), dtype=bool)
    for b, picked in enumerate(some_tokens(name)):
        for pos in picked[:1]:
            blk = pos // 16
            header = raw[int(table[b, blk]), 0, 32 * dim:32 * dim + 8].clone().view(torch.float32)
            header[1] = float("inf")
            raw[int(table[b, blk]), 0, 32 * dim:32 * dim + 8] = header.view(torch.uint8)
            for t in range(16 * blk, min(16 * blk + 16, lens[b])):
                sees |= (of == b) & (at >= t) & ((at - window < t) | (t < sinks))
    assert sees.any() and (name == "rows" or not sees.all())      # (every token of a short run sees those blocks)
    out, launches = served_by(lambda: prefill(w, cache, table, window, sinks), tmp_path)
    check_route(launches, w, name)
    assert not torch.isfinite(out[torch.from_numpy(sees)][:, :group].float()).any()
    out = out.clone()
    hit = np.zeros(ref.shape, dtype=bool)
    hit[sees, :group] = True
    out[torch.from_numpy(hit)] = torch.from_numpy(ref[hit]).to(torch.bfloat16).cuda()
    check(out, ref, spread, "e4m3", prefill=True, vmax=6.0, what=name)


@pytest.mark.parametrize("name,dim", ROUTES)
def test_an_infinite_key(name, dim, tmp_path):
    """E5M2: a logit of -inf has no weight, one of +inf makes the outputs of those who see it NaN.  Elements of the query from large to
    as small as bf16 goes, so that an inexact form of one is zero, or of the other sign, where it is not."""
    lens, q_lens, hkv, group, window, sinks = RUNS[name]
    w, cache, kv, table = make(lens, q_lens, group * hkv, hkv, dim, "e5m2", window, sinks, seed=307)
    gen = torch.Generator().manual_seed(311)
    w.q[:, :, 0] = (2.0 ** -torch.randint(0, 100, w.q.shape[:2], generator=gen)).to(torch.bfloat16) * (1 + torch.rand(w.q.shape[:2], generator=gen))
    assert (w.q[:, :, 0] > 0).all()
    codes = kv[0].copy()
    raw, idx = granules(w, cache)
    of, at = positions(name, w)
    sees = np.zeros(len(of), dtype=bool)
    for b, picked in enumerate(some_tokens(name)):
        for pos in [0] + picked:
            blk, tok = int(table[b, pos // 16]), pos % 16
            raw[blk, 1, int(idx[0, tok, 0])] = codes[blk, 1, 0, tok, 0] = 0xFC       # -inf in dim 0 of its key, kv head 1
            if pos:
                raw[blk, 0, int(idx[0, tok, 0])] = 0x7C                           # +inf, kv head 0
                sees |= (of == b) & (at >= pos) & ((at - window < pos) | (pos < sinks))
    assert sees.any() and not sees.all()
    ref, spread = attention.window_attention(w.q.float().numpy(), (codes, kv[1], e5m2), w.block_table.numpy(), lens, window, sinks, w.cu_q_lens.numpy())
    assert np.isfinite(ref).all()
    out, launches = served_by(lambda: prefill(w, cache, table, window, sinks), tmp_path)
    check_route(launches, w, name)
    assert torch.isnan(out[torch.from_numpy(sees)][:, :group].float()).all()
    out = out.clone()
    hit = np.zeros(ref.shape, dtype=bool)
    hit[sees, :group] = True
    out[torch.from_numpy(hit)] = torch.from_numpy(ref[hit]).to(torch.bfloat16).cuda()
    check(out, ref, spread, "e5m2", prefill=True, vmax=6.0, what=name)


@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
@pytest.mark.parametrize("name,dim", ROUTES)
def test_a_nan_key_reaches_those_who_see_it_and_no_one_else(name, dim, fmt, tmp_path):
    """Keys that only a part of a run sees, of kv head 1."""
    w, cache, table, ref, spread = runs(name, dim, fmt, seed=313)
    group, window, sinks = RUNS[name][3:]
    raw, idx = granules(w, cache)
    of, at = positions(name, w)
    before = prefill(w, cache, table, window, sinks)
    check(before, ref, spread, fmt, prefill=True, vmax=6.0, what=name)
    sees = np.zeros(len(of), dtype=bool)
    for b, picked in enumerate(some_tokens(name)):
        for pos in picked:
            raw[int(table[b, pos // 16]), 1, int(idx[0, pos % 16, 3])] = 0x7F
            sees |= (of == b) & (at >= pos) & ((at - window < pos) | (pos < sinks))
    assert sees.any() and not sees.all()
    out, launches = served_by(lambda: prefill(w, cache, table, window, sinks), tmp_path)
    check_route(launches, w, name)
    sees = torch.from_numpy(sees)
    assert torch.isnan(out[sees][:, group:2 * group].float()).all()
    assert torch.equal(out[~sees], before[~sees]) and torch.equal(out[:, :group], before[:, :group]) and torch.equal(out[:, 2 * group:], before[:, 2 * group:])


@pytest.mark.parametrize("fmt", ["e4m3", "bf16"])
def test_calls_without_a_query(fmt):
    """A step in which no sequence takes part, and a batch of runs that are all empty."""
    w, cache, kv, table = make([40, 70], [1, 1], 4, 2, 64, fmt, 9, 1, seed=317)
    ws = binding.new_workspace(2, 4, 2, 64, table.shape[1])
    q, none = torch.zeros(0, 4, 64, dtype=torch.bfloat16, device="cuda"), torch.zeros(0, dtype=torch.int32, device="cuda")
    new = torch.zeros(0, 2, 64, dtype=torch.bfloat16, device="cuda")
    before = cache.data.clone()
    for more in ((), (new, new, none.long())):
        out = binding.window_decode(cache, q, table[:0].cuda(), none, 9, 1, w.sm_scale, ws, *more)
        assert out.shape == q.shape
    if fmt != "bf16":
        out = binding.window_prefill(cache, q, torch.zeros(3, dtype=torch.int32, device="cuda"), table.cuda(), torch.tensor([40, 70], dtype=torch.int32, device="cuda"),
                                     9, 1, w.sm_scale, ws)
        assert out.shape == q.shape
        with pytest.raises(ValueError):
            binding.window_prefill(cache, q, torch.zeros(2, dtype=torch.int32, device="cuda"), table.cuda(), none, 9, 1, w.sm_scale, ws)
    torch.cuda.synchronize()
    assert binding.workspace_status(ws) == 0 and torch.equal(cache.data, before)


@pytest.mark.parametrize("name,dim", ROUTES)
def test_a_nan_value_under_scales_that_are_zero(name, dim, tmp_path):
    """What a token leaves whose value is NaN where its block holds zeros: NaN codes under a scale of zero."""
    w, cache, table, ref, spread = runs(name, dim, "e4m3", seed=331)
    lens, q_lens, _, group, window, sinks = RUNS[name]
    raw, idx = granules(w, cache)
    raw[:, 0, 16 * dim:32 * dim] = 0
    raw[:, 0, 32 * dim + 4:32 * dim + 8] = 0
    ref[:, :group], spread[:, :group] = 0, 0
    of, at = positions(name, w)
    sees = np.zeros(len(of), dtype=bool)
    for b, picked in enumerate(some_tokens(name)):
        for pos in picked:
            raw[int(table[b, pos // 16]), 0, int(idx[1, pos % 16, 7])] = 0x7F
            sees |= (of == b) & (at >= pos) & ((at - window < pos) | (pos < sinks))
    assert sees.any() and not sees.all()
    out, launches = served_by(lambda: prefill(w, cache, table, window, sinks), tmp_path)
    check_route(launches, w, name)
    out = out.clone()
    hit = np.zeros(ref.shape, dtype=bool)
    hit[sees, :group, 7] = True
    assert torch.isnan(out[torch.from_numpy(hit)].float()).all()
    out[torch.from_numpy(hit)] = 0
    assert not out[:, :group].any()
    check(out, ref, spread, "e4m3", prefill=True, vmax=6.0, what=name)
