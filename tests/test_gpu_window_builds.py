"""Every build of the windowed decode kernel that a call can be served by: a cluster to a unit (a sequence and kv head), a CTA to a
unit of which one, two or three fit an SM, and the line.  Which one a call took is read from the device's own record of its
launches, so that a changed rule on sizes cannot leave one of them untested.  Tolerances: those of tests/test_gpu_window.py."""
import re

import numpy as np
import pytest
import torch

from oracle import attention, e4m3, e5m2, kv_cache
from paper_2602_09323_b200 import binding, workloads
from tests import helpers
from tests.test_gpu_window import FMT, check, decode, make
from tests.test_gpu_window_edges import granules, served_by

pytestmark = pytest.mark.gpu

# name: (sequences, kv heads, window)
CALLS = {"cluster": (3, 2, 700), "one": (19, 7, 150), "two": (33, 8, 150), "three": (52, 8, 90), "line": (60, 8, 90)}
SINKS = 9
BUILDS = [(name, fmt, dim) for name in CALLS for fmt in ("e4m3", "e5m2", "bf16") for dim in (64, 128)]


def lengths(name):
    batch, _, window = CALLS[name]
    lens = [(b * 7919) % (2 * window) for b in range(batch)]
    lens[0], lens[1] = 2 * window + 1, 1
    return lens


def check_route(launches, units, route):
    assert launches is None or route_of(launches, units) == route


def route_of(launches, units):
    """(A bf16 cache takes its new tokens by a launch of its own.)"""
    (name, grid), = [x for x in launches if "paged_decode_kernel" in x[0]]
    layers, window, few, runs = re.search(r"paged_decode_kernel<\d+, \d+, (\d+), (\w+), (\d+), (\w+)>", name).groups()
    assert (layers, window, runs) == ("1", "true", "false"), name
    if few == "1" and grid > units:
        return "cluster"
    return ("line", "one", "two", "three")[int(few)]


def problem(name, fmt, dim, seed, poison=True):
    batch, hkv, window = CALLS[name]
    lens = lengths(name)
    w, cache, kv, table = make(lens, [1] * batch, 2 * hkv, hkv, dim, fmt, window, SINKS, seed=seed, poison=poison)
    return lens, w, cache, kv, table, batch * hkv


@pytest.mark.parametrize("name,fmt,dim", BUILDS)
def test_a_call_against_the_oracle(name, fmt, dim, tmp_path):
    lens, w, cache, kv, table, units = problem(name, fmt, dim, 401)
    window = CALLS[name][2]
    ref, spread = attention.window_attention(w.q.float().numpy(), kv, w.block_table.numpy(), lens, window, SINKS)
    out, launches = served_by(lambda: decode(w, cache, table, lens, window, SINKS), tmp_path)
    check_route(launches, units, name)
    check(out, ref, spread, fmt, what=name)
    assert torch.equal(out, decode(w, cache, table, lens, window, SINKS))


@pytest.mark.parametrize("name,dim", [(name, dim) for name in CALLS for dim in (64, 128)])
def test_a_key_of_minus_infinity_and_queries_from_large_to_small(name, dim, tmp_path):
    """E5M2: elements of the query as small as bf16 goes do not make a NaN of an infinite key."""
    lens, w, cache, kv, table, units = problem(name, "e5m2", dim, 409)
    window = CALLS[name][2]
    gen = torch.Generator().manual_seed(419)
    sign = 1 - 2 * torch.randint(0, 2, (w.batch, w.num_kv_heads, 1), generator=gen)
    w.q[:, :, 0] = ((2.0 ** -torch.randint(0, 133, (w.batch, w.num_kv_heads, 2), generator=gen).double()) * sign).flatten(1).to(torch.bfloat16)
    assert (w.q[:, :, 0] != 0).all()
    codes = kv[0].copy()
    raw, idx = granules(w, cache)
    for b, L in enumerate(lens):
        for pos in {0, L - 1} if L > 1 else set():
            blk = int(table[b, pos // 16])
            for h in range(w.num_kv_heads):
                code = 0xFC if sign[b, h] > 0 else 0x7C
                raw[blk, h, int(idx[0, pos % 16, 0])] = codes[blk, h, 0, pos % 16, 0] = code
    ref, spread = attention.window_attention(w.q.float().numpy(), (codes, kv[1], e5m2), w.block_table.numpy(), lens, window, SINKS)
    assert np.isfinite(ref).all()
    out, launches = served_by(lambda: decode(w, cache, table, lens, window, SINKS), tmp_path)
    check_route(launches, units, name)
    check(out, ref, spread, "e5m2", what=name)


@pytest.mark.parametrize("name,fmt,dim", BUILDS)
def test_new_tokens_in_every_build(name, fmt, dim, tmp_path):
    """Three steps in a row, so that blocks are opened, their scales grow and stay: the bytes are those of the write rule, the output
    that of the call over the written cache."""
    batch, hkv, window = CALLS[name]
    first = [max(0, L - 3) for L in lengths(name)]
    first[0] = 2 * window - 2 + (-(2 * window)) % 16       # its third step opens a block
    w = workloads.make_workload("append", [L + 3 for L in first], 2 * hkv, hkv, dim, seed=421)
    cache = binding.Cache(w.num_blocks, hkv, dim, FMT[fmt])
    kind = {"e4m3": e4m3, "e5m2": e5m2}.get(fmt)
    codes, scales = kv_cache.new_cache(w.num_blocks, hkv, dim)
    values = kv_cache.new_cache_bf16(w.num_blocks, hkv, dim)
    rows = np.concatenate([np.arange(w.kv_offsets[b], w.kv_offsets[b] + L) for b, L in enumerate(first)])

    def oracle_write(rows, slots, **more):
        k, v, slots = w.k[rows].float().numpy(), w.v[rows].float().numpy(), slots.numpy()
        if fmt == "bf16":
            kv_cache.kv_write_bf16(values, k, v, slots)
        else:
            kv_cache.kv_write(codes, scales, k, v, slots, fmt=kind, **more)

    binding.kv_write(cache, w.k[rows].cuda(), w.v[rows].cuda(), w.slot_mapping[rows].cuda())
    oracle_write(rows, w.slot_mapping[rows])
    ws = binding.new_workspace(batch, 2 * hkv, hkv, dim, w.block_table.shape[1])
    table, gen = w.block_table.cuda(), torch.Generator().manual_seed(431)
    for step in range(3):
        lens = [L + step + 1 for L in first]
        lens[2] = 0                                        # a row of the batch without a sequence
        last = torch.tensor([w.kv_offsets[b] + first[b] + step for b in range(batch)])
        slots = w.slot_mapping[last].clone()
        slots[2] = -1
        oracle_write(last.numpy(), slots, **({} if fmt == "bf16" else {"reciprocal": True}))
        q = torch.randn(batch, 2 * hkv, dim, generator=gen).to(torch.bfloat16).cuda()
        args = (cache, q, table, torch.tensor(lens, dtype=torch.int32).cuda(), window, SINKS, w.sm_scale, ws)
        new = (w.k[last].cuda(), w.v[last].cuda(), slots.cuda())
        out, launches = served_by(lambda: binding.window_decode(*args, *new), tmp_path)
        check_route(launches, batch * hkv, name)
        want = binding.window_decode(*args)
        torch.cuda.synchronize()
        assert binding.workspace_status(ws) == 0
        if fmt == "bf16":
            assert np.array_equal(helpers.cache_to_logical(cache), values), step
        else:
            helpers.check_cache_bit_exact(cache, codes, scales, what=f"step {step}")
        assert torch.equal(out, want) and torch.all(out[2] == 0), step


@pytest.mark.parametrize("name,fmt,dim", BUILDS)
def test_a_nan_key_in_every_build(name, fmt, dim, tmp_path):
    """The last token's key of kv head 0: its outputs are NaN, all others as they were."""
    lens, w, cache, kv, table, units = problem(name, fmt, dim, 433)
    window = CALLS[name][2]
    before = decode(w, cache, table, lens, window, SINKS)
    there = torch.tensor([L > 0 for L in lens])
    raw, idx = granules(w, cache)
    for b, L in enumerate(lens):
        if L:
            at = int(idx[0, (L - 1) % 16, dim - 1])
            for byte in range(2 if fmt == "bf16" else 1):
                raw[int(table[b, (L - 1) // 16]), 0, at + byte] = 0xC0 if fmt == "bf16" and byte == 0 else 0x7F
    out, launches = served_by(lambda: decode(w, cache, table, lens, window, SINKS), tmp_path)
    check_route(launches, units, name)
    assert torch.isnan(out[there][:, :2].float()).all()
    assert torch.equal(out[:, 2:], before[:, 2:]) and torch.equal(out[~there], before[~there])


@pytest.mark.parametrize("name,fmt,dim", BUILDS)
def test_a_nan_value_without_weight_in_every_build(name, fmt, dim, tmp_path):
    """Logits so far apart that nearly all weights, and those of whole pieces of a softmax, are zero in fp32: zero times NaN is NaN
    wherever the token lies.  The other dims are as they were."""
    lens, w, cache, kv, table, units = problem(name, fmt, dim, 439)
    window = CALLS[name][2]
    w.q *= 512
    before = decode(w, cache, table, lens, window, SINKS)
    raw, idx = granules(w, cache)
    there = torch.tensor([L > 0 for L in lens])
    for b, L in enumerate(lens):
        if L:
            for h in range(w.num_kv_heads):
                pos = L - 1 - (37 * b + 11 * h) % min(L, window)
                at = int(idx[1, pos % 16, 5])
                for byte in range(2 if fmt == "bf16" else 1):
                    raw[int(table[b, pos // 16]), h, at + byte] = 0xC0 if fmt == "bf16" and byte == 0 else 0x7F
    out, launches = served_by(lambda: decode(w, cache, table, lens, window, SINKS), tmp_path)
    check_route(launches, units, name)
    assert torch.isnan(out[there][:, :, 5].float()).all()
    rest = [d for d in range(dim) if d != 5]
    assert torch.equal(out[there][:, :, rest], before[there][:, :, rest]) and torch.equal(out[~there], before[~there])
