"""Attention with a sliding window and sinks against the float64 oracle, at the sizes, masks and tables where it can go wrong.

Tolerance.  With A = sum_j p_j |v_j| and o the exact output: the bf16 result is off by half a step, 2^-8 |o| at most.  A
probability is rounded to f16 once, 2^-11 A at most.  For these inputs (N(0, 1), D <= 128) sm_scale sum |q_d k_d| is about 8, so
fp32 accumulation moves a logit by less than 2^-16, the scales' products and the exponential's 2 ulp less than that, which moves
the result by less than 2^-13 A.  Decode from an FP8 cache: 2^-8 |o| + 2^-10 A.  A bf16 cache carries probabilities as two bf16
halves (2^-16): 2^-8 |o| + 2^-11 A.  Prefill: the E4M3 terms of the query move a logit by at most sm_scale 2^-17 max|q| sum|k| < 2^-11,
the result by twice that times A; weights below 2^-14 of the reference lose 2^-25 each, below 2^-13 max|v| for 4096 keys:
2^-8 |o| + 2^-9 A + 2^-13 max|v|.
"""
import numpy as np
import pytest
import torch

from oracle import attention, e4m3, e5m2, kv_cache
from paper_2602_09323_b200 import binding, workloads
from tests import helpers

pytestmark = pytest.mark.gpu

FMT = {"e4m3": binding.KV_FP8_E4M3, "e5m2": binding.KV_FP8_E5M2, "bf16": binding.KV_BF16}
LENS = [0, 1, 2, 15, 16, 17, 31, 33, 48, 100, 129, 500, 1000, 1500]
WINDOWS = [(1, 0), (1, 1), (2, 40), (16, 4), (17, 16), (64, 33), (100, 0), (513, 5), (2 ** 31 - 1, 0), (1, 2 ** 31 - 1)]


def visible_blocks(L, n, window, sinks):
    if n <= 0 or L <= 0:
        return []
    j = np.arange(L)
    first = L - n                                       # the queries' windows begin at first - window + 1 and reach to L - 1
    return sorted(set((j[(j < sinks) | (j > first - window)] // 16).tolist()))


def make(lens, q_lens, hq, hkv, dim, fmt, window, sinks, seed, poison=True, width=None):
    """A cache filled through kv_write, a table that names only blocks with visible tokens, hidden tokens of those turned into
    NaN codes; and the oracle's view of the cache from before that."""
    w = workloads.make_workload("window", lens, hq, hkv, dim, seed=seed, q_lens=q_lens, outliers=False)
    cache = helpers.gpu_fill(w, FMT[fmt])
    kv = helpers.cache_to_logical(cache)
    kv = kv if fmt == "bf16" else (kv[0], kv[1], e4m3 if fmt == "e4m3" else e5m2)
    table = torch.full((len(lens), max(w.block_table.shape[1], width or 1)), -1, dtype=torch.int32)
    raw = cache.data.view(w.num_blocks, hkv, cache.granule_bytes)
    idx = torch.from_numpy(helpers.granule_index_map(cache))
    for b, (L, n) in enumerate(zip(lens, q_lens)):
        for j in visible_blocks(L, n, window, sinks):
            blk = int(w.block_table[b, j])
            table[b, j] = blk
            pos = j * 16 + np.arange(16)
            hidden = (pos >= L) | ((pos >= sinks) & (pos <= L - n - window))
            if poison and hidden.any():
                at = idx[:, hidden].reshape(-1)
                for byte in range(2 if fmt == "bf16" else 1):
                    raw[blk][:, (at + byte).cuda()] = 0x7F if fmt != "bf16" or byte == 1 else 0xC0
    return w, cache, kv, table


def check(got, ref, spread, fmt, prefill=False, vmax=0.0, what=""):
    g = got.double().cpu().numpy()
    bound = 2.0 ** -8 * np.abs(ref) + (2.0 ** -9 if prefill else 2.0 ** -11 if fmt == "bf16" else 2.0 ** -10) * spread + 2.0 ** -30
    if prefill:
        bound += 2.0 ** -13 * vmax
    assert np.isfinite(g).all(), f"{what}: not finite"
    bad = np.abs(g - ref) > bound
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size} off, worst {np.max(np.abs(g - ref) / bound):.2f} times the bound, at {np.argwhere(bad)[:3].tolist()}"


def decode(w, cache, table, lens, window, sinks, **more):
    ws = binding.new_workspace(len(lens), w.num_q_heads, w.num_kv_heads, w.head_dim, table.shape[1])
    out = torch.full((len(lens), w.num_q_heads, w.head_dim), float("nan"), dtype=torch.bfloat16, device="cuda")
    binding.window_decode(cache, w.q.cuda(), table.cuda(), torch.tensor(lens, dtype=torch.int32).cuda(), window, sinks, w.sm_scale, ws, out=out, **more)
    torch.cuda.synchronize()
    assert binding.workspace_status(ws) == 0
    return out


def prefill(w, cache, table, window, sinks, extra_rows=0):
    lens = w.context_lens
    ws = binding.new_workspace(max(1, len(lens)), w.num_q_heads, w.num_kv_heads, w.head_dim, table.shape[1])
    q = torch.cat([w.q, torch.full((extra_rows, *w.q.shape[1:]), float("nan"), dtype=torch.bfloat16)]).cuda()
    out = torch.full_like(q, 77.0)
    binding.window_prefill(cache, q, w.cu_q_lens.cuda(), table.cuda(), w.context_lens_tensor.cuda(), window, sinks, w.sm_scale, ws, out=out)
    torch.cuda.synchronize()
    assert binding.workspace_status(ws) == 0
    assert torch.all(out[w.q.shape[0]:] == 77.0)
    return out[:w.q.shape[0]]


@pytest.mark.parametrize("fmt,dim,group", [("e4m3", 128, 5), ("e4m3", 64, 8), ("e5m2", 128, 1), ("e5m2", 64, 4), ("bf16", 128, 2), ("bf16", 64, 7)])
def test_decode_against_the_oracle(fmt, dim, group):
    hkv = 2
    for n, (window, sinks) in enumerate(WINDOWS):
        w, cache, kv, table = make(LENS, [1] * len(LENS), group * hkv, hkv, dim, fmt, window, sinks, seed=100 + n)
        out = decode(w, cache, table, LENS, window, sinks)
        ref, spread = attention.window_attention(w.q.float().numpy(), kv, w.block_table.numpy(), LENS, window, sinks)
        check(out, ref, spread, fmt, what=f"window {window} sinks {sinks}")
        assert torch.all(out[0] == 0)


@pytest.mark.parametrize("fmt,dim,group", [("e4m3", 128, 5), ("e4m3", 64, 1), ("e5m2", 128, 8), ("e5m2", 64, 3), ("e4m3", 128, 1)])
def test_prefill_against_the_oracle(fmt, dim, group):
    lens = [0, 1, 3, 17, 64, 130, 300, 700, 1000, 40]
    q_lens = [0, 1, 2, 17, 1, 130, 45, 600, 256, 0]
    for n, (window, sinks) in enumerate(WINDOWS):
        w, cache, kv, table = make(lens, q_lens, group * 2, 2, dim, fmt, window, sinks, seed=200 + n)
        out = prefill(w, cache, table, window, sinks, extra_rows=3)
        ref, spread = attention.window_attention(w.q.float().numpy(), kv, w.block_table.numpy(), lens, window, sinks, w.cu_q_lens.numpy())
        check(out, ref, spread, fmt, prefill=True, vmax=6.0, what=f"window {window} sinks {sinks}")


def test_prefill_of_one_token_each_and_of_runs_longer_than_their_context():
    lens = [5, 600, 33]
    w, cache, kv, table = make(lens, [1, 1, 1], 8, 2, 128, "e4m3", 40, 4, seed=7)
    ref, spread = attention.window_attention(w.q.float().numpy(), kv, w.block_table.numpy(), lens, 40, 4)
    check(prefill(w, cache, table, 40, 4), ref, spread, "e4m3", prefill=True, vmax=6.0)
    w, cache, kv, table = make([5, 20], [9, 30], 8, 2, 64, "e4m3", 3, 1, seed=8, poison=False)
    out = prefill(w, cache, w.block_table, 3, 1)
    ref, spread = attention.window_attention(w.q.float().numpy(), kv, w.block_table.numpy(), [5, 20], 3, 1, w.cu_q_lens.numpy())
    check(out, ref, spread, "e4m3", prefill=True, vmax=6.0)
    assert torch.all(out[:4] == 0) and torch.all(out[9:19] == 0)


@pytest.mark.parametrize("lens,hq,hkv,dim,window,sinks", [([9000], 8, 1, 128, 8000, 4), ([70000, 200, 30011], 10, 2, 128, 5000, 40), ([4000] * 40, 8, 2, 64, 1111, 3)])
def test_long_windows_are_cut_and_joined(lens, hq, hkv, dim, window, sinks):
    w, cache, kv, table = make(lens, [1] * len(lens), hq, hkv, dim, "e4m3", window, sinks, seed=11)
    out = decode(w, cache, table, lens, window, sinks)
    ref, spread = attention.window_attention(w.q.float().numpy(), kv, w.block_table.numpy(), lens, window, sinks)
    check(out, ref, spread, "e4m3")
    assert torch.equal(out, decode(w, cache, table, lens, window, sinks))


def test_many_sequences():
    lens = [1 + (37 * b) % 400 for b in range(512)]
    w, cache, kv, table = make(lens, [1] * 512, 4, 1, 64, "e5m2", 90, 18, seed=13)
    ref, spread = attention.window_attention(w.q.float().numpy(), kv, w.block_table.numpy(), lens, 90, 18)
    check(decode(w, cache, table, lens, 90, 18), ref, spread, "e5m2")


@pytest.mark.parametrize("fmt", ["e4m3", "e5m2", "bf16"])
def test_a_window_over_everything_is_the_call_without_one(fmt):
    # (both calls are held to the definition: what is joined in which order is each one's own)
    lens = [700, 1, 0, 33, 2000, 129]
    w, cache, kv, table = make(lens, [1] * 6, 10, 2, 128, fmt, 2000, 0, seed=17, poison=False)
    ref, spread = attention.window_attention(w.q.float().numpy(), kv, w.block_table.numpy(), lens, 2000, 0)
    whole, _ = helpers.gpu_decode(w, cache)
    for out in (whole, decode(w, cache, w.block_table, lens, 2000, 0)):
        check(out, ref, spread, fmt)
    if fmt != "bf16":
        lens, q_lens = [700, 33, 300], [500, 2, 40]
        w, cache, kv, table = make(lens, q_lens, 10, 2, 128, fmt, 700, 0, seed=18, poison=False)
        ref, spread = attention.window_attention(w.q.float().numpy(), kv, w.block_table.numpy(), lens, 700, 0, w.cu_q_lens.numpy())
        ws = binding.new_workspace(3, 10, 2, 128, w.block_table.shape[1], 512, 542)
        whole = binding.paged_chunked(cache, w.q.cuda(), w.cu_q_lens.cuda(), w.block_table.cuda(), w.context_lens_tensor.cuda(), 512, True, w.sm_scale, ws)
        for out in (whole, prefill(w, cache, w.block_table, 700, 0)):
            check(out, ref, spread, fmt, prefill=True, vmax=6.0)


@pytest.mark.parametrize("fmt,dim", [("e4m3", 128), ("e5m2", 64), ("bf16", 64)])
def test_new_tokens_are_written_and_seen(fmt, dim):
    """Step after step over a sliding window: the cache's bytes are those of the write rule, the output is that of the call
    over the written cache, and what has left the window is taken out of the table as it goes.  K and V are slices of one wider
    projection."""
    lens0, window, sinks, steps, hkv, hq = [14, 30, 100, 0, 257], 33, 5, 20, 2, 6
    B = len(lens0)
    w = workloads.make_workload("steps", [L + steps for L in lens0], hq, hkv, dim, seed=19)
    width = w.block_table.shape[1]
    cache = binding.Cache(w.num_blocks, hkv, dim, FMT[fmt])
    kind = {"e4m3": e4m3, "e5m2": e5m2}.get(fmt)
    codes, scales = kv_cache.new_cache(w.num_blocks, hkv, dim)
    values = kv_cache.new_cache_bf16(w.num_blocks, hkv, dim)

    def oracle_write(rows, slots, **more):
        k, v, slots = w.k[rows].float().numpy(), w.v[rows].float().numpy(), slots.numpy()
        if fmt == "bf16":
            kv_cache.kv_write_bf16(values, k, v, slots)
        else:
            kv_cache.kv_write(codes, scales, k, v, slots, fmt=kind, **more)

    for b, L in enumerate(lens0):
        if L:
            rows = slice(w.kv_offsets[b], w.kv_offsets[b] + L)
            binding.kv_write(cache, w.k[rows].cuda(), w.v[rows].cuda(), w.slot_mapping[rows].cuda())
            oracle_write(rows, w.slot_mapping[rows])
    ws, ws2 = (binding.new_workspace(B, hq, hkv, dim, width) for _ in range(2))
    table = w.block_table.cuda()
    for s in range(steps):
        lens = [L + s + 1 for L in lens0]
        for b, L in enumerate(lens):
            gone = max(0, L - window) // 16
            if gone > 1:
                table[b, 1:gone] = -1
        rows = torch.tensor([w.kv_offsets[b] + lens[b] - 1 for b in range(B)])
        wide = torch.zeros(B, 3 * hkv, dim, dtype=torch.bfloat16)
        wide[:, hkv:2 * hkv], wide[:, 2 * hkv:] = w.k[rows], w.v[rows]
        wide = wide.cuda()
        k, v, slots = wide[:, hkv:2 * hkv], wide[:, 2 * hkv:], w.slot_mapping[rows].clone()
        if s == 7:
            slots[2] = -1                                   # a token that is not stored
        oracle_write(rows, slots, **({} if fmt == "bf16" else {"reciprocal": True}))
        slots, q = slots.cuda(), torch.randn(B, hq, dim).to(torch.bfloat16).cuda()
        lens_t = torch.tensor(lens, dtype=torch.int32).cuda()
        out = binding.window_decode(cache, q, table, lens_t, window, sinks, w.sm_scale, ws, k, v, slots)
        want = binding.window_decode(cache, q, table, lens_t, window, sinks, w.sm_scale, ws2)
        torch.cuda.synchronize()
        assert binding.workspace_status(ws) == 0 and binding.workspace_status(ws2) == 0
        if fmt == "bf16":
            assert np.array_equal(helpers.cache_to_logical(cache), values), f"step {s}"
        else:
            helpers.check_cache_bit_exact(cache, codes, scales, what=f"step {s}")
        assert torch.equal(out, want), f"step {s}"


def test_blocks_far_into_a_large_cache():
    """Byte offsets past 32 bits."""
    hkv, dim, blocks, lens = 8, 128, 140000, [100, 700]
    w = workloads.make_workload("far", lens, 16, hkv, dim, seed=23, q_lens=[1, 1], outliers=False)
    shift = blocks - w.num_blocks
    w.num_blocks = blocks
    w.slot_mapping += shift * 16
    w.block_table[w.block_table >= 0] += shift
    cache = binding.Cache(blocks, hkv, dim)
    assert cache.data.numel() > 2 ** 32
    binding.kv_write(cache, w.k.cuda(), w.v.cuda(), w.slot_mapping.cuda())
    small = binding.Cache(w.num_blocks - shift, hkv, dim)
    binding.kv_write(small, w.k.cuda(), w.v.cuda(), (w.slot_mapping - shift * 16).cuda())
    low = w.block_table.clone()
    low[low >= 0] -= shift
    assert torch.equal(decode(w, cache, w.block_table, lens, 300, 4), decode(w, small, low, lens, 300, 4))
    assert torch.equal(prefill(w, cache, w.block_table, 300, 4), prefill(w, small, low, 300, 4))


def test_other_streams_and_replayed_graphs_that_share_a_workspace():
    lens = [900, 40, 2222]
    w, cache, kv, table = make(lens, [1] * 3, 8, 2, 128, "e4m3", 600, 4, seed=29)
    want = decode(w, cache, table, lens, 600, 4)
    q, table_d, lens_t = w.q.cuda(), table.cuda(), torch.tensor(lens, dtype=torch.int32).cuda()
    cu = torch.arange(4, dtype=torch.int32).cuda()
    ws = binding.new_workspace(3, 8, 2, 128, table.shape[1])
    want_p = binding.window_prefill(cache, q, cu, table_d, lens_t, 600, 4, w.sm_scale, ws)
    torch.cuda.synchronize()
    graphs, outs = [], []
    side = torch.cuda.Stream()
    for kind in range(2):
        out = torch.zeros_like(q)
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            binding.window_decode(cache, q, table_d, lens_t, 600, 4, w.sm_scale, ws, out=out)
        side.synchronize()
        assert torch.equal(out, want)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            if kind == 0:
                binding.window_decode(cache, q, table_d, lens_t, 600, 4, w.sm_scale, ws, out=out)
            else:
                binding.window_prefill(cache, q, cu, table_d, lens_t, 600, 4, w.sm_scale, ws, out=out)
        graphs.append(g)
        outs.append(out)
    for _ in range(3):
        for out in outs:
            out.zero_()
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        assert torch.equal(outs[0], want) and torch.equal(outs[1], want_p)
    assert binding.workspace_status(ws) == 0


def test_bad_entries_are_reported_where_they_are_looked_at():
    lens = [100, 300]
    w, cache, kv, table = make(lens, [1, 1], 4, 2, 128, "e4m3", 50, 4, seed=31)
    want = decode(w, cache, table, lens, 50, 4)
    bad = table.clone()
    bad[1, 2:15] = 10 ** 6                                # between sinks and window: never read
    assert torch.equal(decode(w, cache, bad, lens, 50, 4), want)
    bad[1, 17] = 10 ** 6
    for call in ("decode", "prefill"):
        ws = binding.new_workspace(2, 4, 2, 128, table.shape[1])
        args = (bad.cuda(), torch.tensor(lens, dtype=torch.int32).cuda(), 50, 4, w.sm_scale, ws)
        if call == "decode":
            binding.window_decode(cache, w.q.cuda(), *args)
        else:
            binding.window_prefill(cache, w.q.cuda(), torch.arange(3, dtype=torch.int32).cuda(), *args)
        torch.cuda.synchronize()
        assert binding.workspace_status(ws) == -1, call
    # a token that is not its sequence's last position
    ws = binding.new_workspace(2, 4, 2, 128, table.shape[1])
    new = torch.zeros(2, 2, 128, dtype=torch.bfloat16).cuda()
    binding.window_decode(cache, w.q.cuda(), table.cuda(), torch.tensor(lens, dtype=torch.int32).cuda(), 50, 4, w.sm_scale, ws, new, new,
                          torch.tensor([5, 6]).cuda())
    torch.cuda.synchronize()
    assert binding.workspace_status(ws) == -1


def test_what_the_binding_refuses():
    w, cache, kv, table = make([40], [1], 4, 2, 128, "e4m3", 9, 1, seed=37)
    ws = binding.new_workspace(1, 4, 2, 128, table.shape[1])
    q, t, n = w.q.cuda(), table.cuda(), torch.tensor([40], dtype=torch.int32).cuda()
    for bad in ((w.q, t, n), (q, table, n), (q.float(), t, n), (q, t.long(), n), (q[:, :, :64], t, n), (q, t, n.repeat(2)), (q.repeat(2, 1, 1), t, n)):
        with pytest.raises(ValueError):
            binding.window_decode(cache, *bad, 9, 1, w.sm_scale, ws)
    with pytest.raises(ValueError):
        binding.window_decode(cache, q, t, n, 9, 1, w.sm_scale, ws, k_new=q[:, :2])
    with pytest.raises(ValueError):
        binding.window_prefill(cache, q, torch.arange(3, dtype=torch.int32).cuda(), t, n, 9, 1, w.sm_scale, ws)
    with pytest.raises(ValueError):
        binding.window_decode(cache, q, t, n, 2 ** 32 + 9, 1, w.sm_scale, ws)
    for window, sinks in ((0, 1), (-1, 0), (5, -1)):
        with pytest.raises(binding.CooptError):
            binding.window_decode(cache, q, t, n, window, sinks, w.sm_scale, ws)
    with pytest.raises(binding.CooptError):
        binding.window_decode(cache, q, t, n, 9, 1, w.sm_scale, ws[:1000])


def test_two_streams_at_once():
    """Calls that overlap on the device, each with a workspace of its own."""
    lens = [2500, 4, 900, 1300, 77, 3000]
    w, cache, kv, table = make(lens, [1] * 6, 16, 4, 64, "e4m3", 1000, 4, seed=43)
    want = decode(w, cache, table, lens, 1000, 4)
    q, t, n = w.q.cuda(), table.cuda(), torch.tensor(lens, dtype=torch.int32).cuda()
    cu = torch.arange(7, dtype=torch.int32).cuda()
    streams = [torch.cuda.Stream() for _ in range(3)]
    spaces = [binding.new_workspace(6, 16, 4, 64, table.shape[1]) for _ in streams]
    outs = [[torch.zeros_like(q) for _ in range(20)] for _ in streams]
    torch.cuda.synchronize()
    for turn in range(20):
        for k, (stream, ws) in enumerate(zip(streams, spaces)):
            with torch.cuda.stream(stream):
                if k < 2:
                    binding.window_decode(cache, q, t, n, 1000, 4, w.sm_scale, ws, out=outs[k][turn])
                else:
                    binding.window_prefill(cache, q, cu, t, n, 1000, 4, w.sm_scale, ws, out=outs[k][turn])
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for k in range(2) for o in outs[k])
    assert all(torch.equal(o, outs[2][0]) for o in outs[2])
    ref, spread = attention.window_attention(w.q.float().numpy(), kv, w.block_table.numpy(), lens, 1000, 4)
    check(outs[2][0], ref, spread, "e4m3", prefill=True, vmax=6.0)


@pytest.mark.parametrize("batch,hkv,window", [(1, 1, 3000), (3, 8, 200), (19, 8, 700), (33, 8, 900), (52, 8, 500), (60, 8, 400), (150, 1, 1100), (301, 1, 350)])
def test_every_way_of_sharing_out_the_work(batch, hkv, window):
    """From a cluster to a unit over one, two and three CTAs on an SM to the line, with contexts of all lengths beside each other."""
    lens = [(b * 7919) % (2 * window) for b in range(batch)]
    lens[0] = 2 * window + 1
    for fmt, dim in (("e4m3", 128), ("bf16", 64)):
        w, cache, kv, table = make(lens, [1] * batch, 2 * hkv, hkv, dim, fmt, window, 9, seed=47 + batch)
        ref, spread = attention.window_attention(w.q.float().numpy(), kv, w.block_table.numpy(), lens, window, 9)
        check(decode(w, cache, table, lens, window, 9), ref, spread, fmt, what=f"{fmt} {batch}")


@pytest.mark.parametrize("group,hkv,batch,most,context,window,sinks", [(1, 8, 12, 300, 3000, 40, 4), (5, 8, 9, 130, 2000, 300, 0), (8, 8, 40, 40, 500, 100, 20),
                                                                     (4, 4, 3, 1500, 1500, 200, 3), (2, 8, 20, 64, 4000, 1000, 1)])
def test_prefill_of_several_rounds(group, hkv, batch, most, context, window, sinks):
    """More pieces of work than the device takes at a time: which goes where, and in what order, is worked out on the device."""
    rng = np.random.default_rng(batch)
    q_lens = [int(x) for x in rng.integers(0, most + 1, batch)]
    q_lens[0], q_lens[-1] = most, 128 // group                # a whole tile
    lens = [n + int(x) for n, x in zip(q_lens, rng.integers(0, max(1, context - most), batch))]
    w, cache, kv, table = make(lens, q_lens, group * hkv, hkv, 64, "e4m3", window, sinks, seed=61 + batch)
    out = prefill(w, cache, table, window, sinks, extra_rows=2)
    ref, spread = attention.window_attention(w.q.float().numpy(), kv, w.block_table.numpy(), lens, window, sinks, w.cu_q_lens.numpy())
    check(out, ref, spread, "e4m3", prefill=True, vmax=6.0)


@pytest.mark.parametrize("batch,hkv,most,window,fmt,dim", [(1, 2, 6, 500, "e4m3", 128), (4, 8, 3, 900, "e5m2", 128), (12, 8, 5, 300, "e4m3", 64), (20, 4, 6, 200, "e5m2", 64),
                                                           (150, 1, 3, 100, "e4m3", 128), (40, 8, 2, 120, "e4m3", 128), (400, 1, 1, 60, "e4m3", 64), (3, 1, 60, 40, "e5m2", 128)])
def test_prefill_of_short_runs(batch, hkv, most, window, fmt, dim):
    """A few new tokens a sequence (drafts to verify, tails of prompts), from one run to hundreds, empty ones and ones longer than
    their context among them."""
    rng = np.random.default_rng(batch + most)
    q_lens = [int(x) for x in rng.integers(0, most + 1, batch)]
    q_lens[-1] = most
    lens = [max(0, n + int(x)) for n, x in zip(q_lens, rng.integers(-1, 2 * window, batch))]
    lens[0] = 2 * window + 37
    w, cache, kv, table = make(lens, q_lens, 3 * hkv, hkv, dim, fmt, window, 5, seed=71 + batch)
    out = prefill(w, cache, table, window, 5, extra_rows=3)
    ref, spread = attention.window_attention(w.q.float().numpy(), kv, w.block_table.numpy(), lens, window, 5, w.cu_q_lens.numpy())
    check(out, ref, spread, fmt, prefill=True, vmax=6.0)


@pytest.mark.parametrize("lens,q_lens", [([403, 64], [4, 3]), ([403, 64], [40, 30]), ([3000, 64], [200, 3]), ([700, 90] * 80, [30, 9] * 80)])
def test_a_key_that_is_nan_reaches_those_who_see_it_and_no_one_else(lens, q_lens):
    """The last token's key of kv head 0, in each of the ways that a run is served."""
    w, cache, kv, table = make(lens, q_lens, 10, 2, 128, "e4m3", 200, 3, seed=73)
    before = prefill(w, cache, table, 200, 3)
    spoil_last_key(w, cache, table, lens)
    after = prefill(w, cache, table, 200, 3)
    last = torch.zeros(len(before), dtype=torch.bool)
    last[w.cu_q_lens[1:].long() - 1] = True
    assert torch.isnan(after[last][:, :5].float()).all()
    assert torch.equal(before[~last], after[~last]) and torch.equal(before[:, 5:], after[:, 5:])


@pytest.mark.parametrize("fmt", ["e4m3", "bf16"])
@pytest.mark.parametrize("lens", [[17], [2000], [350, 900] * 10, [40, 900] * 25, [350, 900, 3] * 40])
def test_a_token_whose_key_is_nan_makes_the_output_nan(lens, fmt):
    w, cache, kv, table = make(lens, [1] * len(lens), 10, 2, 128, fmt, 800, 3, seed=79)
    before = decode(w, cache, table, lens, 800, 3)
    spoil_last_key(w, cache, table, lens)
    after = decode(w, cache, table, lens, 800, 3)
    assert torch.isnan(after[:, :5].float()).all() and torch.equal(before[:, 5:], after[:, 5:])


def spoil_last_key(w, cache, table, lens):
    raw = cache.data.view(w.num_blocks, w.num_kv_heads, cache.granule_bytes)
    idx = torch.from_numpy(helpers.granule_index_map(cache))
    for b, L in enumerate(lens):
        at = idx[0, (L - 1) % 16].cuda()
        for byte in range(1 if cache.dtype != FMT["bf16"] else 2):
            raw[int(table[b, (L - 1) // 16]), 0, at + byte] = 0x7F if cache.dtype != FMT["bf16"] or byte == 1 else 0xC0


@pytest.mark.parametrize("fmt,group,hkv,most,window", [("e4m3", 4, 8, 32, 500), ("e5m2", 1, 8, 128, 100), ("e4m3", 8, 4, 16, 2000), ("e5m2", 3, 8, 42, 1)])
def test_prefill_of_many_runs_that_fit_a_tile(fmt, group, hkv, most, window):
    """More tiles than SMs, most of them of a sequence each; one run needs several, one is empty, one has nothing to see."""
    rng = np.random.default_rng(most)
    q_lens = [int(x) for x in rng.integers(1, most + 1, 40)]
    q_lens[3], q_lens[7], q_lens[9] = 0, most + most // 2, most
    lens = [n + int(x) for n, x in zip(q_lens, rng.integers(0, 3 * window + 60, 40))]
    lens[9] = 0
    w, cache, kv, table = make(lens, q_lens, group * hkv, hkv, 64, fmt, window, 6, seed=83 + most)
    out = prefill(w, cache, table, window, 6, extra_rows=2)
    ref, spread = attention.window_attention(w.q.float().numpy(), kv, w.block_table.numpy(), lens, window, 6, w.cu_q_lens.numpy())
    check(out, ref, spread, fmt, prefill=True, vmax=6.0)


@pytest.mark.parametrize("fmt,dim", [("bf16", 64), ("bf16", 128), ("e5m2", 64), ("e5m2", 128)])
def test_a_key_of_minus_infinity_has_no_weight(fmt, dim):
    """The first token, alone in its block, with logits of -inf: as if there were no sink."""
    lens = [400, 1000, 40, 17] * 3
    w, cache, kv, table = make(lens, [1] * len(lens), 2, 2, dim, fmt, 5, 1, seed=89)
    raw = cache.data.view(w.num_blocks, 2, cache.granule_bytes)
    idx = torch.from_numpy(helpers.granule_index_map(cache))
    for b in range(len(lens)):
        for h in range(2):
            high = 0xFF if float(w.q[b, h, 0]) > 0 else 0x7F
            at = int(idx[0, 0, 0])
            if fmt == "bf16":
                raw[int(table[b, 0]), h, at], raw[int(table[b, 0]), h, at + 1] = 0x80, high
            else:
                raw[int(table[b, 0]), h, at] = high & 0xFC
    ref, spread = attention.window_attention(w.q.float().numpy(), kv, w.block_table.numpy(), lens, 5, 0)
    check(decode(w, cache, table, lens, 5, 1), ref, spread, fmt)
    if fmt == "e5m2":
        check(prefill(w, cache, table, 5, 1), ref, spread, fmt, prefill=True, vmax=6.0)
