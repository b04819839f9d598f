"""Pages of a cache on the device against the oracle's pool: every count, entry, length and byte."""
import numpy as np
import pytest
import torch

from oracle import attention, pages as oracle_pages
from paper_2602_09323_b200 import binding, workloads

pytestmark = pytest.mark.gpu


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Both:
    """The same pool on the device and in the oracle, with caches of random bytes."""

    def __init__(self, num_blocks, rows, width, layers=2, hkv=2, dim=64, dtype=binding.KV_FP8_E4M3, seed=0):
        gen = torch.Generator().manual_seed(seed)
        self.caches = [binding.Cache(num_blocks, hkv, dim, dtype) for _ in range(layers)]
        for c in self.caches:
            c.data.copy_(torch.randint(0, 256, (c.data.numel(),), dtype=torch.uint8, generator=gen))
        self.gran = self.caches[0].granule_bytes if layers else 0
        self.used = 32 * dim + 32 if dtype != binding.KV_BF16 else self.gran
        self.shape = (num_blocks, hkv, self.gran)
        self.set = binding.CacheSet(self.caches)
        self.pages = binding.Pages.empty(num_blocks, rows, width)
        self.ws = binding.new_pages_workspace(num_blocks, rows)
        self.ref = oracle_pages.Pool(num_blocks, rows, width, self.bytes())
        self.padding = self.pads()

    def bytes(self):
        got = [c.data.cpu().numpy().reshape(self.shape)[:, :, :self.used] for c in self.caches]
        return np.stack(got) if got else np.zeros((0, *self.shape[:2], 0))

    def pads(self):
        return [c.data.cpu().numpy().reshape(self.shape)[:, :, self.used:].copy() for c in self.caches]

    def check(self, what=""):
        torch.cuda.synchronize()
        assert np.array_equal(self.pages.refs.cpu().numpy(), self.ref.refs), what
        assert np.array_equal(self.pages.block_table.cpu().numpy(), self.ref.table), what
        assert np.array_equal(self.pages.context_lens.cpu().numpy(), self.ref.lens), what
        assert np.array_equal(self.bytes(), self.ref.contents), what
        assert all(np.array_equal(a, b) for a, b in zip(self.pads(), self.padding)), f"{what}: padding was written"
        status = binding.workspace_status(self.ws)
        want = {frozenset(): (0,), frozenset(["invalid"]): (-1,), frozenset(["pages"]): (-6,)}.get(frozenset(self.ref.problems), (-1, -6))
        assert status in want, (what, status, self.ref.problems)
        if status:
            binding.workspace_init(self.ws)
            self.ref.problems.clear()

    def reserve(self, rows, lens):
        binding.pages_reserve(self.pages, ints(rows), ints(lens), self.ws)
        self.ref.reserve(rows, lens)

    def fork(self, parents, children):
        binding.pages_fork(self.set, self.pages, ints(parents), ints(children), self.ws)
        self.ref.fork(parents, children)

    def release(self, rows, window=0, sinks=0):
        binding.pages_release(self.pages, ints(rows), self.ws, window, sinks)
        self.ref.release(rows, window, sinks)

    def compact(self):
        used = binding.pages_compact(self.set, self.pages, self.ws)
        assert int(used.item()) == self.ref.compact()


@pytest.mark.parametrize("dtype,dim,hkv,layers,blocks,steps", [(binding.KV_FP8_E4M3, 64, 2, 2, 67, 60), (binding.KV_FP8_E5M2, 128, 1, 3, 67, 60),
                                                               (binding.KV_BF16, 64, 3, 1, 67, 60), (binding.KV_BF16, 128, 2, 2, 67, 60),
                                                               (binding.KV_FP8_E4M3, 128, 5, 1, 67, 60), (binding.KV_FP8_E4M3, 64, 1, 1, 33000, 20),
                                                               (binding.KV_FP8_E4M3, 64, 1, 67, 67, 30)])
def test_a_run_of_calls(dtype, dim, hkv, layers, blocks, steps):
    rng = np.random.default_rng(dim + hkv)
    p = Both(blocks, 14, 9, layers, hkv, dim, dtype, seed=1)
    if blocks > 1000:                                     # most of a large pool is held by others, the lowest free blocks lie far up
        p.ref.refs[:blocks - 80] = 1
        p.ref.refs[rng.choice(blocks, 30, replace=False)] = 0
        p.pages.refs.copy_(torch.from_numpy(p.ref.refs))
    for step in range(steps):
        kind = rng.choice(["reserve", "fork", "release", "trim", "compact"], p=[0.4, 0.25, 0.15, 0.12, 0.08])
        n = int(rng.integers(1, 6))
        if kind == "reserve":
            rows = rng.choice(14, n, replace=False)
            p.reserve(rows.tolist(), [int(min(144, p.ref.lens[r] + rng.integers(0, 40))) for r in rows])
        elif kind == "fork":
            empty = np.nonzero(p.ref.lens == 0)[0]
            children = rng.permutation(empty)[:n]
            parents = [r for r in range(14) if r not in set(children.tolist())]
            p.fork([int(rng.choice(parents)) for _ in children], children.tolist())
        elif kind == "release":
            p.release(rng.choice(14, min(n, 3), replace=False).tolist())
        elif kind == "trim":
            p.release(rng.choice(14, n, replace=False).tolist(), int(rng.integers(1, 60)), int(rng.integers(0, 20)))
        else:
            p.compact()
        p.check(f"step {step}: {kind}")


def test_reserve_serves_the_list_in_order_and_reports_what_it_cannot():
    p = Both(20, 6, 40, layers=0)
    p.reserve([4, 0, 2], [33, 0, 16])
    p.check("three rows")
    p.reserve([1, 3, 4, 5], [160, 100, 34, 16])           # 10 of 16, then 7 more than are left, nothing needed, and one that is behind
    p.check("too few")
    assert p.ref.lens.tolist() == [0, 160, 16, 0, 34, 0]
    p.reserve([3], [96])
    p.check("the last ones")
    p.reserve([3], [97])
    p.check("none left")
    p.reserve([2, 2, -1, 6, 4, 1], [16, 16, 1, 1, 33, 641])   # again, out of range, shorter, beyond the table
    p.check("refused")


def test_fork_shares_copies_and_refuses():
    p = Both(30, 10, 8, seed=3)
    p.reserve([0, 1, 2], [40, 32, 5])
    p.release([0], 9, 2)                                  # keeps the sinks' block and the window's
    p.fork([0, 1, 0, 2, 7], [3, 4, 5, 6, 8])              # partly filled, whole blocks, twice, short, empty
    p.check("forks")
    p.fork([0, 0, 1, 9, -1, 0, 2], [3, 9, 9, 7, 7, 10, 2])   # not empty; fine; a second mention; a child as parent; rows out of range; itself
    p.check("refused")
    p.reserve([1], [128])
    p.reserve([4], [16 * int(np.sum(p.ref.refs == 0)) + 32])
    p.check("full")
    p.fork([0, 1, 2], [7, 8, 9])                          # no block for a copy; whole blocks need none
    p.check("no blocks")


def test_a_row_named_twice_is_released_once():
    p = Both(12, 4, 5, layers=1)
    p.reserve([0, 1], [60, 20])
    p.fork([0], [2])
    p.release([0, 0, 2, 5, -3])
    p.check("twice, and rows that are none")
    p.pages.block_table[1, 0] = 11                        # an entry that no count stands for, and one of no pool
    p.pages.block_table[1, 1] = 12
    p.ref.table[1, 0] = 11
    binding.pages_release(p.pages, ints([1]), p.ws)
    torch.cuda.synchronize()
    assert binding.workspace_status(p.ws) == -1 and int(p.pages.refs.min()) == 0 and int(p.pages.block_table.max()) == -1


@pytest.mark.parametrize("num_blocks,used", [(1, 1), (1, 0), (33, 33), (33, 0), (1000, 1), (4097, 2000), (100000, 37777)])
def test_compaction_of_pools_of_any_size(num_blocks, used):
    rng = np.random.default_rng(num_blocks)
    width = max(1, -(-used // 7))
    p = Both(num_blocks, 7, width, layers=1 if num_blocks < 5000 else 0, hkv=1)
    place = rng.choice(num_blocks, used, replace=False)
    table = np.full(7 * width, -1, dtype=np.int32)
    table[rng.choice(7 * width, used, replace=False)] = place
    p.ref.table[:] = table.reshape(7, width)
    p.ref.refs[place] = rng.integers(1, 5, used)
    p.pages.block_table.copy_(torch.from_numpy(p.ref.table))
    p.pages.refs.copy_(torch.from_numpy(p.ref.refs))
    table_out, refs_out = torch.full_like(p.pages.block_table, 99), torch.full_like(p.pages.refs, 99)
    new_ids = torch.full_like(refs_out, 99)
    old_table, old_refs = p.ref.table.copy(), p.ref.refs.copy()
    count = binding.pages_compact(p.set, p.pages, p.ws, table_out, refs_out, new_ids=new_ids)
    assert np.array_equal(p.pages.refs.cpu().numpy(), p.ref.refs) and np.array_equal(p.pages.block_table.cpu().numpy(), p.ref.table)
    assert p.ref.compact() == int(count.item()) == used
    assert np.array_equal(table_out.cpu().numpy(), p.ref.table) and np.array_equal(refs_out.cpu().numpy(), p.ref.refs)
    ids = new_ids.cpu().numpy()
    assert np.array_equal(ids >= 0, old_refs > 0) and np.array_equal(ids[old_table[old_table >= 0]], p.ref.table[p.ref.table >= 0])
    p.pages.refs.copy_(refs_out), p.pages.block_table.copy_(table_out)
    p.check("apart")
    p.compact()                                           # and once more, in place: nothing moves
    p.check("again")
    p.reserve([0, 3], [int(x) for x in (min(16 * width, 40), min(16 * width, 33))])
    p.check("reserve")


def test_entries_of_free_blocks_are_taken_out_and_reported():
    p = Both(10, 2, 4, layers=1)
    p.reserve([0], [64])
    p.pages.block_table[1, 0], p.pages.block_table[1, 1] = 7, 10
    p.ref.table[1, 0], p.ref.table[1, 1] = 7, 10
    p.compact()
    p.check("stale entries")


@pytest.mark.parametrize("layers,hkv,dim,dtype", [(1, 1, 64, binding.KV_FP8_E4M3), (70, 1, 64, binding.KV_FP8_E4M3), (3, 8, 128, binding.KV_BF16), (2, 5, 128, binding.KV_FP8_E5M2)])
def test_copy(layers, hkv, dim, dtype):
    p = Both(50, 1, 1, layers, hkv, dim, dtype, seed=5)
    src, dst = [3, 49, 0, 7, -1, 50, 3, 12], [1, 2, 48, 9, 4, 5, 6, 51]       # the same source twice, ids of no block
    binding.pages_copy(p.set, ints(src), ints(dst))
    p.ref.copy(src, dst)
    p.check("copies")
    binding.pages_copy(p.set, ints([]), ints([]))
    p.check("none")


def test_copy_far_into_a_large_cache():
    cache = binding.Cache(140000, 8, 128)
    assert cache.data.numel() > 2 ** 32
    raw = cache.data.view(140000, 8, -1)
    raw[5] = torch.randint(0, 256, raw[5].shape, dtype=torch.uint8, device="cuda")
    one = binding.CacheSet([cache])
    binding.pages_copy(one, ints([5]), ints([139999]))
    binding.pages_copy(one, ints([139999]), ints([130000]))
    torch.cuda.synchronize()
    used = 32 * 128 + 32
    for b in (139999, 130000):
        assert torch.equal(raw[b, :, :used], raw[5, :, :used]) and not raw[b, :, used:].any()
    assert not raw[139998].any() and not raw[130001].any()


def test_many_rows_and_a_large_pool():
    rows, blocks = 2000, 90000
    p = Both(blocks, rows, 50, layers=0)
    rng = np.random.default_rng(2)
    order = rng.permutation(1200)
    p.reserve(order.tolist(), rng.integers(0, 800, 1200).tolist())
    p.check("reserve")
    p.fork(rng.integers(0, 1200, 700).tolist(), (1200 + rng.permutation(800)[:700]).tolist())
    p.check("fork")
    p.release(rng.permutation(rows)[:900].tolist())
    p.check("release")
    p.compact()
    p.check("compact")


def test_calls_are_captured_and_replayed():
    p = Both(40, 6, 6, layers=2, seed=9)
    p.reserve([0], [37])
    p.check("before")
    kids, parents, grown = ints([2, 3]), ints([0, 0]), ints([50, 37])
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        binding.pages_release(p.pages, kids, p.ws)
        binding.pages_fork(p.set, p.pages, parents, kids, p.ws)
        binding.pages_reserve(p.pages, kids, grown, p.ws)
    for turn in range(3):
        if turn:
            p.ref.release([2, 3])
        p.ref.fork([0, 0], [2, 3])
        p.ref.reserve([2, 3], [50, 37])
        g.replay()
        p.check(f"turn {turn}")


def test_a_server_that_streams_branches_and_compacts():
    """The calls together as they are used: room reserved, tokens written, window attention, blocks behind the window given
    back, branches, a compaction; every output against the oracle over each sequence's own tokens."""
    hq, hkv, dim, window, sinks, width, blocks, rows, layers = 6, 2, 64, 40, 4, 40, 60, 6, 2
    gen = torch.Generator().manual_seed(41)
    pool, caches = binding.Pages.empty(blocks, rows, width), [binding.Cache(blocks, hkv, dim, binding.KV_BF16) for _ in range(layers)]
    cset, pws = binding.CacheSet(caches), binding.new_pages_workspace(blocks, rows)
    ws = binding.new_workspace(rows, hq, hkv, dim, width)
    said = [[[], []] for _ in range(rows)]                 # each row's K, V of all layers: [layers, hkv, dim] a token
    lens = [0] * rows

    def write(row, n):
        kv = torch.randn(2, n, layers, hkv, dim, generator=gen).to(torch.bfloat16)
        for w in range(2):
            said[row][w] = said[row][w] + list(kv[w])
        pos = torch.arange(lens[row] - n, lens[row]).cuda()
        slots = pool.block_table[row, pos // 16].long() * 16 + pos % 16
        for y in range(layers):
            binding.kv_write(caches[y], kv[0, :, y].contiguous().cuda(), kv[1, :, y].contiguous().cuda(), slots)

    def attend(active):
        lens_t = torch.zeros(rows, dtype=torch.int32)
        lens_t[active] = torch.tensor([lens[r] for r in active], dtype=torch.int32)
        q = torch.randn(rows, hq, dim, generator=gen).to(torch.bfloat16)
        for y in range(layers):
            out = binding.window_decode(caches[y], q.cuda(), pool.block_table, lens_t.cuda(), window, sinks, dim ** -0.5, ws).double().cpu().numpy()
            for r in active:
                # the sequence's own tokens as a cache of its own
                n = -(-lens[r] // 16)
                kv = np.zeros((n, hkv, 2, 16, dim))
                for w in range(2):
                    x = torch.stack(said[r][w])[:, y].double().numpy()
                    for t in range(lens[r]):
                        kv[t // 16, :, w, t % 16] = x[t]
                ref, spread = attention.window_attention(q[r:r + 1].float().numpy(), kv, np.arange(n)[None], [lens[r]], window, sinks)
                assert np.all(np.abs(out[r] - ref[0]) <= 2.0 ** -8 * np.abs(ref[0]) + 2.0 ** -11 * spread[0] + 2.0 ** -30), (r, lens[r], y)

    def reserve(active, more):
        for r, n in zip(active, more):
            lens[r] += n
        binding.pages_reserve(pool, ints(active), ints([lens[r] for r in active]), pws)
        for r, n in zip(active, more):
            write(r, n)

    reserve([0, 3], [70, 21])
    attend([0, 3])
    for turn in range(60):
        active = [r for r in range(rows) if lens[r]]
        reserve(active, [1 + (turn + r) % 4 for r in active])
        attend(active)
        binding.pages_release(pool, ints(active), pws, window, sinks)
        if turn in (5, 23, 41):
            old = [r for r in (1, 2) if lens[r]]
            binding.pages_release(pool, ints(old), pws)
            binding.pages_fork(cset, pool, ints([0, 3]), ints([1, 2]), pws)
            for p, c in ((0, 1), (3, 2)):
                lens[c], said[c] = lens[p], [list(said[p][0]), list(said[p][1])]
            attend([0, 1, 2, 3])
        if turn in (6, 30, 50):
            used = int(binding.pages_compact(cset, pool, pws).item())
            assert int((pool.refs > 0).sum()) == used and int(pool.block_table.max()) < used
            attend([r for r in range(rows) if lens[r]])
        assert binding.workspace_status(ws) == 0 and binding.workspace_status(pws) == 0, turn
        # nothing leaks: a block's count is the entries that name it
        names = pool.block_table[pool.block_table >= 0].long()
        assert torch.equal(torch.bincount(names, minlength=blocks).int(), pool.refs), turn


def test_what_the_binding_refuses():
    p = Both(8, 3, 2, layers=1)
    other = binding.Cache(9, 2, 64)
    with pytest.raises(binding.CooptError):
        binding.pages_fork(binding.CacheSet([other]), p.pages, ints([0]), ints([1]), p.ws)
    with pytest.raises(binding.CooptError):
        binding.pages_copy(binding.CacheSet([p.caches[0], other]), ints([0]), ints([1]))
    with pytest.raises(binding.CooptError):
        binding.pages_reserve(p.pages, ints([0, 1, 2, 0]), ints([1] * 4), p.ws)      # more than there are rows
    with pytest.raises(binding.CooptError):
        binding.pages_reserve(p.pages, ints([0]), ints([1]), p.ws[:100])
    with pytest.raises(binding.CooptError):
        binding.pages_release(p.pages, ints([0]), p.ws, window=-1)
    for rows, lens in ((torch.tensor([0], dtype=torch.int32), ints([1])), (ints([0]).long(), ints([1])), (ints([0, 1]), ints([1])), (ints([[0]]), ints([[1]]))):
        with pytest.raises(ValueError):
            binding.pages_reserve(p.pages, rows, lens, p.ws)
    with pytest.raises(ValueError):
        binding.Pages(p.pages.refs, p.pages.block_table.t(), p.pages.context_lens)
    with pytest.raises(ValueError):
        binding.pages_compact(p.set, p.pages, p.ws, table_out=p.pages.block_table[:2])
    with pytest.raises(ValueError):
        binding.pages_compact(p.set, p.pages, p.ws, new_ids=p.pages.refs[:3])
    with pytest.raises(ValueError):
        binding.pages_release(p.pages, ints([0]), p.ws, window=2 ** 32 + 5)
    with pytest.raises(ValueError):
        binding.Cache(8, 2, 64, data=torch.zeros(10, dtype=torch.uint8, device="cuda"))
    p.check("nothing happened")
