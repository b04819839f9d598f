"""Pins of the oracle's window attention and of its pool: by hand, by brute force and by invariants."""
import math

import numpy as np
import pytest

from oracle import attention, pages


def _problem(seed, lens, hq, hkv, dim, q_lens=None):
    rng = np.random.default_rng(seed)
    need = [-(-n // 16) for n in lens]
    order = rng.permutation(sum(need) + 3)
    table = np.full((len(lens), max(max(need), 1)), -1)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    kv = rng.standard_normal((sum(need) + 3, hkv, 2, 16, dim))
    q = rng.standard_normal((sum(q_lens or [1] * len(lens)), hq, dim))
    return q, kv, table


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 3), (7, 2), (16, 16), (40, 0), (1000, 0), (5, 1000)])
def test_window_attention_is_the_sum_over_visible_tokens(window, sinks):
    lens, n = [0, 1, 9, 40], [1, 1, 4, 5]                 # the first sequence's query has no context
    q, kv, table = _problem(3, lens, 4, 2, 3, n)
    cu = np.cumsum([0] + n)
    out, spread = attention.window_attention(q, kv, table, lens, window, sinks, cu)
    for b, L in enumerate(lens):
        for i in range(n[b]):
            t = L - n[b] + i
            seen = [j for j in range(L) if j <= t and (j < sinks or j > t - window)]
            for h in range(4):
                num, den, mag = [0.0] * 3, 0.0, [0.0] * 3
                for j in seen:
                    k, v = (kv[table[b, j // 16], h // 2, w, j % 16] for w in (0, 1))
                    e = math.exp(sum(float(x) * float(y) for x, y in zip(q[cu[b] + i, h], k)) / math.sqrt(3))
                    den += e
                    num = [a + e * float(x) for a, x in zip(num, v)]
                    mag = [a + e * abs(float(x)) for a, x in zip(mag, v)]
                want = [a / den if den else 0.0 for a in num]
                assert np.allclose(out[cu[b] + i, h], want, atol=1e-12)
                assert np.allclose(spread[cu[b] + i, h], [a / den if den else 0.0 for a in mag], atol=1e-12)


def test_a_window_over_everything_is_plain_attention_and_hidden_blocks_are_not_read():
    lens = [5, 70, 33]
    q, kv, table = _problem(5, lens, 4, 4, 8)
    full = attention.paged_attention(q, kv, table, lens)
    assert np.allclose(attention.window_attention(q, kv, table, lens, 70, 0)[0], full, atol=1e-13)
    assert np.allclose(attention.window_attention(q, kv, table, lens, 1, 70)[0], full, atol=1e-13)
    holes = table.copy()
    holes[1, 1:3] = 10 ** 6                               # tokens 16..47 of 70: outside 16 sinks and a window of 20
    assert np.array_equal(attention.window_attention(q, kv, holes, lens, 20, 16)[0], attention.window_attention(q, kv, table, lens, 20, 16)[0])
    # one token more or less is seen in the result
    assert not np.allclose(attention.window_attention(q, kv, table, lens, 20, 16)[0], attention.window_attention(q, kv, table, lens, 21, 16)[0], atol=1e-6)


def test_pool_by_hand():
    contents = np.arange(2 * 8).reshape(2, 8, 1).copy()
    p = pages.Pool(8, 4, 4, contents)
    p.reserve([1, 0], [20, 1])
    assert p.table.tolist()[:2] == [[2, -1, -1, -1], [0, 1, -1, -1]] and p.lens.tolist() == [1, 20, 0, 0] and p.refs.tolist() == [1, 1, 1, 0, 0, 0, 0, 0]
    p.fork([1], [3])                                      # block 0 shared, block 1 (4 tokens) copied to 3
    assert p.table[3].tolist() == [0, 3, -1, -1] and p.refs.tolist() == [2, 1, 1, 1, 0, 0, 0, 0] and contents[:, 3, 0].tolist() == [1, 9]
    p.release([1, 1])
    assert p.refs.tolist() == [1, 0, 1, 1, 0, 0, 0, 0] and p.lens[1] == 0 and not p.problems
    assert p.compact() == 3                               # block 3 moves to 1
    assert p.refs.tolist() == [1, 1, 1, 0, 0, 0, 0, 0] and p.table[3].tolist() == [0, 1, -1, -1] and contents[:, 1, 0].tolist() == [1, 9]
    p.reserve([3, 0, 2], [64, 64, 16])                    # 2 blocks, then 3 more of 3 left, then one too many
    assert p.table[3].tolist() == [0, 1, 3, 4] and p.table[0].tolist() == [2, 5, 6, 7] and p.lens.tolist() == [64, 0, 0, 64] and p.problems == {"pages"}
    p.problems.clear()
    p.release([3], window=20, sinks=1)                    # tokens 16..43 fall out: block positions 1 (16..31)
    assert p.table[3].tolist() == [0, -1, 3, 4]
    p.reserve([0, 9, 3, 3], [10, 5, 64, 64])
    assert p.problems == {"invalid"}


# ---- refusals of the library that need no device -----------------------------------------------------------------

def test_refusals_on_the_host():
    import ctypes

    from paper_2602_09323_b200 import binding, build
    build.build()
    lib = binding.load_library()
    def cache(data=0x1000, blocks=8, heads=2, dim=128, size=16, dtype=0):
        return binding.coopt_cache(data, blocks, heads, dim, size, dtype)

    ok = cache()

    def decode(c=ok, k=None, v=None, stride=0, slots=None, q=0x100, out=0x100, table=0x100, width=4, lens=0x100, batch=2, hq=8, window=5, sinks=1, ws=None, n=0):
        return lib.coopt_window_decode(ctypes.byref(c) if c else None, k, v, stride, slots, q, out, table, width, lens, batch, hq, window, sinks, 0.1, ws, n, None)

    def prefill(c=ok, q=0x100, out=0x100, cu=0x100, table=0x100, width=4, lens=0x100, batch=2, hq=8, total=9, window=5, sinks=1, ws=None, n=0):
        return lib.coopt_window_prefill(ctypes.byref(c) if c else None, q, out, cu, table, width, lens, batch, hq, total, window, sinks, 0.1, ws, n, None)

    for call in (decode, prefill):
        assert call() == -3 and call(ws=0x100, n=100) == -3
        assert call(c=None) == -1 and call(q=None) == -1 and call(table=None) == -1 and call(lens=None) == -1 and call(out=0x108) == -1
        assert call(window=0) == -1 and call(window=-2 ** 31) == -1 and call(sinks=-1) == -1 and call(batch=-1) == -1
        assert call(hq=18) == -2 and call(hq=7) == -2 and call(width=2 ** 26) == -2 and call(batch=513) == -2
        assert call(c=cache(dim=96)) == -2 and call(c=cache(size=32)) == -2 and call(c=cache(data=0x1010)) == -1
        assert call(batch=0) == 0
    assert prefill(cu=None) == -1 and prefill(total=-1) == -1 and prefill(total=0) == 0 and prefill(c=cache(dtype=1)) == -2
    assert decode(k=0x100) == -1 and decode(k=0x100, v=0x100, slots=0x100, stride=255) == -1 and decode(k=0x100, v=0x100, slots=0x100, stride=256) == -3

    n = lib.coopt_pages_workspace_bytes(8, 3)
    assert n > 0 and lib.coopt_pages_workspace_bytes(0, 3) == 0 and lib.coopt_pages_workspace_bytes(8, -1) == 0
    pool = lambda refs=0x100, table=0x100, lens=0x100, blocks=8, rows=3, width=4: binding.coopt_pages(refs, table, lens, blocks, rows, width)     # noqa: E731
    one = (binding.coopt_cache * 1)(ok)
    calls = {
        "reserve": lambda p, ws=0x100, size=n, a=0x100, b=0x100, k=1: lib.coopt_pages_reserve(p, a, b, k, ws, size, None),
        "fork": lambda p, ws=0x100, size=n, a=0x100, b=0x100, k=1: lib.coopt_pages_fork(one, 1, p, a, b, k, ws, size, None),
        "release": lambda p, ws=0x100, size=n, a=0x100, b=0x100, k=1: lib.coopt_pages_release(p, a, k, 0, 0, ws, size, None),
        "compact": lambda p, ws=0x100, size=n, a=0x100, b=0x100, k=1: lib.coopt_pages_compact(one, 1, p, a, b, 0x100, None, ws, size, None),
    }
    for name, call in calls.items():
        ref = lambda **k: ctypes.byref(pool(**k))     # noqa: E731
        assert call(None) == -1 and call(ref(refs=None)) == -1 and call(ref(table=None)) == -1 and call(ref(lens=None)) == -1, name
        assert call(ref(blocks=0)) == -1 and call(ref(rows=0)) == -1 and call(ref(width=0)) == -1, name
        assert call(ref(blocks=2 ** 20 + 1)) == -2 and call(ref(rows=8193)) == -2 and call(ref(width=2 ** 26)) == -2, name
        assert call(ref(), ws=None) == -3 and call(ref(), size=n - 1) == -3 and call(ref(), a=None) == -1, name
        if name != "compact":
            assert call(ref(), k=-1) == -1 and call(ref(), k=0) == 0, name
        if name in ("reserve", "fork"):
            assert call(ref(), b=None) == -1 and call(ref(), k=4) == -1, name
    p = ctypes.byref(pool())
    assert lib.coopt_pages_release(p, 0x100, 1, -1, 0, 0x100, n, None) == -1 and lib.coopt_pages_release(p, 0x100, 1, 4, -1, 0x100, n, None) == -1
    copy = lambda caches, k, a=0x100, b=0x100, m=1: lib.coopt_pages_copy(caches, k, a, b, m, None)     # noqa: E731
    two = lambda **k: (binding.coopt_cache * 2)(ok, cache(**k))     # noqa: E731
    assert copy(one, 0) == -1 and copy(None, 1) == -1 and copy(one, 1, m=-1) == -1 and copy(one, 1, m=0) == 0 and copy(one, 1, a=None) == -1
    assert copy(two(blocks=9), 2) == -1 and copy(two(heads=1), 2) == -1 and copy(two(dim=64), 2) == -1 and copy(two(dtype=2), 2) == -1
    assert copy(two(dim=96), 2) == -2 and copy(two(data=0), 2) == -1 and copy(one, 1, m=2 ** 30) == -2
    assert lib.coopt_pages_fork((binding.coopt_cache * 1)(cache(blocks=9)), 1, p, 0x100, 0x100, 1, 0x100, n, None) == -1
    assert binding.status_string(-6).startswith("too few")


def test_the_reciprocal_rule_is_within_an_ulp_of_the_quotient():
    from oracle import e4m3, e5m2, kv_cache
    rng = np.random.default_rng(11)
    differ = 0
    for fmt in (e4m3, e5m2):
        for trial in range(200):
            k, v = (rng.standard_normal((1, 1, 8)).astype(np.float32) * np.float32(10.0 ** rng.integers(-3, 4)) for _ in range(2))
            one, two = kv_cache.new_cache(1, 1, 8), kv_cache.new_cache(1, 1, 8)
            kv_cache.kv_write(*one, k, v, np.array([0]), fmt=fmt)
            kv_cache.kv_write(*two, k, v, np.array([0]), fmt=fmt, reciprocal=True)
            a, b = one[1].view(np.int32).astype(np.int64), two[1].view(np.int32).astype(np.int64)
            assert np.all(np.abs(a - b) <= 1)
            differ += int(np.sum(a != b))
            # the largest value still takes the largest code
            assert np.isclose(np.abs(fmt.decode(two[0])).max(), fmt.MAX)
    assert differ > 0
