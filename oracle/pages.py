"""TEST INFRASTRUCTURE — CPU oracle, part 3: a pool of pages, one block and one row at a time.

Only the tests may import this; the CUDA path shares no code with it.

``Pool`` holds what the library's page calls work on: ``refs`` (how many table entries hold a block; 0 = free),
``table`` [rows, width] (-1 = no block) and ``lens``, and the contents of every layer's blocks as one array
[layers, blocks, bytes].  Blocks are handed out lowest first.  Every call returns the worst that it met: "ok",
"invalid" or "pages" (too few free blocks); what is refused changes nothing.
"""
from __future__ import annotations

import numpy as np

BLOCK_SIZE = 16


def _blocks(tokens: int) -> int:
    return -(-tokens // BLOCK_SIZE)


class Pool:
    def __init__(self, num_blocks: int, rows: int, width: int, contents: np.ndarray):
        self.refs = np.zeros(num_blocks, dtype=np.int32)
        self.table = np.full((rows, width), -1, dtype=np.int32)
        self.lens = np.zeros(rows, dtype=np.int32)
        self.contents = contents
        self.problems: set = set()

    def _take(self) -> int:
        block = int(np.nonzero(self.refs <= 0)[0][0])
        self.refs[block] = 1
        return block

    def _free(self) -> int:
        return int(np.sum(self.refs <= 0))

    def copy(self, src, dst) -> None:
        for s, d in zip(src, dst):
            if 0 <= s < len(self.refs) and 0 <= d < len(self.refs):
                self.contents[:, d] = self.contents[:, s]

    def reserve(self, row_ids, new_lens) -> None:
        rows, width = self.table.shape
        seen, asked, free = set(), 0, self._free()
        for r, n in zip(row_ids, new_lens):
            r, n = int(r), int(n)
            if not 0 <= r < rows:
                self.problems.add("invalid")
                continue
            again = r in seen
            seen.add(r)
            if again or n < self.lens[r] or n > width * BLOCK_SIZE:
                self.problems.add("invalid")
                continue
            lacking = [j for j in range(_blocks(int(self.lens[r])), _blocks(n)) if self.table[r, j] < 0]
            asked += len(lacking)
            if lacking and asked > free:
                self.problems.add("pages")
                continue
            for j in lacking:
                self.table[r, j] = self._take()
            self.lens[r] = n

    def fork(self, parents, children) -> None:
        rows = self.table.shape[0]
        named = set(int(c) for c in children)
        seen, asked, free, shared, lens, used = set(), 0, self._free(), [], self.lens.copy(), self.refs > 0

        def in_use(x):                                        # .. before the call
            return 0 <= x < len(used) and bool(used[x])

        for p, c in zip(parents, children):
            p, c = int(p), int(c)
            ok = 0 <= p < rows and 0 <= c < rows and c not in seen and p not in named and lens[c] == 0
            if 0 <= c < rows:
                seen.add(c)
            if not ok:
                self.problems.add("invalid")
                continue
            length = int(lens[p])
            row = np.full(self.table.shape[1], -1, dtype=np.int32)
            if length % BLOCK_SIZE:
                if not in_use(int(self.table[p, length // BLOCK_SIZE])):
                    self.problems.add("invalid")
                    continue
                asked += 1
                if asked > free:
                    self.problems.add("pages")
                    continue
                block = self._take()
                row[length // BLOCK_SIZE] = block
                self.contents[:, block] = self.contents[:, self.table[p, length // BLOCK_SIZE]]
            full = length // BLOCK_SIZE
            row[:full] = self.table[p, :full]
            for j in range(full):
                if row[j] >= 0 and not in_use(int(row[j])):
                    self.problems.add("invalid")
                    row[j] = -1
            shared += [int(x) for x in row[:full] if x >= 0]
            self.table[c], self.lens[c] = row, length
        for block in shared:
            self.refs[block] += 1

    def release(self, row_ids, window: int = 0, sinks: int = 0) -> None:
        rows, width = self.table.shape
        for r in row_ids:
            if not 0 <= int(r) < rows:
                self.problems.add("invalid")
                continue
            for j in range(width):
                tokens = range(j * BLOCK_SIZE, (j + 1) * BLOCK_SIZE)
                if window and any(t < sinks or t >= self.lens[r] - window for t in tokens):
                    continue
                block, self.table[r, j] = int(self.table[r, j]), -1
                if block >= 0:
                    if self.refs[block] > 0:
                        self.refs[block] -= 1
                    else:
                        self.problems.add("invalid")
            if not window:
                self.lens[r] = 0

    def compact(self) -> int:
        used = [b for b in range(len(self.refs)) if self.refs[b] > 0]
        count = len(used)
        goes = {b: b for b in used if b < count}
        holes = [b for b in range(count) if self.refs[b] <= 0]
        goes.update(zip([b for b in used if b >= count], holes))
        refs = np.where(np.arange(len(self.refs)) < count, 0, np.zeros_like(self.refs))
        for old, new in goes.items():
            refs[new] = self.refs[old]
            if old != new:
                self.contents[:, new] = self.contents[:, old]
        for r in range(self.table.shape[0]):
            for j in range(self.table.shape[1]):
                old = int(self.table[r, j])
                if old >= 0:
                    if old not in goes:
                        self.problems.add("invalid")
                    self.table[r, j] = goes.get(old, -1)
        self.refs = refs.astype(np.int32)
        return count
