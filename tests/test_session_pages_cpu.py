"""Session streams forked beside each other, truncated, compacted and their
pool resized (host only): after every step, applying what the session says
(block copies by phase, block-table patches, the new rows' slots) to a model of
the device leaves every kept stream's own tokens where its table entries
point."""
import numpy as np
import pytest

import paper_2608_06146_amd as pa
from paper_2608_06146_amd import _lib


class Device:
    """What the caches and the block table hold, as token numbers."""

    def __init__(self, blocks, entries):
        self.cache = np.full((blocks, 16), -1, np.int64)
        self.table = np.full(entries, -1, np.int64)

    def step(self, view, copies, tokens):
        for pairs in copies:
            src, dst = pairs[:, 0], pairs[:, 1]
            assert len(np.unique(dst)) == len(dst) and not np.intersect1d(src, dst).size
            self.cache[dst] = self.cache[src]
        patch = view["patch"]
        for e in np.unique(patch[:, 0]):  # written in any order
            assert len(np.unique(patch[patch[:, 0] == e, 1])) == 1
        self.table[patch[:, 0]] = patch[:, 1]
        slots = view["new_slot"]
        assert len(np.unique(slots[:, 0] * 16 + slots[:, 1])) == len(slots)
        self.cache[slots[:, 0], slots[:, 1]] = tokens

    def read(self, off, n):
        return self.cache[self.table[off:off + (n + 15) // 16]].reshape(-1)[:n].tolist()


class Run:
    def __init__(self, blocks, entries=4096):
        self.s = pa.DecodeSession(4, 2, 64, blocks, block_table_capacity=entries)
        self.dev = Device(blocks, entries)
        self.tokens, self.tree, self.open = {}, {}, []
        self.next = 0

    def add(self, parent=-1, fork=0):
        i = self.s.open(parent, fork)
        self.tokens[i], self.tree[i] = [], (parent, fork)
        self.open.append(i)
        return i

    def clone(self, i, n):
        c = self.s.clone(i, n)
        self.tokens[c], self.tree[c] = self.tokens[i][:n], self.tree[i]
        self.open.append(c)
        return c

    def close(self, i):
        self.s.close(i)
        self.open.remove(i)

    def truncate(self, i, n):
        self.s.truncate(i, n)
        del self.tokens[i][n:]

    def step(self, n_new):
        self.s.prepare(n_new, [min(1, n) for n in n_new])
        v, copies = self.s.view(), self.s.copies()
        total = sum(n_new)
        new = np.arange(self.next, self.next + total)
        self.next += total
        self.dev.step(v, copies, new)
        at = 0
        for i, n in zip(sorted(self.open), n_new):
            self.tokens[i] += new[at:at + n].tolist()
            at += n
        self.s.commit()
        self.check()
        return copies

    def check(self):
        v = self.s.view()
        for g, i in zip(v["seg"], v["seg_id"]):
            i = int(i)
            assert int(g["len"]) == len(self.tokens[i])
            parent, fork = self.tree[i]
            assert int(g["fork"]) == fork and (int(v["seg_id"][g["parent"]]) if g["parent"] >= 0 else -1) == parent
            assert self.dev.read(int(g["kv_off"]), int(g["len"])) == self.tokens[i], i
        used = {int(b) for g in v["seg"] for b in v["block_table"][int(g["kv_off"]):int(g["kv_off"]) + (int(g["len"]) + 15) // 16]}
        assert -1 not in used and len(used) + v["free_blocks"] == self.s.num_blocks
        return used


def status(f, *a):
    with pytest.raises(_lib.PadocError) as e:
        f(*a)
    return e.value.status


def test_clone_shares_blocks_until_one_appends():
    r = Run(64)
    root = r.add()
    r.step([40])
    a = r.add(root, 40)
    r.step([0, 37])
    free = r.s.view()["free_blocks"]
    b, c = r.clone(a, 37), r.clone(a, 33)
    assert r.s.view()["free_blocks"] == free
    copies = r.step([0, 1, 1, 1])
    # three streams in one block: two of them copy it, the last one keeps it
    assert [len(p) for p in copies] == [2] and len(np.unique(copies[0][:, 0])) == 1
    assert r.s.view()["free_blocks"] == free - 2
    assert r.step([0, 1, 1, 1]) == []
    for i in (a, b, c):
        r.close(i)
    assert r.s.view()["free_blocks"] == 64 - 3


def test_a_clone_of_whole_blocks_copies_nothing():
    r = Run(16)
    a = r.add()
    r.step([32])
    b = r.clone(a, 32)
    c = r.clone(a, 0)
    assert r.step([3, 3, 3]) == []
    r.close(a)
    assert r.step([1, 1]) == []
    assert [len(r.tokens[i]) for i in (b, c)] == [36, 4]


def test_a_closed_streams_clone_keeps_the_blocks():
    r = Run(8)
    a = r.add()
    r.step([20])
    b = r.clone(a, 20)
    r.close(a)  # released at once: the clone is no child of it
    assert r.s.view()["free_blocks"] == 6
    assert r.step([1]) == [] and len(r.tokens[b]) == 21


def test_truncate_frees_pages_and_copies_a_shared_one():
    r = Run(16)
    a = r.add()
    r.step([40])
    b = r.clone(a, 40)
    r.truncate(b, 5)
    assert r.s.view()["free_blocks"] == 13
    copies = r.step([0, 2])  # b writes into a's first block: copied
    assert [len(p) for p in copies] == [1]
    r.truncate(a, 0)
    assert r.step([1, 1]) == []
    child = r.add(a, 1)
    assert status(r.s.truncate, a, 0) == _lib.ERR_TREE
    r.close(child)
    r.truncate(a, 0)
    assert r.step([17, 0]) == []


def test_compact_and_resize():
    r = Run(40)
    ids = [r.add() for _ in range(10)]
    r.step([50] * 10)
    for i in ids[:7]:
        r.close(i)
    used = r.check()
    assert max(used) > 12
    assert r.s.compact(2) == 2
    assert r.s.compact() > 0 and r.s.compact() == 0
    assert status(r.s.resize, 12) == _lib.ERR_MODE
    copies = r.step([0, 0, 0])
    assert sum(len(p) for p in copies) == len(used - set(range(12))) and r.check() == set(range(12))
    assert status(r.s.resize, 11) == _lib.ERR_BOUNDS
    r.s.resize(12)
    assert r.s.view()["free_blocks"] == 0
    assert status(r.s.prepare, [15] * 3, [0] * 3) == _lib.ERR_BOUNDS
    r.s.resize(30)
    r.step([15] * 3)
    assert r.check() == set(range(15))  # the smallest free ids first


def test_compact_moves_a_shared_block_for_all_its_streams():
    r = Run(32)
    a = r.add()
    big = r.add()
    r.step([0, 160])
    r.step([20, 0])
    b, c = r.clone(a, 20), r.clone(a, 18)
    r.close(big)
    assert r.s.compact() == 2
    copies = r.step([1, 1, 1])
    # the block moves, then two of its three streams copy it: from where it lies by then
    assert [len(p) for p in copies] == [2, 2]
    assert copies[1][0, 0] in copies[0][:, 1]
    assert (len(r.tokens[b]), len(r.tokens[c])) == (21, 19)


def test_failed_steps_change_nothing():
    r = Run(4)
    a = r.add()
    r.step([40])
    r.clone(a, 40), r.clone(a, 40)
    before = r.s.view()
    # 3 blocks in use and two copies needed, one block free
    assert status(r.s.prepare, [1, 1, 1], [1, 1, 1]) == _lib.ERR_BOUNDS
    after = r.s.view()
    assert np.array_equal(before["block_table"], after["block_table"]) and before["free_blocks"] == after["free_blocks"]
    assert [len(p) for p in r.step([1, 0, 0])] == [1]


def test_one_of_two_holders_appends_without_the_other():
    r = Run(8)
    a = r.add()
    r.step([5])
    r.clone(a, 5)
    assert [len(p) for p in r.step([1, 0])] == [1]  # the clone still holds the old block
    assert r.step([0, 1]) == []


def test_refusals():
    r = Run(8, 16)
    a = r.add()
    r.step([20])
    for bad in (-1, 5):
        assert status(r.s.clone, bad, 0) == _lib.ERR_ARG
        assert status(r.s.truncate, bad, 0) == _lib.ERR_ARG
    for n in (-1, 21):
        assert status(r.s.clone, a, n) == _lib.ERR_TREE
        assert status(r.s.truncate, a, n) == _lib.ERR_TREE
    assert status(r.s.compact, -1) == _lib.ERR_ARG
    assert status(r.s.resize, -1) == _lib.ERR_ARG
    assert status(r.s.resize, 2 ** 31) == _lib.ERR_ARG
    for _ in range(3):
        r.clone(a, 20)
    assert status(r.s.clone, a, 20) == _lib.ERR_BOUNDS  # the table is full
    r.s.prepare([0] * 4, [0] * 4)
    for f, args in ((r.s.clone, (a, 1)), (r.s.truncate, (a, 1)), (r.s.compact, ()), (r.s.resize, (8,))):
        assert status(f, *args) == _lib.ERR_MODE
    with pytest.raises(ValueError):
        r.s.clone(77)
    L = _lib.lib()
    assert L.padoc_session_clone(None, 0, 0, None) == _lib.ERR_ARG
    assert L.padoc_session_clone(r.s.handle, 0, 0, None) in (_lib.ERR_ARG, _lib.ERR_MODE)
    assert L.padoc_session_copies(r.s.handle, None, None, None) == _lib.ERR_ARG
    assert L.padoc_session_compact(None, 0, None) == _lib.ERR_ARG
    assert L.padoc_session_truncate(None, 0, 0) == _lib.ERR_ARG
    assert L.padoc_session_resize(None, 0, None, None) == _lib.ERR_ARG


@pytest.mark.parametrize("seed", range(12))
def test_random_runs(seed):
    rng = np.random.default_rng(seed)
    blocks = int(rng.integers(12, 60))
    r = Run(blocks, 512)
    r.add()
    refused = 0
    for _ in range(150):
        for _ in range(int(rng.integers(0, 4))):
            kept = [int(i) for i in r.s.view()["seg_id"]]
            what = rng.choice(["open", "root", "close", "clone", "truncate", "compact", "resize"])
            try:
                if what == "open" and kept:
                    p = int(rng.choice(kept))
                    r.add(p, int(rng.integers(0, len(r.tokens[p]) + 1)))
                elif what == "root":
                    r.add()
                elif what == "close" and r.open:
                    r.close(int(rng.choice(r.open)))
                elif what == "clone" and kept:
                    i = int(rng.choice(kept))
                    n = len(r.tokens[i])
                    r.clone(i, n if rng.random() < 0.5 else int(rng.integers(0, n + 1)))
                elif what == "truncate" and r.open:
                    i = int(rng.choice(r.open))
                    r.truncate(i, int(rng.integers(0, len(r.tokens[i]) + 1)))
                elif what == "compact":
                    r.s.compact(int(rng.choice([0, 1, 3])))
                elif what == "resize":
                    n = int(rng.integers(8, 70))
                    r.s.resize(n)
                    r.s.num_blocks = n
                    grown = np.full((max(n, len(r.dev.cache)), 16), -1, np.int64)
                    grown[:len(r.dev.cache)] = r.dev.cache
                    r.dev.cache = grown
            except _lib.PadocError:
                refused += 1
        n_new = [int(rng.choice([0, 1, 1, 1, 5, 30], p=[.2, .2, .2, .2, .15, .05])) for _ in r.open]
        try:
            r.step(n_new)
        except _lib.PadocError:
            refused += 1
            for i in list(r.open)[: max(1, len(r.open) // 2)]:
                r.close(i)
            r.step([0] * len(r.open))
    assert refused > 0


def test_a_pool_emptied_and_filled_again():
    """Caches of no blocks have no address: tensors of no elements."""
    import ctypes as C
    L, A = _lib.lib(), 1 << 20
    h = C.c_void_p()
    d = _lib.SessionDesc(4, 2, 64, 0.125, _lib.BF16, 8, 64, A, 2 * A, 3 * A, 0, 0)
    assert L.padoc_session_create(C.byref(d), C.byref(h)) == _lib.OK
    for n, k, v, want in ((4, A, 2 * A, _lib.OK), (4, None, None, _lib.ERR_ARG), (4, A, None, _lib.ERR_ARG), (0, None, None, _lib.OK),
                          (0, None, None, _lib.OK), (5, 4 * A, 5 * A, _lib.OK), (5, None, 5 * A, _lib.ERR_ARG), (0, 4 * A, 5 * A, _lib.OK)):
        assert L.padoc_session_resize(h, n, k, v) == want, (n, k, v)
    L.padoc_session_destroy(h)
    s = pa.DecodeSession(4, 2, 64, 8)  # host only: none, whatever the pool
    for n in (0, 3):
        assert L.padoc_session_resize(s.handle, n, None, None) == _lib.OK
        assert L.padoc_session_resize(s.handle, n, A, 2 * A) == _lib.ERR_ARG
