"""The 4-bit cache and the page calls without a GPU: what their code does on the host, and device functions that are plain C++ run there."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2508_09072_b200", "csrc")

WALK = r"""
#include <cstdio>
#include <cstdlib>
#include <vector>
#include "ancestors.cuh"
// kind (0 bytes, 1 words), then trees of 128 parents on stdin: both halves of every node's ancestors
template <typename P> void run(FILE *f) {
    std::vector<P> all(128);
    while (fread(all.data(), sizeof(P), 128, f) == 128)
        for (int node = 0; node < 128; ++node) {
            unsigned long long word[2][2];
            for (int fill = 0; fill < 2; ++fill) {   // (what is behind the node has no say)
                std::vector<P> parents(all);
                for (int i = node + 1; i < 128; ++i) parents[i] = (P)fill;
                for (int half = 0; half < 2; ++half) word[fill][half] = reader::ancestors(parents.data(), node, half);
            }
            if (word[0][0] != word[1][0] || word[0][1] != word[1][1]) abort();
            fwrite(word[0], 8, 2, stdout);
        }
}
int main(int argc, char **argv) { argv[1][0] == '0' ? run<unsigned char>(stdin) : run<int>(stdin); return argc - 2; }
"""


@pytest.fixture(scope="module")
def walk(tmp_path_factory):
    d = tmp_path_factory.mktemp("walk")
    (d / "walk.cpp").write_text(WALK)
    subprocess.run([os.environ.get("CXX", "g++"), "-std=c++17", "-O1", "-x", "c++", "-I", CSRC,
                    str(d / "walk.cpp"), "-o", str(d / "walk")], check=True)

    def run(parents):
        kind = "0" if parents.dtype == np.uint8 else "1"
        r = subprocess.run([str(d / "walk"), kind], input=parents.tobytes(), stdout=subprocess.PIPE, timeout=60, check=True)
        return np.frombuffer(r.stdout, dtype=np.uint64).reshape(len(parents), 128, 2)
    return run


def seen_by(parents):
    """128 x 128 truth values of a tree."""
    s = np.zeros((128, 128), bool)
    for j, a in enumerate(parents):
        if a >= 0:
            s[j] = s[a]
        s[j, j] = True
    return s


def test_ancestors_of_trees(walk):
    rng = np.random.default_rng(1)
    trees = np.full((40, 128), -1, np.int32)
    for i, t in enumerate(trees):
        for j in range(1, 128):
            t[j] = j - 1 if i == 0 else 0 if i == 1 else rng.integers(max(0, j - 1 - i), j)
    for kind in (np.uint8, np.int32):
        got = walk(trees.astype(kind))
        bits = np.unpackbits(got.view(np.uint8).reshape(40, 128, 16), axis=-1, bitorder="little").astype(bool)
        assert np.array_equal(bits, np.stack([seen_by(t) for t in trees]))


def test_the_walk_ends_whatever_the_parents_are(walk):
    """Loops, parents above their children and outside the tree: what a thread block that gave up may find."""
    rng = np.random.default_rng(2)
    loops = np.tile(np.arange(128), (4, 1))
    loops[1] = np.arange(128) ^ 1
    loops[2] = (np.arange(128) + 1) % 128
    loops[3] = 127 - np.arange(128)
    for kind in (np.uint8, np.int32):
        wild = rng.integers(0, 256, (200, 128)) if kind == np.uint8 else rng.integers(-2 ** 31, 2 ** 31, (200, 128))
        near = rng.integers(0, 129, (200, 128))
        for trees in (loops, wild, near):
            got = walk(trees.astype(kind))
            for j in range(128):   # the node itself, and none above it
                word = got[:, j, 0].astype(object) + (got[:, j, 1].astype(object) << 64)
                assert all((w >> j) == 1 for w in word)


# ---------------------------------------------------------------------------------------------- refusals
class Pages(ctypes.Structure):
    _fields_ = [("refs", ctypes.c_void_p), ("num_pages", ctypes.c_int32), ("page_table", ctypes.c_void_p), ("rows", ctypes.c_int32),
                ("max_pages_per_seq", ctypes.c_int32), ("seq_lens", ctypes.c_void_p), ("pools", ctypes.c_void_p), ("n_pools", ctypes.c_int32),
                ("page_bytes", ctypes.c_size_t)]


class Cache(ctypes.Structure):
    _fields_ = [("k_pool", ctypes.c_void_p), ("v_pool", ctypes.c_void_p), ("num_pages", ctypes.c_int32), ("page_size", ctypes.c_int32),
                ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("page_table", ctypes.c_void_p), ("max_pages_per_seq", ctypes.c_int32),
                ("seq_lens", ctypes.c_void_p), ("shared_prefix_len", ctypes.c_int32)]


@pytest.mark.parametrize("many", [2 ** 30 + 1, 2 ** 31 - 1])
def test_counts_that_32_bit_loops_cannot_pass_are_refused(many):
    """Before anything is launched, and before anything behind an address is looked at (here none is one)."""
    from paper_2508_09072_b200 import binding
    lib = binding.load_library()
    at, i, size, no, bad = ctypes.c_void_p(1 << 20), ctypes.c_int32, ctypes.c_size_t, ctypes.c_void_p(None), binding.ERR_UNSUPPORTED
    pool = (ctypes.c_void_p * 1)(1 << 20)
    pools = ctypes.cast(pool, ctypes.c_void_p)

    def pages(num_pages):
        return ctypes.byref(Pages(1 << 20, num_pages, 1 << 20, 8, 1, 1 << 20, pools, 1, 16))
    few, huge = pages(100), pages(many)
    ws, room, n = ctypes.c_void_p(1 << 20), size(1 << 50), i(many)
    for p, count in ((huge, i(1)), (few, n)):
        assert lib.reader_pages_fork(at, p, at, at, count, ws, room, at, no) == bad
        assert lib.reader_pages_reserve(at, p, at, at, count, ws, room, at, no) == bad
        assert lib.reader_pages_free(at, p, at, at, count, at, no) == bad
    assert lib.reader_pages_compact(at, huge, at, ws, room, no) == lib.reader_pages_compact_map(at, huge, at, at, ws, room, no) == bad
    assert lib.reader_pages_copy(at, pools, i(9), pools, i(9), i(1), size(16), at, at, n, at, no) == bad
    need = lib.reader_pages_workspace_bytes
    assert need(many, 8, 1, 1) == 0 and need(100, 8, 1, many) == 0 and need(2 ** 30, 8, 1, 2 ** 30) > 0
    wide, narrow = (Cache(1 << 20, 1 << 20, 4, 64, 2, 64, 1 << 20, 1, 1 << 20, 0) for _ in range(2))
    assert lib.reader_q4_store(at, ctypes.byref(wide), ctypes.byref(narrow), i(1), n, at, at, at, no) == bad
    assert lib.reader_q4_load(at, ctypes.byref(narrow), ctypes.byref(wide), i(1), n, at, at, at, no) == bad
    assert lib.reader_q4_commit(at, ctypes.byref(narrow), pools, pools, i(1), n, i(4), at, at, i(4), i(1), at, at, no) == bad
