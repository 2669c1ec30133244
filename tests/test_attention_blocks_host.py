"""The arithmetic that attention's kernels and launch plan share (csrc/blocks.hpp), compiled
for the host: numbers of blocks, the tiles they see, the ranges that the plan makes of them."""

import ctypes as C
import os
import subprocess

import numpy as np
import pytest

import paper_2608_15531_amd as fq
from test_layer_host import attn, cache, lib  # noqa: F401  (lib: fixture)

CSRC = os.path.join(os.path.dirname(fq.LIB_PATH), "csrc")

SHIM = r"""
#include "blocks.hpp"
template <int T>
static int tiles(int p_lo, int p_hi, int window, int sinks, int* out, int most) {
  const fqi::TileRange r = fqi::tile_range<T>(p_lo, p_hi, window, sinks);
  for (int i = 0; i < r.n && i < most; ++i) out[i] = r.tile(i);
  return r.n;
}
extern "C" {
int64_t number(int64_t t0, int group, int rows, int seq, int rb) { return fqi::dense_number(t0, group, rows, seq, rb); }
int64_t blocks(int64_t total, int64_t group, int rows, int64_t n_seqs) { return fqi::dense_blocks(total, group, rows, n_seqs); }
int tiles32(int a, int b, int w, int s, int* out, int most) { return tiles<32>(a, b, w, s, out, most); }
int tiles64(int a, int b, int w, int s, int* out, int most) { return tiles<64>(a, b, w, s, out, most); }
int ranges(int n, int split_tiles, int split) { return fqi::range_count(n, split_tiles, split); }
}
"""


@pytest.fixture(scope="module")
def shim(tmp_path_factory):
    d = tmp_path_factory.mktemp("blocks")
    (d / "shim.cpp").write_text(SHIM)
    subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", "-Werror", "-fPIC", "-shared", "-I", CSRC, str(d / "shim.cpp"),
                    "-o", str(d / "shim.so")], check=True)
    s = C.CDLL(str(d / "shim.so"))
    s.number.argtypes = [C.c_int64, C.c_int, C.c_int, C.c_int, C.c_int]
    s.blocks.argtypes = [C.c_int64, C.c_int64, C.c_int, C.c_int64]
    s.number.restype = s.blocks.restype = C.c_int64
    return s


def tiles_of(shim, size, p_lo, p_hi, window, sinks, most=1 << 14):
    out = (C.c_int * most)()
    n = (shim.tiles32 if size == 32 else shim.tiles64)(p_lo, p_hi, window, sinks, out, most)
    assert n <= most
    return list(out[:n])


@pytest.mark.parametrize("rows", [16, 128])
@pytest.mark.parametrize("group", [1, 3, 4, 8, 24])
def test_block_numbers_differ_and_are_bounded(shim, group, rows):
    """Whatever the lengths: also those that max_q cuts and sequences without a token."""
    rng = np.random.default_rng(group)
    for case in range(300):
        q = rng.integers(0, [2, 40, 400][case % 3], int(rng.integers(1, 12)))
        max_q = int(max(q.max(), 1)) if case % 2 else int(rng.integers(1, 400))
        cu = np.concatenate([[0], np.cumsum(q)])
        seen = [shim.number(int(cu[b]), group, rows, b, rb) for b in range(len(q))
                for rb in range(-(-min(int(q[b]), max_q) * group // rows))]
        assert len(set(seen)) == len(seen)
        assert all(0 <= n < shim.blocks(int(cu[-1]), group, rows, len(q)) for n in seen)


@pytest.mark.parametrize("size", [32, 64])
def test_tiles_are_those_with_a_seen_key(shim, size):
    """In order, each once, and none beyond the last key; every tile with a key that a row of
    the block sees is among them."""
    rng = np.random.default_rng(size)
    for _ in range(3000):
        p_lo = int(rng.integers(-3, 700))
        p_hi = p_lo + int(rng.integers(0, 130))
        window = int(rng.choice([0, 1, 2, 17, 63, 64, 65, 300, 1 << 30]))
        sinks = int(rng.choice([0, 1, 4, 63, 64, 129, 2**31 - 1]))
        got = tiles_of(shim, size, p_lo, p_hi, window, sinks)
        j = np.arange(max(p_hi + 1, 0))
        see = ((j > p_lo - window) | (j < sinks)) if window else np.ones(len(j), bool)
        need = sorted(set((j[see] // size).tolist()))
        where = (p_lo, p_hi, window, sinks)
        assert got == sorted(set(got)), where
        assert set(need) <= set(got) and (not got or got[-1] <= max(p_hi, 0) // size), where


@pytest.mark.parametrize("head_dim", [64, 128])
@pytest.mark.parametrize("heads", [(1, 1), (32, 8), (64, 8), (6, 2), (5, 1), (24, 1)])
def test_plans_cover_the_tiles_of_their_kernel(lib, shim, heads, head_dim):  # noqa: F811
    """The ranges of the plan hold every tile, of the size that its kernel takes, of any block
    of rows at any place, and the kernel's count of them is within the plan's."""
    G = heads[0] // heads[1]
    kernels = set()
    for max_q in (1, 5, 16, 100, 2048):
        for max_kv in (1, 31, 65, 1000, 32768, 131072):
            for window, sinks in ((0, 0), (1, 0), (100, 4), (4096, 200), (4097, 63)):
                for n_seqs in (1, 7, 64):
                    c = cache(n_kv_heads=heads[1], head_dim=head_dim, kind=fq.FQ_KV_BF16, n_pages=1 << 20)
                    a = attn(n_seqs=n_seqs, n_heads=heads[0], max_q=max_q, max_kv=max_kv, table_cols=2048,
                             window=window, sinks=sinks, total_q=n_seqs * max_q)
                    out = (C.c_int32 * 8)()
                    assert lib.fq_paged_attention_launch(C.byref(a), C.byref(c), out) == 0
                    size = 32 if out[0] == fq.FQ_ATTN_ROWS else 64
                    kernels.add(out[0])
                    assert out[4] % size == 0 and out[4] > 0
                    tokens = min(max_q, (out[1] - 1 + G - 1) // G + 1)   # that a block's rows can touch
                    for p in {0, 1, 31, 63, 64, 1000, 5000, max_kv - tokens, max_kv - 1}:
                        p_lo = max(0, min(p, max_kv - 1))
                        p_hi = min(p_lo + tokens - 1, max_kv - 1)
                        n = len(tiles_of(shim, size, p_lo, p_hi, window, sinks))
                        where = (max_q, max_kv, window, sinks, n_seqs, p, list(out))
                        assert n <= out[3] * (out[4] // size), where
                        parts = shim.ranges(n, out[4] // size, out[3])
                        assert 1 <= parts <= out[3] and n <= parts * (out[4] // size), where
    assert kernels == {fq.FQ_ATTN_ROWS, fq.FQ_ATTN_TILES}
