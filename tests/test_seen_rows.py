"""Which rows a query sees and where they lie (seen_rows.hpp, compiled for the host) against the same said row by row."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2503_01586_amd", "csrc")


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    d = tmp_path_factory.mktemp("rows")
    (d / "m.cpp").write_text('''#include "seen_rows.hpp"
extern "C" void seen(const int* table, int cols, int shift, int n_pages, const int* nodes, const unsigned* mask, int words, const int* len,
                     int b, int q, long stride, long cap, long* out_len, unsigned* tiles, long* rows, unsigned char* sees) {
  ekv::RowMap m{table, cols, shift, n_pages, nodes, mask, words};
  const ekv::SeenRows s(m, len, b, q, stride, cap);
  *out_len = s.len;
  for (long j = 0; j < s.len; j += 16) tiles[j / 16] = s.tile(j);
  for (long j = 0; j < s.len; ++j) { rows[j] = s.row(j, s.page(j)); sees[j] = s.sees(j); }
}
''')
    subprocess.run(["g++", "-O1", "-fsanitize=undefined", "-fno-sanitize-recover", "-shared", "-fPIC", "-I", CSRC, str(d / "m.cpp"),
                    "-o", str(d / "m.so")], check=True)
    return ctypes.CDLL(str(d / "m.so"))


def ask(lib, b, q, lens, stride, cap, table=None, shift=0, n_pages=0, nodes=None, mask=None):
    P = lambda a: None if a is None else a.ctypes.data_as(ctypes.c_void_p)
    n, tiles, rows, sees = ctypes.c_long(), np.zeros(64, np.uint32), np.zeros(1024, np.int64), np.zeros(1024, np.uint8)
    lib.seen(P(table), 0 if table is None else table.shape[1], shift, n_pages, P(nodes), P(mask), 0 if mask is None else mask.shape[2],
             P(lens), b, q, ctypes.c_long(stride), ctypes.c_long(cap), ctypes.byref(n), P(tiles), P(rows), P(sees))
    n = n.value
    bits = [bool(tiles[j // 16] >> (j % 16) & 1) for j in range(n)]
    assert all(not tiles[j] >> 16 for j in range(64)) and all(not tiles[j // 16] >> (j % 16) & 1 for j in range(n, -(-n // 16) * 16))
    assert bits == [bool(v) for v in sees[:n]] and (n == 0 or bits[-1])
    return [int(rows[j]) for j in range(n) if bits[j]]


def test_the_first_rows_back_to_back_and_in_pages(lib):
    lens = np.array([0, 1, 15, 16, 17, 63, 64, 65, 100, -3, 2**31 - 1], dtype=np.int32)
    for b, n in enumerate(lens.tolist()):
        for cap in (0, 1, 16, 70, 96):
            want = max(0, min(n, cap))
            assert ask(lib, b, 1, lens, 1000, cap) == [b * 1000 + j for j in range(want)]
    rng = np.random.default_rng(0)
    for shift in (4, 5, 6):
        page, cols = 1 << shift, 7
        table = rng.permutation(11 * cols).reshape(11, cols).astype(np.int32)
        table[3, 1], table[8, 0] = -1, 77
        for b, n in enumerate(lens.tolist()):
            want = max(0, min(n, cols * page))
            real = lambda p: p if 0 <= p < 77 else 0
            assert ask(lib, b, 1, lens, 0, cols * page, table=table, shift=shift, n_pages=77) == [
                real(int(table[b, j // page])) * page + j % page for j in range(want)]


@pytest.mark.parametrize("T", [1, 5, 31, 32, 33, 64, 97, 128])
def test_masks_behind_a_prefix(lib, T):
    rng = np.random.default_rng(T)
    prefix = np.array([0, 1, 15, 16, 37, 200, -5], dtype=np.int32)
    nodes = np.array([T, T, max(T - 3, 0), T + 9, 1, T, T], dtype=np.int32)
    B = len(prefix)
    for density in (0.0, 0.03, 0.5, 1.0):
        sees = rng.random((B, T, 32 * -(-T // 32))) < density            # bits past the nodes set as well
        mask = np.packbits(sees, axis=-1, bitorder="little").view(np.uint32).copy()
        for cap in (1000, 210, 40, 3):
            for b in range(B):
                P = min(max(int(prefix[b]), 0), cap)
                for t in {0, T // 2, T - 1}:
                    want = []
                    if t < min(nodes[b], T):
                        want = list(range(P)) + [P + j for j in range(min(nodes[b], T)) if sees[b, t, j] and P + j < cap]
                    got = ask(lib, b * T + t, T, prefix, 500, cap, nodes=nodes, mask=mask)
                    assert got == [b * 500 + j for j in want], (density, cap, b, t)
