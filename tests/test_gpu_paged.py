"""A cache in pages and trees of drafted tokens on the GPU, against the oracle's 64 bits, through the package's entry points.

Bounds.  fp32: the parity gate of the decode kernels, max-abs-rel 1e-5.  bf16: their 2e-2, and as a 2-norm 5e-3: the absorbed query,
the probabilities, the splits' accumulators and the result are each rounded to bf16 once, a step of 2^-8 relative at most, uniform, so
2^-8 / sqrt(3) x 0.72 (mean of the mantissa's square) = 1.6e-3 in the 2-norm each, the query's twice (through the scores of two sums):
sqrt(5) x 1.6e-3 = 3.6e-3, with a third as much again for what depends on the draw: 5e-3.  A query g times as large has scores, and so
errors of its own rounding in them (absolute ones, which are the probabilities' relative ones), g times as large: sqrt(3 + 2 g^2) x
1.6e-3 and the third, for g = 4 1.3e-2.  A tile lost or seen twice among the few hundred rows here is more than 5e-2.
Plans, masks and moved rows are whole numbers and copies: equal."""
import numpy as np
import pytest
import torch

import elitekv_synth as synth
import paper_2503_01586_amd as ekv
from oracle import elitekv_oracle as orc

from gpu_util import DEV, TOL, dev, dims_of, host64, i32, i64
from test_gpu_parity import _draw, shape

pytestmark = pytest.mark.gpu

# kernels of every path: matrix cores with 8, 4 and 2 waves, one and two head groups, separated latents; fp32 tiled; any shape
SHAPES = {
    "7b": (shape(64, 32, 128, 8, 1536, "bf16"), 0),
    "13b": (shape(64, 40, 128, 8, 1920, "bf16"), 0),
    "12pct": (shape(64, 32, 128, 4, 768, "bf16"), 0),
    "narrow": (shape(64, 6, 64, 4, 128, "bf16"), 0),
    "r16_72_heads": (shape(64, 72, 128, 16, 256, "bf16"), 0),
    "slrd": (shape(64, 32, 128, 8, 1536, "bf16"), 768),
    "fp32_tiled": (shape(64, 5, 64, 4, 96, "fp32"), 0),
    "fp32_tiled_slrd": (shape(64, 18, 64, 8, 160, "fp32"), 64),
    "bf16_tiled": (shape(64, 3, 64, 6, 208, "bf16"), 0),
    "fp32_any": (shape(64, 3, 24, 5, 37, "fp32"), 0),
    "bf16_any_slrd": (shape(64, 4, 40, 3, 51, "bf16"), 20),
    "fp32_r0": (shape(64, 3, 32, 0, 48, "fp32"), 0),
}


def _close(name, got, ref, dtype, g=1):
    assert np.all(np.isfinite(got)), name
    err = orc.max_abs_rel(got, ref)
    norm = np.linalg.norm(got - ref) / max(np.linalg.norm(ref), 1e-30)
    print("%-40s max-abs-rel %.2e  2-norm %.2e" % (name, err, norm), flush=True)
    assert err <= TOL[dtype], name
    if dtype == "bf16":
        assert norm <= {1: 5e-3, 4: 1.3e-2}[g], name


class Cache:
    """Planes whose rows lie in pages or back to back, every row that belongs to no sequence NaN, and the weights."""

    def __init__(self, name, lens, page, seed, spare_cols=1):
        self.sh, self.d_ck = SHAPES[name]
        sh, self.lens, self.page, self.dt = self.sh, lens, page, self.sh["dtype"]
        rng = self.rng = np.random.default_rng(seed)
        B, n_h, d_h, r, d_c = len(lens), sh["n_heads"], sh["head_dim"], sh["r"], sh["d_c"]
        dk, dv = (self.d_ck, d_c - self.d_ck) if self.d_ck else (d_c, d_c)
        self.idx = synth.draw_elite_idx(rng, n_h, d_h, r)
        self.W_uk = dev(rng.standard_normal((dk, n_h, d_h - 2 * r)) / dk ** 0.5, self.dt)
        self.W_uv = dev(rng.standard_normal((dv, n_h, d_h)) / dv ** 0.5, self.dt)
        self.dims = dims_of(sh)
        S = max(max(lens), 1)
        if page:
            need = [-(-n // page) for n in lens]
            self.cols = max(max(need), 1) + spare_cols
            self.n_pages = sum(need) + 2
            order = rng.permutation(self.n_pages)
            table = rng.integers(-5, self.n_pages + 5, (B, self.cols))       # entries past a sequence's pages: anything
            at = 0
            for b, n in enumerate(need):
                table[b, :n] = order[at:at + n]
                at += n
            self.table = table.astype(np.int32)
            rows, self.stride = self.n_pages * page, 0
            self.rows = [np.array([table[b, j // page] * page + j % page for j in range(n)], dtype=np.int64) for b, n in enumerate(lens)]
        else:
            self.stride = S + 3
            self.table, self.cols = None, 0
            rows = B * self.stride
            self.rows = [b * self.stride + np.arange(n) for b, n in enumerate(lens)]
        ke, c = np.full((rows, n_h, 2 * r), np.nan), np.full((rows, d_c), np.nan)
        for at in self.rows:
            ke[at], c[at] = rng.standard_normal((len(at), n_h, 2 * r)), rng.standard_normal((len(at), d_c))
        self.ke, self.c = dev(ke, self.dt), dev(c, self.dt)

    def queries(self, T):
        return dev(self.rng.standard_normal((len(self.lens), T, self.sh["n_heads"], self.sh["head_dim"])), self.dt)

    def reference(self, q, pos, seen):
        """seen[b]: [T, lens[b]] truth values"""
        ke, c, q = host64(self.ke), host64(self.c), host64(q)
        return np.stack([orc.seen_attn(q[b], pos[b], ke[at], c[at], seen[b], host64(self.W_uk), host64(self.W_uv), self.idx,
                                       self.sh["head_dim"], self.sh["rope_base"], self.d_ck) for b, at in enumerate(self.rows)])

    def blank(self, q):
        return torch.full_like(q, float("nan"))

    def paged(self, q, pos, kv, ns=0, max_seq=None, out=None, stream=None, ws=None):
        B, T = q.shape[:2]
        max_seq = max(max(self.lens), 1) if max_seq is None else max_seq
        out = self.blank(q) if out is None else out
        if ws is None:
            ws = torch.full((ekv.elitekv_paged_attn_workspace_bytes(self.dims, B, T, max_seq, ns, self.d_ck),), 0xFF, dtype=torch.uint8, device=DEV)
        ekv.elitekv_paged_attn(self.dims, q, i32(pos), i32(kv), max_seq, i32(self.table), self.page, self.W_uk, self.W_uv, i32(self.idx), self.ke,
                               self.c, out, ws, n_splits=ns, d_ck=self.d_ck, stream=stream)
        torch.cuda.synchronize()
        return out

    def tree(self, q, pos, prefix, nodes, sees, ns=0, max_seq=None):
        B, T = q.shape[:2]
        max_seq = max(max(self.lens), 1) if max_seq is None else max_seq
        out = self.blank(q)
        ws = torch.full((ekv.elitekv_tree_attn_workspace_bytes(self.dims, B, T, max_seq, ns, self.d_ck),), 0xFF, dtype=torch.uint8, device=DEV)
        mask = torch.from_numpy(orc.mask_words(sees).view(np.int32)).to(DEV)
        ekv.elitekv_tree_attn(self.dims, q, i32(pos), i32(prefix), i32(nodes), mask, max_seq, self.stride, self.W_uk, self.W_uv, i32(self.idx),
                              self.ke, self.c, out, ws, block_table=i32(self.table) if self.page else None, page_rows=self.page,
                              n_splits=ns, d_ck=self.d_ck)
        torch.cuda.synchronize()
        return out


# ---- attention over pages ----

@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("name", list(SHAPES))
def test_one_query_over_pages(name, page):
    print("one query over pages", name, page, flush=True)
    lens = [1, 0, 16, 17, 333, 64, 65, 15]
    k = Cache(name, lens, page, seed=len(name) + page)
    q = k.queries(1)
    pos = np.array([[max(n - 1, 0)] for n in lens])
    kv = np.array(lens)[:, None]
    ref = k.reference(q, pos, [np.ones((1, n), dtype=bool) for n in lens])
    for ns in (0, 1, 3):
        got = host64(k.paged(q, pos, kv, ns))
        _close("%s page %d splits %d" % (name, page, ns), got, ref, k.dt)
        assert np.all(got[1] == 0.0)


@pytest.mark.parametrize("name", ["7b", "13b", "12pct", "slrd", "fp32_tiled", "fp32_any"])
def test_several_queries_over_pages(name):
    print("several queries over pages", name, flush=True)
    lens, T = [70, 3, 260], 5
    k = Cache(name, lens, 32, seed=7)
    q = k.queries(T)
    kv = np.array([[max(n - T + t + 1, 0) for t in range(T)] for n in lens])
    pos = np.maximum(kv - 1, 0)
    ref = k.reference(q, pos, [np.arange(n)[None] < kv[b][:, None] for b, n in enumerate(lens)])
    for ns in (0, 2):
        got = host64(k.paged(q, pos, kv, ns))
        _close("%s splits %d" % (name, ns), got, ref, k.dt)
        assert np.all(got[kv == 0] == 0.0)


@pytest.mark.parametrize("name", ["7b", "fp32_tiled", "fp32_any"])
def test_lengths_past_the_table_and_the_bound_are_cut(name):
    lens = [64, 40]
    k = Cache(name, lens, 16, seed=3, spare_cols=0)        # four columns: 64 rows; the second sequence's last entry is anything
    k.table[1, 3] = k.n_pages + 3
    q, pos = k.queries(1), np.array([[500], [39]])
    full = [np.ones((1, n), dtype=bool) for n in lens]
    got = host64(k.paged(q, pos, [[1000], [40]], max_seq=4096))
    _close("cut by the table", got, k.reference(q, pos, full), k.dt)
    got = host64(k.paged(q, pos, [[1000], [-7]], max_seq=33))
    seen = [np.arange(64)[None] < 33, np.zeros((1, 40), dtype=bool)]
    _close("cut by the bound", got, k.reference(q, pos, seen), k.dt)
    assert np.all(got[1] == 0.0)


@pytest.mark.parametrize("name", ["7b", "13b", "12pct", "r16_72_heads", "slrd", "fp32_tiled", "fp32_any"])
def test_long_caches_and_peaked_scores(name):
    """Many tiles per work-group and a query four times as large: maxima rise in many tiles, and a tile lost or read twice shows.  One
    request alone as well."""
    print("long caches", name, flush=True)
    for lens, splits in (([3001, 1777], (0, 1, 7)), ([2500], (0, 1))):
        k = Cache(name, lens, 64, seed=51)
        q = k.queries(1) * 4
        pos = np.array([[n - 1] for n in lens])
        ref = k.reference(q, pos, [np.ones((1, n), dtype=bool) for n in lens])
        for ns in splits:
            _close("%s %s splits %d" % (name, lens, ns), host64(k.paged(q, pos, pos + 1, ns)), ref, k.dt, g=4)


@pytest.mark.parametrize("name", ["7b", "13b", "slrd", "fp32_tiled"])
def test_trees_over_long_caches(name):
    print("trees over long caches", name, flush=True)
    prefix, nodes, T = np.array([1990, 700]), np.array([9, 7]), 9
    lens = [int(p + n) for p, n in zip(prefix, nodes)]
    k = Cache(name, lens, 32, seed=52)
    q = k.queries(T) * 4
    sees = np.stack([orc.tree_sees(_random_tree(k.rng, T), n) for n in nodes])
    pos = prefix[:, None] + np.maximum(sees.sum(axis=2) - 1, 0)
    seen = []
    for b, n in enumerate(lens):
        s = np.zeros((T, n), dtype=bool)
        s[:nodes[b], :prefix[b]] = True
        s[:, prefix[b]:] = sees[b][:, :nodes[b]]
        seen.append(s)
    ref = k.reference(q, pos, seen)
    for ns in (0, 1, 5):
        _close("%s splits %d" % (name, ns), host64(k.tree(q, pos, prefix, nodes, sees, ns)), ref, k.dt, g=4)


@pytest.mark.parametrize("name,planes_gb", [("12pct", 5.0), ("fp32_tiled", 5.0), ("fp32_any", 5.0)])
def test_pages_beyond_four_gigabytes(name, planes_gb):
    """Planes of which both are larger than 2^32 bytes, the cached rows in their last pages; attention, and a commit among them."""
    print("beyond 4 GiB", name, flush=True)
    sh, _ = SHAPES[name]
    dt = torch.bfloat16 if sh["dtype"] == "bf16" else torch.float32
    e, page = dt.itemsize, 16
    rows = int(planes_gb * 2**30 / (min(2 * sh["r"] * sh["n_heads"], sh["d_c"]) * e)) // page * page
    lens = [40, 21]
    k = Cache(name, lens, page, seed=53)
    small_ke, small_c, old = k.ke, k.c, [r.copy() for r in k.rows]
    k.ke = torch.empty(rows, sh["n_heads"], 2 * sh["r"], dtype=dt, device=DEV)
    k.c = torch.empty(rows, sh["d_c"], dtype=dt, device=DEV)
    assert k.ke.numel() * e > 2**32 and k.c.numel() * e > 2**32
    shift = rows // page - k.n_pages
    need = [-(-n // page) for n in lens]
    for b, n in enumerate(need):
        k.table[b, :n] += shift
    k.rows = [r + shift * page for r in k.rows]
    for b in range(2):
        k.ke[torch.from_numpy(k.rows[b]).to(DEV)] = small_ke[torch.from_numpy(old[b]).to(DEV)]
        k.c[torch.from_numpy(k.rows[b]).to(DEV)] = small_c[torch.from_numpy(old[b]).to(DEV)]
    q, pos = k.queries(1), np.array([[n - 1] for n in lens])
    got = host64(k.paged(q, pos, pos + 1))
    big_ke, big_c, big_rows, k.ke, k.c, k.rows = k.ke, k.c, k.rows, small_ke, small_c, old
    _close(name, got, k.reference(q, pos, [np.ones((1, n), dtype=bool) for n in lens]), k.dt)
    path = np.zeros((2, 10), dtype=int)                    # (trees of ten nodes: an entry is a node below ten)
    path[0, :3], path[1, :2] = [3, 5, 9], [1, 2]
    ekv.elitekv_tree_commit(k.dims, i32(path), i32([3, 2]), i32([30, 17]), 0, big_ke, big_c, block_table=i32(k.table), page_rows=page)
    torch.cuda.synchronize()
    for b, (P, n) in enumerate([(30, 3), (17, 2)]):
        for i in range(n):
            to, of = int(big_rows[b][P + i]), int(old[b][P + path[b, i]])
            assert torch.equal(big_c[to], small_c[of]) and torch.equal(big_ke[to], small_ke[of])
    del big_ke, big_c
    torch.cuda.empty_cache()


def test_a_call_on_another_stream_and_pages_of_many_rows():
    lens = [1000, 77]
    k = Cache("7b", lens, 1024, seed=54)
    q, pos = k.queries(1), np.array([[n - 1] for n in lens])
    ref = k.reference(q, pos, [np.ones((1, n), dtype=bool) for n in lens])
    side = torch.cuda.Stream()
    out = k.blank(q)
    torch.cuda.synchronize()
    _close("by argument", host64(k.paged(q, pos, pos + 1, stream=side, out=out)), ref, k.dt)
    with torch.cuda.stream(side):
        _close("current", host64(k.paged(q, pos, pos + 1)), ref, k.dt)


def test_nothing_to_see():
    """A bound of zero rows, planes without a whole page, an empty batch."""
    k = Cache("7b", [40, 30], 64, seed=55)
    q, pos = k.queries(2), np.array([[38, 39], [28, 29]])
    assert torch.all(k.paged(q, pos, pos + 1, max_seq=0) == 0)
    out = k.blank(q)
    ws = torch.empty(ekv.elitekv_paged_attn_workspace_bytes(k.dims, 2, 2, 40), dtype=torch.uint8, device=DEV)
    ekv.elitekv_paged_attn(k.dims, q, i32(pos), i32(pos + 1), 40, i32(k.table), 64, k.W_uk, k.W_uv, i32(k.idx), k.ke, k.c, out, ws, plane_rows=63)
    torch.cuda.synchronize()
    assert torch.all(out == 0)
    ekv.elitekv_paged_attn(k.dims, q[:0], i32(pos[:0]), i32(pos[:0]), 40, i32(k.table[:0]), 64, k.W_uk, k.W_uv, i32(k.idx), k.ke, k.c, out, ws)


PROMPTS = {
    "7b": (shape(64, 32, 128, 8, 1536, "bf16"), 0),
    "r4": (shape(64, 16, 128, 4, 256, "bf16"), 0),
    "slrd": (shape(64, 16, 128, 8, 1536, "bf16"), 768),
}


@pytest.mark.parametrize("page", [16, 128])
@pytest.mark.parametrize("name", list(PROMPTS))
def test_prompts_over_pages(name, page, monkeypatch):
    """Many queries per sequence: rows gathered, keys and values rebuilt.  The same workspace then serves a bound of few rows, whose
    queries are absorbed, and a table too short for the bound."""
    print("prompts", name, page, flush=True)
    monkeypatch.setitem(SHAPES, name, PROMPTS[name])
    lens, T = [300, 61, 190], 70
    k = Cache(name, lens, page, seed=41)
    assert ekv.elitekv_prefill_plan(k.dims, 3, T, 300, 1 << 40, d_ck=k.d_ck) != ekv.PREFILL_ABSORBED
    q = k.queries(T)
    kv = np.array([[max(n - T + t + 1, 0) for t in range(T)] for n in lens])
    pos = np.maximum(kv - 1, 0)
    seen = lambda cut: [np.arange(n)[None] < np.minimum(kv[b], cut)[:, None] for b, n in enumerate(lens)]
    ws = torch.full((ekv.elitekv_paged_attn_workspace_bytes(k.dims, 3, T, 333, 0, k.d_ck),), 0xFF, dtype=torch.uint8, device=DEV)
    got = host64(k.paged(q, pos, kv, max_seq=333, ws=ws))
    _close("%s page %d" % (name, page), got, k.reference(q, pos, seen(333)), k.dt)
    assert np.all(got[kv == 0] == 0.0)
    got = host64(k.paged(q, pos, kv, max_seq=50, ws=ws))
    _close("%s page %d, 50 rows" % (name, page), got, k.reference(q, pos, seen(50)), k.dt)
    k.table = np.ascontiguousarray(k.table[:, :-(-200 // page)])
    cut = k.table.shape[1] * page
    got = host64(k.paged(q, pos, kv, max_seq=333, ws=ws))
    _close("%s page %d, short table" % (name, page), got, k.reference(q, pos, seen(cut)), k.dt)


def test_pages_in_order_give_the_bits_of_the_rows_back_to_back():
    sh, _ = SHAPES["7b"]
    lens, stride = [300, 129], 320
    k = Cache("7b", lens, 64, seed=5)
    planes_ke, planes_c = (torch.zeros(2 * stride, *p.shape[1:], dtype=p.dtype, device=DEV) for p in (k.ke, k.c))
    for b, at in enumerate(k.rows):
        planes_ke[b * stride:b * stride + lens[b]] = k.ke[torch.from_numpy(at).to(DEV)]
        planes_c[b * stride:b * stride + lens[b]] = k.c[torch.from_numpy(at).to(DEV)]
    q, pos = k.queries(1), np.array([[n - 1] for n in lens])
    got = k.paged(q, pos, [[n] for n in lens], ns=4)
    out = torch.empty(2, 32, 128, dtype=torch.bfloat16, device=DEV)
    ws = torch.empty(ekv.elitekv_decode_workspace_bytes(k.dims, 2, 300, 4), dtype=torch.uint8, device=DEV)
    ekv.elitekv_decode_attn(k.dims, q.reshape(2, 32, 128), i32(pos.reshape(-1)), i32(lens), 300, stride, k.W_uk, k.W_uv, i32(k.idx), planes_ke,
                            planes_c, out, ws, n_splits=4)
    torch.cuda.synchronize()
    norm = (got.reshape(-1).double() - out.reshape(-1).double()).norm() / out.double().norm()
    assert norm <= 5e-3


# ---- trees ----

def _random_tree(rng, T):
    return np.array([-1] + [int(rng.integers(max(0, t - 5), t)) if rng.random() < 0.9 else -1 for t in range(1, T)])


@pytest.mark.parametrize("page", [0, 16, 64])
@pytest.mark.parametrize("name", list(SHAPES))
def test_tree_attention(name, page):
    print("tree", name, page, flush=True)
    T = 19
    prefix, nodes = np.array([0, 37, 3, 250, 64]), np.array([19, 19, 0, 17, 1])
    lens = [int(p + max(n, 1)) for p, n in zip(prefix, nodes)]
    k = Cache(name, lens, page, seed=11 + page)
    q = k.queries(T)
    sees = np.stack([orc.tree_sees(_random_tree(k.rng, T), n) for n in nodes])
    pos = prefix[:, None] + np.maximum(sees.sum(axis=2) - 1, 0)
    seen = []
    for b, n in enumerate(lens):
        s = np.zeros((T, n), dtype=bool)
        s[:nodes[b], :prefix[b]] = True
        s[:, prefix[b]:prefix[b] + nodes[b]] = sees[b][:, :nodes[b]]
        seen.append(s)
    ref = k.reference(q, pos, seen)
    for ns in (0, 1, 4):
        got = host64(k.tree(q, pos, prefix, nodes, sees, ns))
        _close("%s page %d splits %d" % (name, page, ns), got, ref, k.dt)
        assert np.all(got[2] == 0.0) and np.all(got[3, 17:] == 0.0) and np.all(got[4, 1:] == 0.0)


@pytest.mark.parametrize("T", [1, 33, 64, 128])
@pytest.mark.parametrize("name", ["7b", "13b", "12pct", "slrd", "fp32_tiled", "fp32_any"])
def test_any_mask_and_rows_that_nobody_sees(name, T):
    """Masks without order, rows without a bit, whole tiles hidden, and NaN and infinities in every row that no query of the sequence sees;
    nodes that only some see hold large values."""
    print("any mask", name, T, flush=True)
    prefix, nodes = np.array([0, 21, 0]), np.array([T, T, T])
    lens = [int(p + T) for p in prefix]
    k = Cache(name, lens, 32, seed=T)
    q = k.queries(T)
    sees = k.rng.random((3, T, T)) < 0.3
    sees[0, :, :min(T - 1, 40)] = False                    # the first tiles of a sequence without a prefix: nothing seen
    sees[0, :, T - 1] = True
    sees[1, T // 2] = False                                # the prefix alone
    sees[2, 0] = False                                     # nothing at all
    sees[2, -1] = False
    hidden = k.rng.random((3, T)) < 0.2
    hidden[0, T - 1] = False
    sees &= ~hidden[:, None, :]
    for b in range(3):
        for j in np.flatnonzero(~sees[b].any(axis=0)):
            row = int(k.rows[b][prefix[b] + j])
            k.c[row] = float("nan") if j % 2 else float("inf")
            k.ke[row] = float("-inf") if j % 3 else float("nan")
    pos = prefix[:, None] + np.arange(T)[None]
    seen = [np.concatenate([np.ones((T, prefix[b]), dtype=bool), sees[b]], axis=1) for b in range(3)]
    ref = k.reference(q, pos, seen)
    for ns in (0, 1, 3):
        got = host64(k.tree(q, pos, prefix, nodes, sees, ns))
        _close("%s T %d splits %d" % (name, T, ns), got, ref, k.dt)
        for b in range(3):
            assert np.all(got[b][~seen[b].any(axis=1)] == 0.0)


# the kernels in fp32 arithmetic: one block of latent columns a wave, a last wave whose window is moved back and waves without blocks, the
# widest rows, elite keys that are not all requested ahead, separated latents whose boundary lies inside a wave's blocks
F32 = {
    "c16": (shape(64, 3, 64, 4, 16, "fp32"), 0),
    "c144": (shape(64, 5, 64, 4, 144, "fp32"), 0),
    "c576_r16": (shape(64, 17, 128, 16, 576, "fp32"), 0),
    "c2048": (shape(64, 32, 128, 8, 2048, "fp32"), 0),
    "c1536_r32": (shape(64, 18, 128, 32, 1536, "fp32"), 0),
    "c256_r48_head_256": (shape(64, 4, 256, 48, 256, "fp32"), 0),
    "slrd_48_of_208": (shape(64, 5, 64, 4, 208, "fp32"), 48),
    "slrd_768_of_1536": (shape(64, 32, 128, 8, 1536, "fp32"), 768),
    "bf16_c1040": (shape(64, 16, 128, 8, 1040, "bf16"), 0),
}


@pytest.mark.parametrize("T,page", [(2, 16), (11, 0), (37, 32)])
@pytest.mark.parametrize("name", list(F32))
def test_widths_in_fp32_arithmetic(name, T, page, monkeypatch):
    print("fp32 arithmetic", name, T, page, flush=True)
    monkeypatch.setitem(SHAPES, name, F32[name])
    prefix = np.array([260, 0, 33])
    nodes = np.array([T, T - 1, T])
    lens = [int(p + n) for p, n in zip(prefix, nodes)]
    k = Cache(name, lens, page, seed=71)
    q = k.queries(T)
    sees = np.stack([orc.tree_sees(_random_tree(k.rng, T), n) for n in nodes])
    pos = prefix[:, None] + np.maximum(sees.sum(axis=2) - 1, 0)
    seen = []
    for b, n in enumerate(lens):
        s = np.zeros((T, n), dtype=bool)
        s[:nodes[b], :prefix[b]] = True
        s[:, prefix[b]:] = sees[b][:, :nodes[b]]
        seen.append(s)
    ref = k.reference(q, pos, seen)
    for ns in (0, 1, 3, 40):
        got = host64(k.tree(q, pos, prefix, nodes, sees, ns))
        _close("%s T %d page %d splits %d" % (name, T, page, ns), got, ref, k.dt)
        assert np.all(got[1, T - 1:] == 0.0)


# two queries a work-group: the widths that are compiled, four and eight elite chunks, one and more groups of 32 heads
PAIRS = {
    "768_r4": (shape(64, 8, 128, 4, 768, "bf16"), 0),
    "768_r8_40_heads": (shape(64, 40, 128, 8, 768, "bf16"), 0),
    "512_r8": (shape(64, 8, 64, 8, 512, "bf16"), 0),
    "256_r4_33_heads": (shape(64, 33, 64, 4, 256, "bf16"), 0),
    "slrd_768": (shape(64, 8, 128, 8, 1536, "bf16"), 768),
    "slrd_512_r4_40_heads": (shape(64, 40, 128, 4, 1024, "bf16"), 512),
    "slrd_256": (shape(64, 5, 64, 8, 512, "bf16"), 256),
}


def _close_rows(name, got, ref):
    """Queries one by one: a tile lost for one query among hundreds is not in the norm of all."""
    norms = np.linalg.norm((got - ref).reshape(*got.shape[:2], -1), axis=2) / np.maximum(np.linalg.norm(ref.reshape(*got.shape[:2], -1), axis=2), 1e-30)
    assert norms.max() <= 1.5e-2, (name, np.unravel_index(norms.argmax(), norms.shape), norms.max())


@pytest.mark.parametrize("T,page", [(128, 16), (127, 64), (127, 0)])
@pytest.mark.parametrize("name", list(PAIRS))
def test_pairs_of_queries(name, T, page, monkeypatch):
    """Masks that differ from query to query, nodes that see the prefix alone or nothing, an odd last query, and rows of NaN that one
    query of a pair sees and the other does not.  One query's norm: sqrt(5) x 2^-8 / sqrt(3) x 0.72 = 3.6e-3 on average, four times that at
    most."""
    print("pairs", name, T, page, flush=True)
    monkeypatch.setitem(SHAPES, name, PAIRS[name])
    prefix, nodes = np.array([490, 0, 333]), np.array([T, T - 3, T])
    lens = [int(p + n) for p, n in zip(prefix, nodes)]
    k = Cache(name, lens, page, seed=T + page)
    q = k.queries(T)
    sees = np.stack([orc.tree_sees(_random_tree(k.rng, T), n) for n in nodes])
    sees[2] = k.rng.random((T, T)) < 0.4
    sees[2, 10] = sees[2, 11] = sees[2, 40] = False
    for node in (6, 51):                                   # seen by one query alone
        sees[2, :, node] = False
        sees[2, node, node] = True
        row = int(k.rows[2][prefix[2] + node])
        k.c[row], k.ke[row] = float("nan"), float("inf")
    pos = prefix[:, None] + np.maximum(sees.sum(axis=2) - 1, 0)
    seen = []
    for b, n in enumerate(lens):
        s = np.zeros((T, n), dtype=bool)
        s[:nodes[b], :prefix[b]] = True
        s[:, prefix[b]:] = sees[b][:, :nodes[b]]
        seen.append(s)
    with np.errstate(invalid="ignore"):
        ref = k.reference(q, pos, seen)
    bound = -(-(12 * 256) // (3 * ((T + 1) // 2))) * 32    # tiles enough for two queries a work-group
    for ns in (0, 1, 2, 5):
        got = host64(k.tree(q, pos, prefix, nodes, sees, ns, max_seq=max(bound, max(lens)) if not page else None))
        for node in (6, 51):
            assert not np.any(np.isfinite(got[2, node])), node
            got[2, node] = ref[2, node] = 0.0
        _close("%s T %d page %d splits %d" % (name, T, page, ns), got, ref, k.dt)
        _close_rows(name, got, ref)
        assert np.all(got[1, T - 3:] == 0.0)


@pytest.mark.parametrize("name", ["768_r4", "512_r8", "slrd_768", "slrd_256"])
def test_pairs_of_queries_over_pages(name, monkeypatch):
    """Drafted chains: every query sees one row more than the one before it, from none to all."""
    monkeypatch.setitem(SHAPES, name, PAIRS[name])
    T, lens = 47, [1200, 47, 700, 33]
    k = Cache(name, lens, 32, seed=81)
    q = k.queries(T)
    kv = np.array([[max(n - T + t + 1, 0) for t in range(T)] for n in lens])
    pos = np.maximum(kv - 1, 0)
    ref = k.reference(q, pos, [np.arange(n)[None] < kv[b][:, None] for b, n in enumerate(lens)])
    for ns in (0, 1, 7):
        got = host64(k.paged(q, pos, kv, ns))
        _close("%s splits %d" % (name, ns), got, ref, k.dt)
        _close_rows(name, got, ref)
        assert np.all(got[kv == 0] == 0.0)


def test_pairs_of_queries_replay_from_a_graph(monkeypatch):
    """A captured call replayed between the program's own work, with other trees and lengths in its arrays: every replay is the eager call."""
    name, T = "768_r4", 64
    monkeypatch.setitem(SHAPES, name, PAIRS[name])
    lens = [900, 300, 64, 1100]
    k = Cache(name, lens, 16, seed=91)
    q = k.queries(T)
    bound = 1600                                           # 128 pairs x 50 tiles: two queries a work-group
    prefix, nodes = i32([0] * 4), i32([0] * 4)
    pos, mask = i32(np.zeros((4, T))), i32(np.zeros((4, T, 2)))
    out = k.blank(q)
    ws = torch.full((ekv.elitekv_tree_attn_workspace_bytes(k.dims, 4, T, bound),), 0xFF, dtype=torch.uint8, device=DEV)
    args = (k.dims, q, pos, prefix, nodes, mask, bound, 0, k.W_uk, k.W_uv, i32(k.idx), k.ke, k.c, out, ws)
    table = i32(k.table)
    call = lambda: ekv.elitekv_tree_attn(*args, block_table=table, page_rows=16)
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for seed in range(3):
        rng = np.random.default_rng(seed)
        n = rng.integers(1, T + 1, 4)
        sees = np.stack([orc.tree_sees(_random_tree(rng, T), int(m)) for m in n])
        nodes.copy_(i32(n))
        prefix.copy_(i32(np.array(lens) - n))
        pos.copy_(i32((np.array(lens) - n)[:, None] + np.maximum(sees.sum(axis=2) - 1, 0)))
        mask.copy_(torch.from_numpy(orc.mask_words(sees).view(np.int32)).to(DEV))
        out.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        replayed = out.clone()
        out.fill_(float("nan"))
        call()
        torch.cuda.synchronize()
        assert torch.equal(replayed, out) and torch.all(torch.isfinite(out.float()))
        assert torch.all(out[0, int(n[0]):] == 0) and torch.any(out[0, 0] != 0)


MANY = {
    "72_heads": (shape(64, 72, 128, 16, 256, "bf16"), 0),
    "head_64": (shape(64, 72, 64, 4, 128, "bf16"), 0),
    "slrd_320": (shape(64, 64, 128, 4, 640, "bf16"), 320),
}


@pytest.mark.parametrize("name", list(MANY))
def test_many_rows(name, monkeypatch):
    """Enough rows and heads for the merge that keeps its sum in the accumulators, with one to four splits, a last stage of 64 latent
    columns and rows past the last; five splits take the other one."""
    print("many rows", name, flush=True)
    monkeypatch.setitem(SHAPES, name, MANY[name])
    T, prefix = 100, np.array([60, 0, 33])
    nodes = np.array([100, 97, 100])
    lens = [int(p + n) for p, n in zip(prefix, nodes)]
    k = Cache(name, lens, 16, seed=61)
    q = k.queries(T)
    sees = np.stack([orc.tree_sees(_random_tree(k.rng, T), n) for n in nodes])
    pos = prefix[:, None] + np.maximum(sees.sum(axis=2) - 1, 0)
    seen = []
    for b, n in enumerate(lens):
        s = np.zeros((T, n), dtype=bool)
        s[:nodes[b], :prefix[b]] = True
        s[:, prefix[b]:] = sees[b][:, :nodes[b]]
        seen.append(s)
    ref = k.reference(q, pos, seen)
    for ns in (1, 2, 3, 4, 5):
        got = host64(k.tree(q, pos, prefix, nodes, sees, ns))
        _close("%s splits %d" % (name, ns), got, ref, k.dt)
        assert np.all(got[1, 97:] == 0.0)


@pytest.mark.parametrize("name", ["7b", "fp32_tiled", "fp32_any"])
def test_a_tree_past_the_bound_is_cut(name):
    prefix, nodes, T = np.array([40, 90]), np.array([9, 9]), 9
    lens = [49, 99]
    k = Cache(name, lens, 0, seed=21)
    q = k.queries(T)
    sees = np.tril(np.ones((2, T, T), dtype=bool))
    pos = prefix[:, None] + np.arange(T)[None]
    got = host64(k.tree(q, pos, prefix, nodes, sees, max_seq=45))
    seen = [np.concatenate([np.ones((T, prefix[b]), dtype=bool), sees[b]], axis=1) & (np.arange(lens[b])[None] < 45) for b in range(2)]
    _close("cut", got, k.reference(q, pos, seen), k.dt)


def test_bits_past_the_nodes_do_not_count():
    prefix, nodes, T = np.array([20]), np.array([5]), 40
    k = Cache("7b", [25], 16, seed=22)
    q = k.queries(T)
    sees = np.ones((1, T, T), dtype=bool)
    pos = np.full((1, T), 24)
    got = host64(k.tree(q, pos, prefix, nodes, sees, max_seq=60))
    seen = np.zeros((T, 25), dtype=bool)
    seen[:5] = True
    _close("bits", got, k.reference(q, pos, [seen]), k.dt)


# ---- plans ----

def _server(rng, B, cols, n_pages, held_most):
    held = rng.integers(0, held_most + 1, B)
    order = rng.permutation(n_pages)
    table = np.full((B, cols), -1)
    at = 0
    for b in range(B):
        held[b] = min(held[b], n_pages - at)
        table[b, :held[b]] = order[at:at + held[b]]
        at += held[b]
    first = int(rng.integers(0, 5 * n_pages))
    free = np.full(n_pages, -9)
    for i, p in enumerate(order[at:]):
        free[(first + i) % n_pages] = p
    return table, held, free, np.array([first, first + n_pages - at])


def _plan(cached, new, T, page, n_pages, table, held, free, span, same=False):
    B = len(cached)
    t, h, f, s = i32(table), i32(held), i32(free), i64(span)
    h2, s2 = (h, s) if same else (torch.full_like(h, -5), torch.full_like(s, -5))
    pos, kv = (torch.full((B, T), -77, dtype=torch.int32, device=DEV) for _ in range(2))
    slot = torch.full((B, T), -77, dtype=torch.int64, device=DEV)
    ws = torch.full((ekv.elitekv_page_plan_workspace_bytes(B, T),), 0xFF, dtype=torch.uint8, device=DEV)
    ekv.elitekv_page_plan(i32(cached), i32(new), page, n_pages, t, h, h2, f, s, s2, pos, slot, kv, ws)
    torch.cuda.synchronize()
    return [a.cpu().numpy() for a in (t, h2, f, s2, pos, slot, kv)]


@pytest.mark.parametrize("same", [False, True])
@pytest.mark.parametrize("B,T,page", [(1, 1, 16), (7, 3, 16), (64, 1, 64), (1000, 4, 32), (1024, 5, 16), (1500, 1, 64), (3, 2047, 16), (300, 40, 16)])
def test_page_plan(B, T, page, same):
    print("plan", B, T, page, same, flush=True)
    rng = np.random.default_rng(B + T)
    S = 3 * T + 200
    cols = -(-S // page)
    for pool in (B * cols + 3, max(B * cols // 3, 2)):     # room for all, and too little
        table, held, free, span = _server(rng, B, cols, pool, cols // 2)
        cached = rng.integers(0, S - T, B) * (rng.random(B) < 0.8)
        new = rng.integers(-1, T + 3, B)
        cached[rng.random(B) < 0.05] = -4
        want = orc.page_plan(cached, new, T, page, pool, table, held, free, span)
        got = _plan(cached, new, T, page, pool, table, held, free, span, same)
        for g, w, what in zip(got, want, ("table", "held", "free", "span", "pos", "slot", "kv_len")):
            np.testing.assert_array_equal(g, w, err_msg=what)


def test_page_plan_of_requests_longer_than_their_tables():
    cached, new = np.array([100, 2**31 - 1, 5]), np.array([3, 3, 200])
    table, held, free, span = np.full((3, 2), -1), np.zeros(3, int), np.arange(20), np.array([0, 20])
    want = orc.page_plan(cached, new, 200, 16, 20, table, held, free, span)
    got = _plan(cached, new, 200, 16, 20, table, held, free, span)
    want[4][1] = want[4][1].astype(np.int32)               # (a position past 31 bits: the token has no row)
    for g, w in zip(got, want):
        np.testing.assert_array_equal(g, w)
    assert (got[5][1] == -1).all() and (got[5][2, 27:] == -1).all() and got[5][2, 26] >= 0


@pytest.mark.parametrize("B,T", [(1, 1), (3, 7), (2, 32), (5, 33), (300, 64), (2, 100), (9, 128)])
def test_tree_plan(B, T):
    rng = np.random.default_rng(T)
    parent = np.stack([_random_tree(rng, T) for _ in range(B)])
    parent[0] = np.arange(T) - 1                           # a chain
    if B > 1:
        parent[1] = rng.integers(-3, T + 3, T)             # anything: entries that are no earlier node are roots
    nodes = rng.integers(-1, T + 2, B)
    nodes[0] = T
    prefix = rng.integers(0, 100000, B)
    pos = torch.full((B, T), -77, dtype=torch.int32, device=DEV)
    mask = torch.full((B, T, -(-T // 32)), -77, dtype=torch.int32, device=DEV)
    ekv.elitekv_tree_plan(i32(parent), i32(prefix), i32(nodes), pos, mask)
    torch.cuda.synchronize()
    sees = np.stack([orc.tree_sees(parent[b], int(np.clip(nodes[b], 0, T))) for b in range(B)])
    np.testing.assert_array_equal(mask.cpu().numpy().view(np.uint32), orc.mask_words(sees))
    depth = sees.sum(axis=2) - 1
    np.testing.assert_array_equal(pos.cpu().numpy(), np.where(depth >= 0, prefix[:, None] + depth, 0))


# ---- the accepted path ----

@pytest.mark.parametrize("page", [0, 16])
@pytest.mark.parametrize("name", ["7b", "13b", "fp32_any", "bf16_any_slrd", "fp32_r0"])
def test_commit(name, page):
    T = 30
    prefix = np.array([5, 0, 40, 7, 12])
    lens = [int(p + T) for p in prefix]
    k = Cache(name, lens, page, seed=31)
    path = np.full((5, T), -1)
    chosen = [[0, 2, 3, 9, 10, 11, 12, 20, 21, 29], list(range(T)), [], [29], [4, 1, 3, 77, -2, 29, 8]]
    for b, c in enumerate(chosen):
        path[b, :len(c)] = c
    n = [len(c) for c in chosen]
    n[1], n[2] = T + 5, -3                                 # lengths past the array and below zero
    want_ke, want_c = k.ke.clone(), k.c.clone()
    for b, c in enumerate(chosen):
        for i, node in enumerate(c):
            if i <= node < T:
                to, of = int(k.rows[b][prefix[b] + i]), int(k.rows[b][prefix[b] + node])
                want_ke[to], want_c[to] = k.ke[of], k.c[of]
    ekv.elitekv_tree_commit(k.dims, i32(path), i32(n), i32(prefix), k.stride, k.ke, k.c, block_table=i32(k.table) if page else None, page_rows=page)
    torch.cuda.synchronize()
    whole = torch.int16 if k.dt == "bf16" else torch.int32
    assert torch.equal(k.ke.view(whole), want_ke.view(whole)) and torch.equal(k.c.view(whole), want_c.view(whole))


def test_commit_stays_inside_a_sequences_rows():
    k = Cache("fp32_any", [20, 20], 0, seed=33)            # 23 rows each
    path, before = np.array([[1, 2, 3, 4, 5]] * 2), k.c.clone()
    ekv.elitekv_tree_commit(k.dims, i32(path), i32([5, 5]), i32([20, 44]), k.stride, k.ke, k.c)
    torch.cuda.synchronize()
    want = before.clone()
    want[20:22] = before[21:23]                            # rows 23 and up are the next sequence's; 44 is past the second one's
    assert torch.equal(k.c.nan_to_num(7.0), want.nan_to_num(7.0))


# ---- together ----

@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_a_server_drafts_verifies_and_commits(dtype):
    """Requests come and go; each step drafts a tree per request, verifies it over the pages, keeps a path.  At the end every request's
    cache is, row by row, what appending its tokens one after the other gives, and a decode over the pages is a decode over those rows."""
    sh = shape(64, 4, 64, 4, 128, dtype)
    rng, idx, W_ke, W_dkv, W_uk, W_uv, _, _ = _draw(sh, 1, 1, 77)
    dims = dims_of(sh)
    Wked, Wdkvd, Wukd, Wuvd, idxd = dev(W_ke, dtype), dev(W_dkv, dtype), dev(W_uk, dtype), dev(W_uv, dtype), i32(idx)
    B, T, page, n_pages, cols = 3, 7, 16, 20, 6
    ke = torch.zeros(n_pages * page, 4, 8, dtype=ekv.torch_dtype(dims), device=DEV)
    c = torch.zeros(n_pages * page, 128, dtype=ekv.torch_dtype(dims), device=DEV)
    table, held = i32(np.zeros((B, cols))), i32(np.zeros(B))
    free, span = i32(np.arange(n_pages)), i64([0, n_pages])
    cached, zero = i32([0, 0, 0]), i32([0, 0, 0])
    history = [[] for _ in range(B)]                       # the hidden states of every request's kept tokens
    pos, kv = (torch.zeros(B, T, dtype=torch.int32, device=DEV) for _ in range(2))
    slot, tree_pos = torch.zeros(B, T, dtype=torch.int64, device=DEV), torch.zeros(B, T, dtype=torch.int32, device=DEV)
    mask = torch.zeros(B, T, 1, dtype=torch.int32, device=DEV)
    pws = torch.empty(ekv.elitekv_page_plan_workspace_bytes(B, T), dtype=torch.uint8, device=DEV)
    aws = torch.empty(max(ekv.elitekv_append_workspace_bytes(dims, B * T), 16), dtype=torch.uint8, device=DEV)
    tws = torch.empty(ekv.elitekv_tree_attn_workspace_bytes(dims, B, T, cols * page), dtype=torch.uint8, device=DEV)
    for step in range(9):
        if step == 5:                                      # the second request ends and another takes its place
            cached[1] = 0
            history[1] = []
            ekv.elitekv_page_plan(cached, zero, page, n_pages, table, held, held, free, span, span, pos, slot, kv, pws)
        nodes = i32(rng.integers(1, T + 1, B))
        parent = np.stack([_random_tree(rng, T) for _ in range(B)])
        x = dev(rng.standard_normal((B * T, 64)), dtype)
        q = dev(rng.standard_normal((B, T, 4, 64)), dtype)
        ekv.elitekv_page_plan(cached, nodes, page, n_pages, table, held, held, free, span, span, pos, slot, kv, pws)
        ekv.elitekv_tree_plan(i32(parent), cached, nodes, tree_pos, mask)
        ekv.elitekv_append(dims, x, tree_pos, slot, Wked, Wdkvd, idxd, ke, c, ws=aws)
        out = torch.full_like(q, float("nan"))
        ekv.elitekv_tree_attn(dims, q, tree_pos, cached, nodes, mask, cols * page, 0, Wukd, Wuvd, idxd, ke, c, out, tws, block_table=table,
                              page_rows=page)
        torch.cuda.synchronize()
        paths, n = np.zeros((B, T), dtype=int), []
        for b in range(B):
            leaf = int(rng.integers(0, int(nodes[b])))
            path = np.flatnonzero(orc.tree_sees(parent[b], T)[leaf])
            rows = np.concatenate([np.array(history[b]).reshape(-1, 64), host64(x).reshape(B, T, 64)[b][path]])
            ke64, c64 = orc.append(rows, np.arange(len(rows)), host64(Wked), host64(Wdkvd), idx, 64, sh["rope_base"])
            ref = orc.decode_attn(host64(q)[b, leaf][None], [len(rows) - 1], [ke64], [c64], [len(rows)], host64(Wukd), host64(Wuvd), idx, 64,
                                  sh["rope_base"])[0]
            assert orc.max_abs_rel(host64(out)[b, leaf], ref) <= TOL[dtype]
            paths[b, :len(path)] = path
            n.append(len(path))
            history[b] = list(rows)
        ekv.elitekv_tree_commit(dims, i32(paths), i32(n), cached, 0, ke, c, block_table=table, page_rows=page)
        cached += i32(n)
    assert [int(v) for v in cached] == [len(h) for h in history]
    ekv.elitekv_page_plan(cached, zero, page, n_pages, table, held, held, free, span, span, pos, slot, kv, pws)
    torch.cuda.synchronize()
    used = [int(table[b, i]) for b in range(B) for i in range(int(held[b]))]
    spare = [int(free[i % n_pages]) for i in range(int(span[0]), int(span[1]))]
    assert sorted(used + spare) == list(range(n_pages)) and [int(v) for v in held] == [-(-len(h) // page) for h in history]
    q = dev(rng.standard_normal((B, 1, 4, 64)), dtype)
    last = np.array([[len(h) - 1] for h in history])
    out = torch.full_like(q, float("nan"))
    ws = torch.empty(ekv.elitekv_paged_attn_workspace_bytes(dims, B, 1, cols * page), dtype=torch.uint8, device=DEV)
    ekv.elitekv_paged_attn(dims, q, i32(last), i32(last + 1), cols * page, table, page, Wukd, Wuvd, idxd, ke, c, out, ws)
    torch.cuda.synchronize()
    for b in range(B):
        rows = [int(table[b, j // page]) * page + j % page for j in range(len(history[b]))]
        ke64, c64 = orc.append(np.array(history[b]), np.arange(len(rows)), host64(Wked), host64(Wdkvd), idx, 64, sh["rope_base"])
        assert orc.max_abs_rel(host64(ke)[rows], ke64) <= TOL[dtype] and orc.max_abs_rel(host64(c)[rows], c64) <= TOL[dtype]
        ref = orc.decode_attn(host64(q)[b], [len(rows) - 1], [ke64], [c64], [len(rows)], host64(Wukd), host64(Wuvd), idx, 64, sh["rope_base"])
        assert orc.max_abs_rel(host64(out)[b], ref) <= TOL[dtype]


def test_a_step_replays_from_a_graph_and_its_books_advance():
    """Plan, append, tree attention and commit captured once; every replay advances the same books in place and gives the eager result."""
    sh = shape(64, 32, 128, 8, 1536, "bf16")
    rng, idx, W_ke, W_dkv, W_uk, W_uv, _, _ = _draw(sh, 1, 1, 78)
    dims = dims_of(sh)
    w = [dev(a, "bf16") for a in (W_ke, W_dkv, W_uk, W_uv)]
    idxd = i32(idx)
    B, T, page, n_pages, cols = 2, 5, 16, 40, 20
    parent = i32([[-1, 0, 0, 1, 2], [-1, 0, 1, 2, 3]])
    nodes, path, n = i32([5, 4]), i32([[0, 2, 4, 0, 0], [0, 1, 0, 0, 0]]), i32([3, 2])

    def fresh():
        return dict(ke=torch.zeros(n_pages * page, 32, 16, dtype=torch.bfloat16, device=DEV), c=torch.zeros(n_pages * page, 1536, dtype=torch.bfloat16, device=DEV),
                    table=i32(np.zeros((B, cols))), held=i32([0, 0]), free=i32(np.arange(n_pages)), span=i64([0, n_pages]), cached=i32([0, 0]),
                    x=torch.zeros(B * T, 64, dtype=torch.bfloat16, device=DEV), q=torch.zeros(B, T, 32, 128, dtype=torch.bfloat16, device=DEV),
                    out=torch.zeros(B, T, 32, 128, dtype=torch.bfloat16, device=DEV), pos=torch.zeros(B, T, dtype=torch.int32, device=DEV),
                    kv=torch.zeros(B, T, dtype=torch.int32, device=DEV), slot=torch.zeros(B, T, dtype=torch.int64, device=DEV),
                    tpos=torch.zeros(B, T, dtype=torch.int32, device=DEV), mask=torch.zeros(B, T, 1, dtype=torch.int32, device=DEV),
                    pws=torch.empty(ekv.elitekv_page_plan_workspace_bytes(B, T), dtype=torch.uint8, device=DEV),
                    aws=torch.empty(max(ekv.elitekv_append_workspace_bytes(dims, B * T), 16), dtype=torch.uint8, device=DEV),
                    tws=torch.empty(ekv.elitekv_tree_attn_workspace_bytes(dims, B, T, cols * page), dtype=torch.uint8, device=DEV))

    def step(s):
        ekv.elitekv_page_plan(s["cached"], nodes, page, n_pages, s["table"], s["held"], s["held"], s["free"], s["span"], s["span"], s["pos"],
                              s["slot"], s["kv"], s["pws"])
        ekv.elitekv_tree_plan(parent, s["cached"], nodes, s["tpos"], s["mask"])
        ekv.elitekv_append(dims, s["x"], s["tpos"], s["slot"], w[0], w[1], idxd, s["ke"], s["c"], ws=s["aws"])
        ekv.elitekv_tree_attn(dims, s["q"], s["tpos"], s["cached"], nodes, s["mask"], cols * page, 0, w[2], w[3], idxd, s["ke"], s["c"], s["out"],
                              s["tws"], block_table=s["table"], page_rows=page)
        ekv.elitekv_tree_commit(dims, path, n, s["cached"], 0, s["ke"], s["c"], block_table=s["table"], page_rows=page)
        s["cached"].add_(n)

    eager, graphed = fresh(), fresh()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        step(fresh())                                      # warm-up on the capture stream
        side.synchronize()
        with torch.cuda.graph(graph, stream=side):
            step(graphed)
    torch.cuda.synchronize()
    for rep in range(12):
        x, q = dev(rng.standard_normal((B * T, 64)), "bf16"), dev(rng.standard_normal((B, T, 32, 128)), "bf16")
        for s in (eager, graphed):
            s["x"].copy_(x)
            s["q"].copy_(q)
            s["tws"].fill_(0xFF)
            s["aws"].fill_(0xFF)
        torch.cuda.synchronize()
        step(eager)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for key in ("out", "table", "held", "free", "span", "cached", "ke", "c", "pos", "slot", "kv", "tpos", "mask"):
            assert torch.equal(eager[key], graphed[key]), "replay %d: %s" % (rep, key)
    assert [int(v) for v in graphed["cached"]] == [36, 24]
