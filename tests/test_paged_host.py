"""Refusals and sizes of the paged cache's and the trees' entry points, none of which reaches a GPU."""
import ctypes as C

import pytest

import paper_2503_01586_amd as ekv

lib = ekv.raw()
FAKE = 0x10000


def _dims(**kw):
    base = dict(d_model=128, n_heads=4, head_dim=32, r=2, d_c=64, dtype="fp32", rope_base=10000.0)
    base.update(kw)
    return ekv.make_dims(**base)


def _plan(**kw):
    a = dict(cached=FAKE, new=FAKE, B=2, T=3, page=16, n_pages=8, table=FAKE, cols=4, held=FAKE, held_out=FAKE, free=FAKE, span=FAKE,
             span_out=FAKE, pos=FAKE, slot=FAKE, kv=FAKE, ws=FAKE, wsb=1 << 20)
    a.update(kw)
    return lib.elitekv_page_plan(*a.values(), None)


def test_page_plan_refusals():
    assert _plan(B=0) == ekv.OK
    for bad in (dict(B=-1), dict(T=0), dict(page=0), dict(page=8), dict(page=48), dict(page=-16), dict(page=1 << 21), dict(n_pages=0),
                dict(cols=0)):
        assert _plan(**bad) == ekv.EINVAL, bad
    assert _plan(B=65536) == ekv.EUNSUPPORTED and _plan(T=65537) == ekv.EUNSUPPORTED
    for k in ("cached", "new", "table", "held", "held_out", "free", "span", "span_out", "pos", "slot", "kv", "ws"):
        assert _plan(**{k: None}) == ekv.ENULL, k
    assert _plan(ws=FAKE + 8) == ekv.EALIGN
    assert _plan(wsb=ekv.elitekv_page_plan_workspace_bytes(2, 3) // 256 * 16) == ekv.EWORKSPACE
    sizes = [ekv.elitekv_page_plan_workspace_bytes(B, 3) for B in (1, 7, 1024, 65535)]
    assert sizes == sorted(sizes) and sizes[0] > 0
    assert ekv.elitekv_page_plan_workspace_bytes(0, 3) == ekv.elitekv_page_plan_workspace_bytes(65536, 3) == 0


def _paged(d, **kw):
    a = dict(d_ck=0, q=FAKE, q_pos=FAKE, kv=FAKE, B=2, T=3, max_seq=128, table=FAKE, cols=8, page=16, W_uk=FAKE, W_uv=FAKE, idx=FAKE,
             ke=FAKE, c=FAKE, rows=256, out=FAKE, ws=FAKE, wsb=1 << 30, ns=0)
    a.update(kw)
    return lib.elitekv_paged_attn(C.byref(d) if d else None, *a.values(), None)


@pytest.mark.parametrize("shape", [dict(), dict(d_model=64, n_heads=32, head_dim=128, r=8, d_c=1536, dtype="bf16")])
def test_paged_attn_refusals(shape):
    d = _dims(**shape)
    assert _paged(None) == ekv.ENULL
    assert _paged(d, B=0) == ekv.OK
    for bad in (dict(B=-1), dict(T=0), dict(page=0), dict(page=17), dict(page=24), dict(cols=0), dict(cols=-1), dict(rows=-1),
                dict(max_seq=-1), dict(ns=-1), dict(d_ck=d.d_c), dict(d_ck=-1)):
        assert _paged(d, **bad) == ekv.EINVAL, bad
    for bad in (dict(B=300, T=300, max_seq=60), dict(B=1 << 40, T=1 << 40), dict(T=(1 << 24) + 1), dict(ns=4096)):
        assert _paged(d, **bad) == ekv.EUNSUPPORTED, bad
    for k in ("q", "q_pos", "kv", "table", "W_uk", "W_uv", "idx", "ke", "c", "out", "ws"):
        assert _paged(d, **{k: None}) == ekv.ENULL, k
    for k in ("q", "W_uk", "W_uv", "ke", "c", "out", "ws"):
        assert _paged(d, **{k: FAKE + 8}) == ekv.EALIGN, k
    assert _paged(_dims(head_dim=31)) == ekv.EINVAL
    assert _paged(d, wsb=64) == ekv.EWORKSPACE
    for d_ck in (0, d.d_c // 2):
        sizes = [ekv.elitekv_paged_attn_workspace_bytes(d, 2, 3, s, d_ck=d_ck) for s in (1, 16, 100, 128, 5000)]
        assert sizes == sorted(sizes) and sizes[0] > 0
    assert ekv.elitekv_paged_attn_workspace_bytes(d, 2, 0, 128) == 0
    assert ekv.elitekv_paged_attn_workspace_bytes(d, 300, 300, 60) == 0


def test_a_table_with_gaps_between_its_rows_is_refused():
    import torch
    d, t = _dims(), torch.zeros(2, 8, dtype=torch.int32)
    q, planes = torch.zeros(2, 1, 4, 32), torch.zeros(64, 64)
    with pytest.raises(ValueError):
        ekv.elitekv_paged_attn(d, q, t, t, 16, t[:, :4], 16, q, q, t, planes, planes, q, None, stream=0)
    with pytest.raises(ValueError):
        ekv.elitekv_tree_commit(d, t, t, t, 0, planes, planes, block_table=t[:, ::2], page_rows=16, stream=0)


def test_prompt_workspaces():
    """Many queries: room for the gathered rows and what the prefill's kernels need; a size serves every shorter bound."""
    d = ekv.make_dims(64, 32, 128, 8, 1536, "bf16")
    for d_ck in (0, 768):
        sizes = [ekv.elitekv_paged_attn_workspace_bytes(d, 2, 100, s, d_ck=d_ck) for s in (1, 64, 65, 100, 512, 513, 4000)]
        assert sizes == sorted(sizes)
        need = 2 * 4000 * (2 * 8 * 32 + 1536) * 2 + 2 * 4000 * 32 * 240 * 2
        assert need <= sizes[-1]
        small = dict(B=2, T=100, max_seq=4000, cols=63, page=64, rows=1 << 20, d_ck=d_ck)
        assert _paged(d, **small, wsb=need - 1) == ekv.EWORKSPACE
        for k in ("q", "q_pos", "kv", "table", "W_uk", "W_uv", "idx", "ke", "c", "out", "ws"):
            assert _paged(d, **{**small, k: None}) == ekv.ENULL, k
        for k in ("q", "W_uk", "W_uv", "ke", "c", "out", "ws"):
            assert _paged(d, **{**small, k: FAKE + 8}) == ekv.EALIGN, k
    assert _paged(d, B=60000, T=1000, max_seq=4000, cols=63, page=64) == ekv.EUNSUPPORTED


def _tree(d, **kw):
    a = dict(d_ck=0, q=FAKE, q_pos=FAKE, prefix=FAKE, nodes=FAKE, mask=FAKE, B=2, T=3, max_seq=128, stride=128, table=None, cols=0, page=0,
             W_uk=FAKE, W_uv=FAKE, idx=FAKE, ke=FAKE, c=FAKE, rows=256, out=FAKE, ws=FAKE, wsb=1 << 30, ns=0)
    a.update(kw)
    return lib.elitekv_tree_attn(C.byref(d) if d else None, *a.values(), None)


def test_tree_attn_refusals():
    d = _dims()
    assert _tree(None) == ekv.ENULL
    assert _tree(d, B=0) == ekv.OK
    pages = dict(table=FAKE, cols=8, page=16)
    for bad in (dict(B=-1), dict(T=0), dict(stride=-1), dict(rows=-1), dict(max_seq=-1), dict(pages, page=8), dict(pages, cols=0)):
        assert _tree(d, **bad) == ekv.EINVAL, bad
    for bad in (dict(T=129), dict(B=1000, T=128), dict(B=1 << 62)):
        assert _tree(d, **bad) == ekv.EUNSUPPORTED, bad
    for k in ("q", "q_pos", "prefix", "nodes", "mask", "W_uk", "W_uv", "idx", "ke", "c", "out", "ws"):
        assert _tree(d, **{k: None}) == ekv.ENULL, k
    assert _tree(d, page=16) == ekv.ENULL                  # pages without a table
    for k in ("q", "W_uk", "W_uv", "ke", "c", "out", "ws"):
        assert _tree(d, **{k: FAKE + 8}) == ekv.EALIGN, k
    assert _tree(d, wsb=64) == ekv.EWORKSPACE
    assert ekv.elitekv_tree_attn_workspace_bytes(d, 2, 129, 128) == 0 < ekv.elitekv_tree_attn_workspace_bytes(d, 2, 128, 128)


def test_tree_plan_and_commit_refusals():
    plan = lambda B=2, T=3, **kw: lib.elitekv_tree_plan(*[kw.get(k, FAKE) for k in ("parent", "prefix", "nodes")], B, T,
                                                        *[kw.get(k, FAKE) for k in ("pos", "mask")], None)
    assert plan(B=0) == ekv.OK
    assert plan(B=-1) == ekv.EINVAL and plan(T=0) == ekv.EINVAL
    assert plan(T=129) == ekv.EUNSUPPORTED and plan(B=65536) == ekv.EUNSUPPORTED
    for k in ("parent", "prefix", "nodes", "pos", "mask"):
        assert plan(**{k: None}) == ekv.ENULL, k

    def commit(d, **kw):
        a = dict(path=FAKE, n=FAKE, prefix=FAKE, B=2, T=3, stride=64, table=None, cols=0, page=0, ke=FAKE, c=FAKE, rows=128)
        a.update(kw)
        return lib.elitekv_tree_commit(C.byref(d) if d else None, *a.values(), None)
    d = _dims()
    assert commit(None) == ekv.ENULL and commit(_dims(d_c=0)) == ekv.EINVAL
    assert commit(d, B=0) == ekv.OK
    for bad in (dict(B=-1), dict(T=0), dict(stride=-1), dict(rows=-1), dict(table=FAKE, cols=3, page=40)):
        assert commit(d, **bad) == ekv.EINVAL, bad
    assert commit(d, T=129) == ekv.EUNSUPPORTED and commit(d, B=65536) == ekv.EUNSUPPORTED
    for k in ("path", "n", "prefix", "ke", "c"):
        assert commit(d, **{k: None}) == ekv.ENULL, k
    assert commit(d, page=16) == ekv.ENULL
    for k in ("ke", "c"):
        assert commit(d, **{k: FAKE + 4}) == ekv.EALIGN, k
    assert commit(_dims(r=0), ke=None, B=0) == ekv.OK


@pytest.mark.parametrize("B,T", [(1, 2), (1, 64), (3, 26), (8, 5), (8, 64), (64, 3), (200, 128)])
@pytest.mark.parametrize("shape,d_ck", [(dict(r=4, d_c=768), 0), (dict(r=8, d_c=768), 0), (dict(r=8, d_c=512, n_heads=40), 0), (dict(r=4, d_c=256), 0),
                                        (dict(r=8, d_c=1536), 768), (dict(r=4, d_c=512), 256), (dict(r=8, d_c=1536), 0),
                                        (dict(r=8, d_c=1536, dtype="fp32"), 0)])
def test_a_workspace_of_a_longer_bound_serves_every_shorter_one(shape, d_ck, B, T):
    """Also across the length from which two queries share a work-group, which are split by another count."""
    d = _dims(**dict(dict(n_heads=32, head_dim=128, dtype="bf16"), **shape))
    bounds = list(range(0, 200, 7)) + list(range(200, 9000, 37)) + [20000, 131072]
    sizes = [ekv.elitekv_tree_attn_workspace_bytes(d, B, T, s, d_ck=d_ck) for s in bounds]
    assert sizes == sorted(sizes) and sizes[0] > 0
    if T < 48:
        paged = [ekv.elitekv_paged_attn_workspace_bytes(d, B, T, s, d_ck=d_ck) for s in bounds]
        assert paged == sizes
