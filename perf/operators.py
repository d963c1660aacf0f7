"""Timed cases of what a server keeps its cache in and verifies drafted tokens with: pages and trees.

  plan       pages handed out and taken back by request lengths, and where every new token goes (elitekv_page_plan)
  paged      attention of one query, a few or a prompt's chunk per sequence over a cache in pages (elitekv_paged_attn)
  tree_plan  which drafted tokens of a tree see which, and their positions (elitekv_tree_plan)
  tree       attention of a tree of drafted tokens over the cache and the tree's own rows (elitekv_tree_attn)
  commit     the rows of the accepted path moved to follow the sequence (elitekv_tree_commit)

Shapes are the 7B and 13B ones of the repository's workloads, bf16 as served and fp32 as results are checked in.
"""
import random

import numpy as np
import torch

own = False
DEV = "cuda:0"
BASE = 10000.0

# name: (hidden size, heads, head size, elite chunks, latent columns, of which for keys; 0 = the latent is shared)
SHAPES = {
    "7b_25": (4096, 32, 128, 8, 1536, 0),
    "7b_12": (4096, 32, 128, 4, 768, 0),
    "13b_25": (5120, 40, 128, 8, 1920, 0),
    "7b_25_slrd_768": (4096, 32, 128, 8, 1536, 768),
}


def listed():
    return [
        # every step of a server: 64 chats of one new token each, a page now and then
        dict(name="plan_b64_t1", op="plan", B=64, T=1, S=4096, page=64),
        # a large batch of prompts let in at once, in small pages
        dict(name="plan_b256_t2048", op="plan", B=256, T=2048, S=8192, page=16),
        # a chat that has just begun: launches and latency are all there is
        dict(name="paged_7b25_b1_s300", op="paged", shape="7b_25", dtype="bf16", B=1, T=1, S=300, page=16, ragged=False),
        # the larger model, a long-context batch: the most cache bytes
        dict(name="paged_13b25_b16_s8192", op="paged", shape="13b_25", dtype="bf16", B=16, T=1, S=8192, page=64, ragged=False),
        # chunks of two prompts over what is already cached
        dict(name="paged_7b25_b2_t500_s4000", op="paged", shape="7b_25", dtype="bf16", B=2, T=500, S=4000, page=128, ragged=False),
        # one user's small tree
        dict(name="tree_plan_b1_t8", op="tree_plan", B=1, T=8),
        # the widest trees of a large batch
        dict(name="tree_plan_b256_t128", op="tree_plan", B=256, T=128),
        # two users' trees checked in fp32, the cache in one piece per sequence
        dict(name="tree_fp32_b2_t12_s1000", op="tree", shape="7b_25", dtype="fp32", B=2, T=12, S=1000, page=0, ragged=True),
        # wide trees of a small batch over the smallest cache
        dict(name="tree_7b12_b8_t64_s2048", op="tree", shape="7b_12", dtype="bf16", B=8, T=64, S=2048, page=64, ragged=True),
        # separated latents, odd counts and lengths
        dict(name="tree_slrd_b3_t26_s5001", op="tree", shape="7b_25_slrd_768", dtype="bf16", B=3, T=26, S=5001, page=32, ragged=True),
        # one user's accepted tokens
        dict(name="commit_7b25_b1_t8", op="commit", shape="7b_25", dtype="bf16", B=1, T=8, S=1000, page=0),
        # a full batch's
        dict(name="commit_13b25_b128_t26", op="commit", shape="13b_25", dtype="bf16", B=128, T=26, S=700, page=16),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(lo * (hi / lo) ** rng.random()))))


def draw(rng):
    """Another case of the same kinds, none larger than the largest listed one."""
    op = rng.choice(("plan", "paged", "paged", "paged", "tree_plan", "tree", "tree", "tree", "commit"))
    page = 16 << rng.randint(0, 4)
    if op == "plan":
        B = _log(rng, 1, 1024)
        T = 1 if rng.random() < 0.4 else _log(rng, 2, min(2048, 256 * 2048 // B))
        return dict(op=op, B=B, T=T, S=T + _log(rng, 16, 6000), page=page)
    if op == "tree_plan":
        return dict(op=op, B=_log(rng, 1, 256), T=_log(rng, 2, 128))
    if op == "commit":
        B, T = _log(rng, 1, 64), _log(rng, 2, 48)
        return dict(op=op, shape=rng.choice(tuple(SHAPES)), dtype="bf16", B=B, T=T, S=T + _log(rng, 1, 900),
                    page=rng.choice((0, page)))
    fp32 = rng.random() < 0.2
    shape = rng.choice(("7b_25", "7b_12") if fp32 else tuple(SHAPES))
    dtype, rows = ("fp32", 2000) if fp32 else ("bf16", 16 * 8192)
    if op == "paged":
        kind = rng.random()
        B, T = (_log(rng, 1, 4 if fp32 else 64), 1) if kind < 0.5 else (rng.randint(1, 4), rng.randint(2, 8)) if kind < 0.75 else (
            rng.randint(1, 2), _log(rng, 16, 48 if fp32 else 500))
        most = min(32768, rows // B) if T == 1 else min(rows // B, 4000 if T > 8 else 8000)
        return dict(op=op, shape=shape, dtype=dtype, B=B, T=T, S=T + _log(rng, 100, max(101, most - T)), page=page,
                    ragged=rng.random() < 0.6)
    B, T = rng.randint(1, 2 if fp32 else 8), _log(rng, 3, 24 if fp32 else 64)
    most = min(rows // B, 8 * 64 * 2048 // (B * T), 8000)
    return dict(op=op, shape=shape, dtype=dtype, B=B, T=T, S=T + _log(rng, 100, max(101, most - T)),
                page=rng.choice((0, page)), ragged=rng.random() < 0.6)


def _lengths(case):
    """Cached tokens of every sequence, the new ones included: all S, or spread between S/4 and S."""
    B, S, T = case["B"], case["S"], case["T"]
    if not case.get("ragged"):
        return [S] * B
    return [max(T, S - (S * 3 // 4) * ((37 * b) % 64) // 64) for b in range(B)]


def _counts(case):
    """Drafted tokens of every sequence: all T, or a few short of it."""
    B, T = case["B"], case["T"]
    return [max(1, T - b % 3) if case.get("ragged") else T for b in range(B)]


def _parents(host, B, T):
    """Trees as a draft model grows them: a node hangs on one of the last few, now and then on an early one."""
    rows = []
    for _ in range(B):
        rows.append([-1] + [host.randint(max(0, t - 6), t - 1) if host.random() < 0.8 else host.randint(0, t - 1) for t in range(1, T)])
    return np.array(rows, dtype=np.int32)


def _ancestors(parent):
    """[B, T, T] truth values: node t sees node j."""
    B, T = parent.shape
    sees = np.zeros((B, T, T), dtype=bool)
    for t in range(T):
        sees[:, t, t] = True
        has = parent[:, t] >= 0
        sees[has, t] |= sees[has, parent[has, t]]
    return sees


def _words(sees):
    """Truth values over the last axis as 32-bit words, the first in the lowest bit."""
    T = sees.shape[-1]
    bits = np.zeros(sees.shape[:-1] + ((T + 31) // 32 * 32,), dtype=np.uint8)
    bits[..., :T] = sees
    return np.packbits(bits, axis=-1, bitorder="little").view(np.int32)


def _pages(host, lens, page, cols):
    """A table [B, cols] of pages in no order, and how many pages there are."""
    need = [-(-n // page) for n in lens]
    n_pages = sum(need) + 3
    order = list(range(n_pages))
    host.shuffle(order)
    table, at = np.zeros((len(lens), cols), dtype=np.int32), 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    return table, n_pages


def _dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV)


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    host = random.Random(seed)
    op, B, T = case["op"], case["B"], case["T"]
    st = dict(op=op, B=B, T=T, page=case.get("page", 0))

    if op == "plan":
        S, page = case["S"], case["page"]
        cached, new = [], []
        for b in range(B):
            n = host.randint(1, T) if T > 1 else int(host.random() < 0.95)
            c = 0 if T > 64 and host.random() < 0.7 else host.randint(0, S - T)
            if host.random() < 0.05:                       # a request that has ended: its pages go back
                c = n = 0
            cached.append(c)
            new.append(n)
        cols = -(-S // page)
        held = [min(cols, -(-c // page) + (host.random() < 0.1)) if c or n else host.randint(0, cols // 2) for c, n in zip(cached, new)]
        n_pages = B * cols + 5
        order = list(range(n_pages))
        host.shuffle(order)
        table, at = np.full((B, cols), -1, dtype=np.int32), 0
        for b, h in enumerate(held):
            table[b, :h] = order[at:at + h]
            at += h
        taken = host.randint(0, 3 * n_pages)               # the ring has been round before
        free = np.zeros(n_pages, dtype=np.int32)
        for i, p in enumerate(order[at:]):
            free[(taken + i) % n_pages] = p
        i32 = lambda v: _dev(np.array(v, dtype=np.int32))
        st.update(n_pages=n_pages, cols=cols, cached=i32(cached), new=i32(new), held=i32(held), held_out=i32(held), table=_dev(table),
                  free=_dev(free), span=_dev(np.array([taken, taken + n_pages - at], dtype=np.int64)),
                  span_out=torch.zeros(2, dtype=torch.int64, device=DEV), pos=torch.zeros(B, T, dtype=torch.int32, device=DEV),
                  slot=torch.zeros(B, T, dtype=torch.int64, device=DEV), kv_len=torch.zeros(B, T, dtype=torch.int32, device=DEV))
        return st

    if op == "tree_plan":
        st.update(parent=_dev(_parents(host, B, T)), prefix=_dev(np.array([host.randint(0, 5000) for _ in range(B)], dtype=np.int32)),
                  nodes=_dev(np.array([host.randint(max(1, T - 3), T) for _ in range(B)], dtype=np.int32)),
                  pos=torch.zeros(B, T, dtype=torch.int32, device=DEV),
                  mask=torch.zeros(B, T, (T + 31) // 32, dtype=torch.int32, device=DEV))
        return st

    d, n_h, d_h, r, d_c, d_ck = SHAPES[case["shape"]]
    dt = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32

    def normal(*size, std=1.0):
        return torch.randn(*size, generator=g, device=DEV, dtype=torch.float32).mul_(std).to(dt)

    lens = _lengths(case)
    host.shuffle(lens)
    S, page = max(lens), case["page"]
    if page:
        cols = -(-S // page) + 1
        table, n_pages = _pages(host, lens, page, cols)
        rows = n_pages * page
        st.update(table=_dev(table), cols=cols)
    else:
        rows = B * (S + 16)
    st.update(shape=case["shape"], dtype=case["dtype"], S=S, stride=S + 16, rows=rows, ke=normal(rows, n_h, 2 * r), c=normal(rows, d_c))

    if op == "commit":
        n = [host.randint(1, T) for _ in range(B)] if B > 1 else [max(1, T // 2)]
        path = np.zeros((B, T), dtype=np.int32)
        for b in range(B):
            path[b, :n[b]] = sorted(host.sample(range(T), n[b]))
        st.update(path=_dev(path), path_len=_dev(np.array(n, dtype=np.int32)), prefix=_dev(np.array([m - T for m in lens], dtype=np.int32)))
        return st

    dk, dv = (d_ck, d_c - d_ck) if d_ck else (d_c, d_c)
    idx = np.stack([np.array(host.sample(range(d_h // 2), r), dtype=np.int32) for _ in range(n_h)])
    rest = np.stack([[i for i in range(d_h) if i // 2 not in set(row.tolist())] for row in idx]).astype(np.int64)
    st.update(idx=_dev(idx), rest=_dev(rest), W_uk=normal(dk, n_h, d_h - 2 * r, std=dk ** -0.5), W_uv=normal(dv, n_h, d_h, std=dv ** -0.5),
              q=normal(B, T, n_h, d_h), out=torch.zeros(B, T, n_h, d_h, dtype=dt, device=DEV))
    if op == "paged":
        pos = np.array([[n - T + t for t in range(T)] for n in lens], dtype=np.int32)
        st.update(pos=_dev(pos), kv_len=_dev(pos + 1))
        return st
    nodes = _counts(case)
    parent = _parents(host, B, T)
    sees = _ancestors(parent)
    prefix = np.array([n - T for n in lens], dtype=np.int32)
    st.update(prefix=_dev(prefix), nodes=_dev(np.array(nodes, dtype=np.int32)), mask=_dev(_words(sees)),
              pos=_dev((prefix[:, None] + sees.sum(axis=2) - 1).astype(np.int32)))
    return st


def run(st):
    if own:
        return _own(st)
    return {"plan": _plain_plan, "paged": _plain_paged, "tree_plan": _plain_tree_plan, "tree": _plain_tree, "commit": _plain_commit}[st["op"]](st)


def _own(st):
    import paper_2503_01586_amd as ekv
    op, B, T, page = st["op"], st["B"], st["T"], st["page"]

    def workspace(nbytes):                                 # kept with the state, as a program keeps it from call to call
        if "ws" not in st:
            st["ws"] = torch.empty(max(int(nbytes()), 16), dtype=torch.uint8, device=DEV)
        return st["ws"]

    if op == "plan":
        ws = workspace(lambda: ekv.elitekv_page_plan_workspace_bytes(B, T))
        ekv.elitekv_page_plan(st["cached"], st["new"], page, st["n_pages"], st["table"], st["held"], st["held_out"], st["free"], st["span"],
                              st["span_out"], st["pos"], st["slot"], st["kv_len"], ws)
        return {k: st[k] for k in ("table", "held_out", "free", "span_out", "pos", "slot", "kv_len")}
    if op == "tree_plan":
        ekv.elitekv_tree_plan(st["parent"], st["prefix"], st["nodes"], st["pos"], st["mask"])
        return dict(pos=st["pos"], mask=st["mask"])
    if "dims" not in st:
        d, n_h, d_h, r, d_c, d_ck = SHAPES[st["shape"]]
        st["dims"], st["d_ck"] = ekv.make_dims(d, n_h, d_h, r, d_c, st["dtype"], BASE), d_ck
    dims, d_ck, table = st["dims"], st["d_ck"], st.get("table")
    if op == "commit":
        ekv.elitekv_tree_commit(dims, st["path"], st["path_len"], st["prefix"], st["stride"], st["ke"], st["c"], block_table=table, page_rows=page)
        return dict(ke=st["ke"], c=st["c"])
    up = (st["W_uk"], st["W_uv"], st["idx"], st["ke"], st["c"], st["out"])
    if op == "paged":
        ws = workspace(lambda: ekv.elitekv_paged_attn_workspace_bytes(dims, B, T, st["S"], d_ck=d_ck))
        ekv.elitekv_paged_attn(dims, st["q"], st["pos"], st["kv_len"], st["S"], table, page, *up, ws, d_ck=d_ck)
    else:
        ws = workspace(lambda: ekv.elitekv_tree_attn_workspace_bytes(dims, B, T, st["S"], d_ck=d_ck))
        ekv.elitekv_tree_attn(dims, st["q"], st["pos"], st["prefix"], st["nodes"], st["mask"], st["S"], st["stride"], *up, ws,
                              block_table=table, page_rows=page, d_ck=d_ck)
    return dict(out=st["out"])


# ---- plain forms ----

def _plain_plan(st):
    T, page, n_pages, cols = st["T"], st["page"], st["n_pages"], st["cols"]
    cached, new, held = st["cached"].long().clamp(min=0), st["new"].long().clamp(0, T), st["held"].long().clamp(0, cols)
    want = ((cached + new + page - 1) // page).clamp(max=cols)
    grow, back = (want - held).clamp(min=0), (held - want).clamp(min=0)
    taken, given = st["span"][0], st["span"][1]
    before = grow.cumsum(0) - grow
    granted = torch.minimum(grow, (given - taken - before).clamp(min=0))
    held_out = torch.where(back > 0, want, held + granted)
    col = torch.arange(cols, device=DEV)[None, :]
    h, w = held[:, None], want[:, None]
    fresh = st["free"][(taken + before[:, None] + col - h) % n_pages]
    table = torch.where((col >= h) & (col < h + granted[:, None]), fresh, st["table"])
    # pages that go back; what does not is written to a place past the ring's end
    to = torch.where((col >= w) & (col < h), (given + (back.cumsum(0) - back)[:, None] + col - w) % n_pages, n_pages)
    free = torch.cat((st["free"], st["free"][:1])).scatter(0, to.reshape(-1), st["table"].reshape(-1))[:n_pages]
    t = torch.arange(T, device=DEV)[None, :]
    pos = cached[:, None] + t
    at = pos // page
    real = t < new[:, None]
    there = real & (at < held_out[:, None])
    block = table.long().gather(1, at.clamp(max=cols - 1))
    slot = torch.where(there, block * page + pos % page, -1)
    return dict(table=table, held_out=held_out.int(), free=free, span_out=torch.stack((taken + granted.sum(), given + back.sum())),
                pos=torch.where(real, pos, 0).int(), slot=slot, kv_len=torch.where(there, pos + 1, 0).int())


def _plain_tree_plan(st):
    parent, T = st["parent"].long(), st["T"]
    node = torch.arange(T, device=DEV)
    # I + A + A A + ... with A[t, parent of t] = 1 is the inverse of I - A: whole numbers, 1 where t sees j
    A = (parent[:, :, None] == node).float()
    eye = torch.eye(T, device=DEV).expand_as(A)
    sees = torch.linalg.solve_triangular(eye - A, eye, upper=False, unitriangular=True) > 0.5
    real = node[None, :] < st["nodes"][:, None]
    sees = sees & real[:, :, None]
    pos = torch.where(real, st["prefix"][:, None] + sees.sum(dim=2) - 1, 0).int()
    W = (T + 31) // 32
    bits = torch.nn.functional.pad(sees, (0, 32 * W - T)).reshape(*parent.shape, W, 32).long()
    words = (bits << torch.arange(32, device=DEV)).sum(dim=3)
    return dict(pos=pos, mask=torch.where(words >= 1 << 31, words - (1 << 32), words).int())


def _rows_of(st, j):
    """Plane rows of the cached tokens j [B, ...] of every sequence."""
    flat = j.reshape(j.shape[0], -1)
    if st["page"]:
        row = st["table"].long().gather(1, flat // st["page"]) * st["page"] + flat % st["page"]
    else:
        row = torch.arange(st["B"], device=DEV)[:, None] * st["stride"] + flat
    return row.reshape(j.shape)


def _plain_commit(st):
    k = torch.arange(st["T"], device=DEV)[None, :].expand(st["B"], -1)
    prefix = st["prefix"].long()[:, None]
    source = torch.where(k < st["path_len"][:, None], st["path"].long(), k)
    to, source = _rows_of(st, prefix + k).reshape(-1), _rows_of(st, prefix + source).reshape(-1)
    st["ke"][to] = st["ke"][source]
    st["c"][to] = st["c"][source]
    return dict(ke=st["ke"], c=st["c"])


def _plain_paged(st):
    seen = torch.arange(st["S"], device=DEV)[None, None, :] < st["kv_len"][:, :, None]
    return dict(out=_plain_attention(st, seen))


def _plain_tree(st):
    j = torch.arange(st["S"], device=DEV)[None, None, :]
    prefix = st["prefix"].long()[:, None, None]
    bits = (st["mask"][..., None] >> torch.arange(32, device=DEV)) & 1          # [B, T, words, 32]
    bits = bits.reshape(st["B"], st["T"], -1).bool()
    node = (j - prefix).expand(-1, st["T"], -1)
    drafted = (node >= 0) & (node < st["nodes"][:, None, None]) & bits.gather(2, node.clamp(0, bits.shape[2] - 1))
    real = torch.arange(st["T"], device=DEV)[None, :, None] < st["nodes"][:, None, None]
    return dict(out=_plain_attention(st, ((j < prefix) | drafted) & real))


def _plain_attention(st, seen):
    """B^k absorbed into the query, one softmax over both score terms, B^v applied to the averaged latent; 32 bits."""
    _, n_h, d_h, r, d_c, d_ck = SHAPES[st["shape"]]
    B, T, S, dk = st["B"], st["T"], st["S"], d_ck or d_c
    rows = _rows_of(st, torch.arange(S, device=DEV)[None, :].expand(B, -1))
    ke, c = st["ke"][rows].float(), st["c"][rows].float()                       # [B, S, n_h, 2r], [B, S, d_c]
    q = st["q"].float()
    idx = st["idx"].long()
    angle = st["pos"].double()[:, :, None, None] * (BASE ** (-2.0 * idx.double() / d_h))
    cos, sin = angle.cos().float(), angle.sin().float()
    u = q.gather(3, (2 * idx).expand(B, T, -1, -1))
    v = q.gather(3, (2 * idx + 1).expand(B, T, -1, -1))
    q_e = torch.stack((u * cos - v * sin, u * sin + v * cos), dim=4).reshape(B, T, n_h, 2 * r)
    q_n = q.gather(3, st["rest"].expand(B, T, -1, -1))
    W_uk, W_uv = st["W_uk"].float(), st["W_uv"].float()
    absorbed = q_n.reshape(B * T, n_h, -1).transpose(0, 1).contiguous() @ W_uk.permute(1, 2, 0).contiguous()     # [n_h, B T, dk]
    absorbed = absorbed.reshape(n_h, B, T, dk).permute(1, 0, 2, 3).reshape(B, n_h * T, dk)
    s = (absorbed @ c[:, :, :dk].transpose(1, 2).contiguous()).reshape(B, n_h, T, S)
    s = s + q_e.transpose(1, 2).contiguous() @ ke.permute(0, 2, 3, 1).contiguous()
    s = (s * d_h ** -0.5).masked_fill(~seen[:, None], float("-inf"))
    top = s.amax(dim=3, keepdim=True)
    p = (s - torch.where(top == float("-inf"), 0.0, top)).exp()
    total = p.sum(dim=3, keepdim=True)
    p = p / torch.where(total > 0, total, 1.0)
    latent = p.reshape(B, n_h * T, S) @ c[:, :, d_ck:].contiguous()
    latent = latent.reshape(B, n_h, T, -1).permute(1, 0, 2, 3).reshape(n_h, B * T, -1)
    out = latent @ W_uv.transpose(0, 1).contiguous()                            # [n_h, B T, d_h]
    return out.transpose(0, 1).reshape(B, T, n_h, d_h).to(st["q"].dtype)


# ---- floors ----

def _pairs(case):
    """(query, visible row) pairs of the whole call."""
    T, lens = case["T"], _lengths(case)
    if case["op"] == "paged":
        return sum(T * n - T * (T - 1) // 2 for n in lens)
    return sum(k * (n - T) + k * (k + 1) // 2 for n, k in zip(lens, _counts(case)))


def work(case):
    """Bytes: every input and every visible cached row read once, results written once.  Operations: the attention in the
    cheaper of its two orders (B^k, B^v absorbed, or keys and values rebuilt)."""
    op, B, T = case["op"], case["B"], case["T"]
    if op == "plan":
        return dict(bytes=16 * B + 16 * B * T + 8 * B * -(-T // case["page"]), flops=0)
    if op == "tree_plan":
        return dict(bytes=8 * B + B * T * (8 + 4 * ((T + 31) // 32)), flops=0)
    _, n_h, d_h, r, d_c, d_ck = SHAPES[case["shape"]]
    e = 2 if case["dtype"] == "bf16" else 4
    row = 2 * r * n_h + d_c
    if op == "commit":
        return dict(bytes=e * row * B * T + 4 * B * T, flops=0)                 # half of the nodes on the average, read and written
    dk, dv = (d_ck, d_c - d_ck) if d_ck else (d_c, d_c)
    lens, pairs = _lengths(case), _pairs(case)
    up = 2.0 * n_h * (dk * (d_h - 2 * r) + dv * d_h)
    absorbed = pairs * n_h * 2.0 * (2 * r + dk + dv) + B * T * up
    rebuilt = pairs * n_h * 4.0 * d_h + sum(lens) * up
    weights = n_h * (dk * (d_h - 2 * r) + dv * d_h)
    return dict(bytes=e * (weights + 2 * B * T * n_h * d_h + sum(lens) * row), flops=min(absorbed, rebuilt))


# ---- in 64 bits ----

def exact(case, seed):
    """Attention from its definition: full keys [stored elite dims | c B^k] and values c B^v of every head, one softmax over the
    rows a query sees.  Plans are whole numbers: they are compared as they are."""
    if case["op"] in ("plan", "tree_plan"):
        return None
    st = prepare(case, seed)
    if case["op"] == "commit":
        return _exact_commit(st)
    _, n_h, d_h, r, d_c, d_ck = SHAPES[case["shape"]]
    B, T, S = st["B"], st["T"], st["S"]
    host = {k: st[k].cpu().numpy() for k in ("pos", "idx", "kv_len", "prefix", "nodes", "mask", "table") if k in st}
    theta = BASE ** (-2.0 * np.arange(d_h // 2) / d_h)
    out = torch.zeros(B, T, n_h, d_h, dtype=torch.float64, device=DEV)
    for b in range(B):
        seen = np.zeros((T, S), dtype=bool)
        for t in range(T):
            if case["op"] == "paged":
                seen[t, :host["kv_len"][b, t]] = True
            elif t < host["nodes"][b]:
                P = host["prefix"][b]
                seen[t, :P] = True
                for j in range(host["nodes"][b]):
                    seen[t, P + j] = (int(host["mask"][b, t, j // 32]) >> (j % 32)) & 1
        n = int(seen.any(axis=0).nonzero()[0][-1]) + 1
        at = [int(host["table"][b, j // st["page"]]) * st["page"] + j % st["page"] if st["page"] else b * st["stride"] + j for j in range(n)]
        at = torch.tensor(at, device=DEV)
        ke, c = st["ke"][at].double(), st["c"][at].double()
        ck, cv = (c[:, :d_ck], c[:, d_ck:]) if d_ck else (c, c)
        hide = _dev(~seen[:, :n])
        for h in range(n_h):
            elite = host["idx"][h]
            angle = _dev(host["pos"][b].astype(np.float64)[:, None] * theta[elite][None, :])
            qh = st["q"][b, :, h].double()
            cols = torch.from_numpy(elite.astype(np.int64)).to(DEV)
            z = torch.complex(qh[:, 2 * cols], qh[:, 2 * cols + 1]) * torch.polar(torch.ones_like(angle), angle)
            query = torch.cat((torch.view_as_real(z).reshape(T, 2 * r), qh[:, st["rest"][h]]), dim=1)
            keys = torch.cat((ke[:, h], ck @ st["W_uk"][:, h].double()), dim=1)
            s = (query @ keys.T / d_h ** 0.5).masked_fill_(hide, float("-inf"))
            p = torch.nan_to_num(s.softmax(dim=1)) if case["op"] == "tree" else s.softmax(dim=1)
            out[b, :, h] = p @ (cv @ st["W_uv"][:, h].double())
    return dict(out=out)


def _exact_commit(st):
    host = {k: st[k].cpu().numpy() for k in ("path", "path_len", "prefix", "table") if k in st}
    row = lambda b, j: int(host["table"][b, j // st["page"]]) * st["page"] + j % st["page"] if st["page"] else b * st["stride"] + j
    to, source = [], []
    for b in range(st["B"]):
        P = int(host["prefix"][b])
        to += [row(b, P + k) for k in range(host["path_len"][b])]
        source += [row(b, P + int(j)) for j in host["path"][b, :host["path_len"][b]]]
    planes = {k: st[k].double() for k in ("ke", "c")}
    for v in planes.values():
        v[to] = v[source]
    return planes
