"""The operators that grow a paged tree KV cache: their cases, plain forms and 64-bit values.

A search step adds tokens to blocks of the tree: slots are reserved for them, queries and
keys are normed and rotated and the rows written into the pool, and the new tokens attend
over their chains.  A search also forks blocks and takes tokens back.

Kinds
  attend  arbor_prefill_plan and arbor_tree_prefill_attn, a call for each layer: causal
          attention of packed new tokens over their ancestors' and their own resident tokens
  append  arbor_append: norm of each query and key head, rotation, rows into the pool
  beam    arbor_truncate and arbor_fork: blocks that lost are emptied and become copies
          of blocks that won
  draft   arbor_truncate and arbor_extend: drafted tokens are taken back, and slots
          reserved for the next ones
  grow    a whole step: truncate, extend, plan, and append and attention for each layer

Shapes are those of the synthetic configurations (paper_2605_22106_amd/synth.py: 8B, 70B,
dpts and tiny) or lie around them; `draw` gives more of the same ranges.  Everything is
made from the seed, on the GPU.
"""
from __future__ import annotations

import math
import random

import torch

own = False
P = 16          # slots of a page


def listed():
    b8 = dict(heads=8, group=4, dim=128, dtype="bf16")
    b70 = dict(heads=8, group=8, dim=128, dtype="bf16")
    none = dict(branching=1, depth=0, root=0, node=0, kept=1.0)
    dpts = dict(branching=4, depth=3, root=1024, node=128)
    return [
        # the tiny fp32 tree gets one short block: what a call costs in launches
        dict(name="attend_tiny", kind="attend", heads=4, group=1, dim=64, dtype="f32", branching=2,
             depth=1, root=64, node=32, kept=1.0, seqs=2, new=24, had=0, ragged=False, layers=1,
             shape=0),
        # the prompt of the 8B tree, the root block, all at once
        dict(name="attend_prompt_8b", kind="attend", **b8, **none, seqs=1, new=4096, had=0,
             ragged=False, layers=2, shape=1),
        # a long prompt of the 70B shape: the largest call
        dict(name="attend_prompt_70b", kind="attend", **b70, **none, seqs=1, new=8192, had=0,
             ragged=False, layers=1, shape=2),
        # a frontier of 16 new thoughts, ragged, over ancestors that an event has thinned out
        dict(name="attend_frontier", kind="attend", **b8, **dpts, kept=0.4, seqs=16, new=128,
             had=0, ragged=True, layers=4, shape=3),
        # drafts of up to eight tokens of 64 leaves, all below one long prompt
        dict(name="attend_prefix", kind="attend", **b8, branching=1, depth=0, root=32000, node=0,
             kept=1.0, seqs=64, new=8, had=100, ragged=True, layers=2, shape=4),
        # one new token of each of 16 leaves: the single-token step of a layer
        dict(name="append_step", kind="append", **b8, tokens=16, pad=0, norm=True, rotary=128,
             interleaved=False, record=False, far=40000, shape=5),
        # the rows of a long prompt, 70B shape
        dict(name="append_prompt", kind="append", **b70, tokens=8192, pad=0, norm=True, rotary=128,
             interleaved=False, record=False, far=0, shape=6),
        # an odd, padded fp32 batch, a part of each head rotated in neighbouring pairs,
        # with the token record that restores evicted rows
        dict(name="append_ragged", kind="append", heads=4, group=3, dim=64, dtype="f32",
             tokens=1531, pad=37, norm=False, rotary=32, interleaved=True, record=True, far=300000,
             shape=7),
        # four losing thoughts of the 8B tree become copies of four that won, 32 layers
        dict(name="beam_8b", kind="beam", **b8, branching=8, depth=1, root=1024, node=256,
             kept=1.0, ragged=False, pairs=4, layers=32, shape=8),
        # 128 pairs of ragged, partly evicted thoughts of a wide frontier
        dict(name="beam_wide", kind="beam", **b8, branching=17, depth=2, root=512, node=128,
             kept=0.5, ragged=True, pairs=128, layers=4, shape=9),
        # drafts of 48 leaves of a 341-block tree taken back and reserved again
        dict(name="draft_wide", kind="draft", **b8, branching=4, depth=4, root=1024, node=128,
             kept=0.5, seqs=48, new=6, had=90, ragged=True, layers=1, shape=10),
        # a whole step of the same frontier's new thoughts through four layers
        dict(name="grow_step", kind="grow", **b8, **dpts, kept=1.0, seqs=16, new=64, had=20,
             ragged=True, layers=4, norm=True, rotary=128, interleaved=False, shape=11),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the ranges that the listed ones span."""
    while True:
        kind = rng.choice(["attend"] * 9 + ["append"] * 5 + ["beam"] * 2 + ["draft", "grow", "grow"])
        c = dict(kind=kind, heads=rng.choice([2, 4, 8]), group=rng.choice([1, 2, 3, 4, 4, 7, 8]),
                 dim=rng.choice([64, 128, 128]), dtype=rng.choice(["bf16", "bf16", "bf16", "f32"]),
                 shape=rng.randrange(1 << 16))
        if kind in ("append", "grow"):
            c.update(norm=rng.random() < 0.6, interleaved=rng.random() < 0.3,
                     rotary=rng.choice([c["dim"], c["dim"], c["dim"] // 2, 32, 0]))
        if kind == "append":
            c.update(tokens=_log(rng, 1, 8192), pad=rng.choice([0, 0, rng.randint(1, 40)]),
                     record=rng.random() < 0.3, far=rng.choice([0, _log(rng, 1000, 1000000)]))
            return c
        prompt = kind == "attend" and rng.random() < 0.35
        c.update(branching=rng.randint(2, 5), depth=rng.randint(0, 4), root=_log(rng, 16, 32000),
                 node=_log(rng, 16, 512), kept=rng.choice([1.0, round(rng.uniform(0.2, 0.9), 3)]),
                 ragged=rng.random() < 0.7, layers=rng.choice([1, 2, 4]))
        if kind == "beam":
            c.update(depth=rng.randint(1, 3), root=_log(rng, 16, 4096), layers=rng.choice([2, 8, 32]))
            leaves = c["branching"] ** c["depth"]
            c.update(pairs=_log(rng, 1, max(1, leaves // 2)))
            if leaves < 2 or c["pairs"] * 2 > leaves or _pool_bytes(c) > (2 << 30):
                continue
            return c
        if prompt:
            c.update(branching=1, depth=0, root=0, node=0, kept=1.0, seqs=1, had=0,
                     new=_log(rng, 1, 8192))
        else:
            c.update(seqs=_log(rng, 1, 64), new=_log(rng, 1, 2048),
                     had=rng.choice([0, _log(rng, 1, 300)]))
        if kind == "draft":
            c.update(new=_log(rng, 1, 64), layers=1)
        t = _tree(c)
        rows = sum(t["m"]) * c["heads"] * c["group"]
        seen = sum(t["c"])
        most = 3e9 if c["dtype"] == "bf16" else 1e9
        if rows * seen * c["layers"] > most or _pool_bytes(c) > (3 << 30) or seen > 120000:
            continue
        return c


# ---- the tree of a case (host side, from the case alone) ---------------------

def _tree(case):
    """parent; cap, n and c of every block (capacity, tokens, resident tokens, the step's new
    ones among them); nodes, m: the blocks that get tokens, and how many of their newest are new."""
    r = random.Random(case["shape"])
    parent, n, deepest = [], [], []
    if case["root"]:
        level = [0]
        parent, n = [-1], [case["root"]]
        for _ in range(case["depth"]):
            nxt = []
            for p in level:
                for _ in range(case["branching"]):
                    nxt.append(len(parent))
                    parent.append(p)
                    n.append(case["node"])
            level = nxt
        deepest = level
    if case["ragged"]:
        n = [max(1, round(x * r.uniform(0.3, 1.0))) for x in n]
    c = list(n)
    if case["kept"] < 1.0:
        c = [min(x, max(1, round(x * case["kept"] * r.uniform(0.4, 1.6)))) for x in n]
    cap, nodes, m = list(n), [], []
    if case["kind"] == "beam":
        return dict(parent=parent, cap=[x + 7 for x in n], n=n, c=c, nodes=[], m=[], deepest=deepest)
    for e in range(case["seqs"]):
        parent.append(deepest[e * len(deepest) // case["seqs"]] if deepest else -1)
        nodes.append(len(parent) - 1)
        m.append(r.randint(1, case["new"]) if case["ragged"] else case["new"])
        had = r.randint(0, case["had"]) if case["ragged"] else case["had"]
        n.append(had + m[-1])
        c.append(had + m[-1])
        cap.append(had + m[-1] + r.randint(0, 20))
    return dict(parent=parent, cap=cap, n=n, c=c, nodes=nodes, m=m, deepest=deepest)


def _chain(parent, i):
    out = []
    while i >= 0:
        out.append(i)
        i = parent[i]
    return out[::-1]


def _size(case):
    return 2 if case["dtype"] == "bf16" else 4


def _dt(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _pool_bytes(case):
    pages = sum((x + P - 1) // P for x in _tree(dict(case, seqs=case.get("seqs", 0)))["cap"])
    return 2 * case["layers"] * pages * P * case["heads"] * case["dim"] * _size(case)


def _gen(seed, purpose):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 7919 + purpose)
    return g


# ---- states on the GPU -------------------------------------------------------

def _pool(case, seed, t):
    """The paged pool with c[i] of block i's n[i] tokens resident, pages shuffled.  The last
    m tokens of a block in t["nodes"] are all resident."""
    dev, g, i32 = "cuda", _gen(seed, 1), torch.int32
    V, Lr, H, D = len(t["parent"]), case["layers"], case["heads"], case["dim"]
    cap, nt, ct = (torch.tensor(t[k], device=dev) for k in ("cap", "n", "c"))
    tok_off = torch.zeros(V + 1, dtype=torch.int64, device=dev)
    tok_off[1:] = cap.cumsum(0)
    page_off = torch.zeros(V + 1, dtype=torch.int64, device=dev)
    page_off[1:] = ((cap + P - 1) // P).cumsum(0)
    pages = int(page_off[-1])
    perm = torch.randperm(pages, generator=g, device=dev)
    node_of_page = torch.repeat_interleave(torch.arange(V, device=dev), page_off.diff())
    q = torch.arange(pages, device=dev) - page_off[node_of_page]
    used = q < ((ct + P - 1) // P)[node_of_page]
    page_table = torch.where(used, perm, -torch.ones_like(perm)).to(i32)
    free = perm[~used].to(i32)
    free_stack = torch.full((pages,), -1, dtype=i32, device=dev)
    free_stack[:free.numel()] = free
    # the resident positions of each block: c[i] of n[i] at random, ascending
    N = int(nt.sum())
    first = nt.cumsum(0) - nt
    node = torch.repeat_interleave(torch.arange(V, device=dev), nt)
    pos = torch.arange(N, device=dev) - first[node]
    key = torch.rand(N, generator=g, device=dev, dtype=torch.float64)
    rank = torch.empty(N, dtype=torch.int64, device=dev)
    rank[torch.argsort(node + key)] = pos
    tok = torch.nonzero(rank < ct[node]).flatten()
    cfirst = ct.cumsum(0) - ct
    slot = torch.arange(tok.numel(), device=dev) - cfirst[node[tok]]
    phys = page_table[page_off[node[tok]] + slot // P].to(torch.int64)
    slot_pos = torch.full((pages, P), -1, dtype=i32, device=dev)
    slot_pos[phys, slot % P] = pos[tok].to(i32)
    dt = _dt(case)
    k = torch.randn((Lr, pages, H, P, D), generator=g, device=dev, dtype=dt)
    v = torch.randn((Lr, pages, H, P, D), generator=g, device=dev, dtype=dt)
    # 2 % of the keys are heavy (x 4)
    scale = torch.where(torch.rand((pages, P), generator=g, device=dev) < 0.02, 4.0, 1.0).to(dt)
    k.mul_(scale[None, :, None, :, None])
    return dict(parent=torch.tensor(t["parent"], dtype=i32, device=dev), n_full=nt.to(i32),
                tok_off=tok_off, page_off=page_off, n_kept=ct.to(i32), page_table=page_table,
                k=k, v=v, slot_pos=slot_pos, free_stack=free_stack,
                free_top=torch.tensor([free.numel()], dtype=i32, device=dev),
                num_tokens=int(tok_off[-1]))


def _i32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _rope_inputs(case, seed, tokens, layers):
    """Projections of `tokens` tokens as the rows of one product, q, k and v side by side;
    norm weights; frequencies."""
    g, dt, D = _gen(seed, 2), _dt(case), case["dim"]
    H, Hq = case["heads"], case["heads"] * case["group"]
    st = dict(qkv=[torch.randn((tokens, (Hq + 2 * H) * D), generator=g, device="cuda", dtype=dt)
                   for _ in range(layers)])
    for x in st["qkv"]:
        x[:, :Hq * D].mul_(1.7)
        x[:, Hq * D:(Hq + H) * D].mul_(0.6)
    st["q_norm"] = st["k_norm"] = None
    if case["norm"]:
        st["q_norm"] = (1 + 0.3 * torch.randn(D, generator=g, device="cuda")).to(dt)
        st["k_norm"] = (1 + 0.3 * torch.randn(D, generator=g, device="cuda")).to(dt)
    rd = case["rotary"]
    st["inv_freq"] = None
    if rd:
        e = torch.arange(0, rd, 2, device="cuda", dtype=torch.float64) / rd
        st["inv_freq"] = (500000.0 ** -e).to(torch.float32)
    return st


def prepare(case, seed):
    dev, kind, dt = "cuda", case["kind"], _dt(case)
    H, D = case["heads"], case["dim"]
    Hq = H * case["group"]
    st = dict(case=case, status=torch.zeros(1, dtype=torch.int32, device=dev))
    if kind == "append":
        T = case["tokens"]
        rows = T + case["pad"]
        pages = (T + P - 1) // P + 4
        g = _gen(seed, 3)
        st.update(_rope_inputs(case, seed, rows, 1))
        slots = torch.full((rows,), -1, dtype=torch.int64, device=dev)
        slots[:T] = torch.randperm(pages, generator=g, device=dev).repeat_interleave(P)[:T] * P + \
            torch.arange(T, device=dev) % P
        pos = torch.arange(rows, device=dev) + (case["far"] * (torch.arange(rows, device=dev) % 5)) // 4
        st.update(slots=slots, positions=pos.to(torch.int32),
                  k=torch.randn((1, pages, H, P, D), generator=g, device=dev, dtype=dt),
                  v=torch.randn((1, pages, H, P, D), generator=g, device=dev, dtype=dt),
                  q_out=torch.zeros((rows, Hq, D), dtype=dt, device=dev), tokens=None)
        if case["record"]:
            st["tokens"] = torch.full((rows,), -1, dtype=torch.int64, device=dev)
            st["tokens"][:T] = torch.randperm(T + 9, generator=g, device=dev)[:T]
            st["record_k"] = torch.zeros((T + 9, 1, H, D), dtype=dt, device=dev)
            st["record_v"] = torch.zeros((T + 9, 1, H, D), dtype=dt, device=dev)
        return st
    t = _tree(case)
    st.update(_pool(case, seed, t))
    g = _gen(seed, 4)
    if kind == "beam":
        half = case["pairs"]
        pick = random.Random(case["shape"]).sample(t["deepest"], 2 * half)
        lose = sorted(pick[:half])
        st.update(src=_i32([pick[half + lose.index(x)] for x in lose]), dst=_i32(lose),
                  keep=_i32([0] * half),
                  A=torch.rand(st["num_tokens"], generator=g, device=dev),
                  rows=torch.randint(1000, (len(t["parent"]),), generator=g, device=dev))
        return _fits(st, t, lose, pick, half)
    T = sum(t["m"])
    cu = [0]
    for x in t["m"]:
        cu.append(cu[-1] + x)
    chains = [_chain(t["parent"], i) for i in t["nodes"]]
    deep = max(len(c) for c in chains)
    st.update(nodes=_i32(t["nodes"]), cu=_i32(cu), n_tokens=T,
              chains=torch.tensor([c + [-1] * (deep - len(c)) for c in chains], device=dev))
    if kind in ("draft", "grow"):
        st.update(keep=_i32([t["n"][i] - x for i, x in zip(t["nodes"], t["m"])]),
                  slots=torch.zeros(T, dtype=torch.int64, device=dev),
                  positions=torch.zeros(T, dtype=torch.int32, device=dev),
                  tokens=torch.zeros(T, dtype=torch.int64, device=dev))
    if kind == "grow":
        st.update(_rope_inputs(case, seed, T, case["layers"]))
        st["q_out"] = torch.zeros((T, Hq, D), dtype=dt, device=dev)
    if kind == "attend":
        st["q"] = [torch.randn((T, Hq, D), generator=g, device=dev, dtype=dt)
                   for _ in range(case["layers"])]
    if kind in ("attend", "grow"):
        st["out"] = [torch.zeros((T, Hq, D), dtype=dt, device=dev) for _ in range(case["layers"])]
        st["lse"] = [torch.zeros((T, Hq), device=dev) for _ in range(case["layers"])]
    return st


def _fits(st, t, lose, pick, half):
    """Room for the copies: a loser's capacity holds its winner (blocks differ by their ragged
    sizes), so the winners are the shorter ones of each pair's two sorted halves."""
    order = sorted(pick, key=lambda i: (t["cap"][i], i))
    win, lose = order[:half], sorted(order[half:])
    st["dst"], st["src"] = _i32(lose), _i32(win)
    return st


# ---- plain forms ---------------------------------------------------------------

def _pages_of(st):
    """Owner and index in its block of every logical page."""
    V, total = st["parent"].numel(), st["page_table"].numel()
    dev = st["parent"].device
    node = torch.repeat_interleave(torch.arange(V, device=dev), st["page_off"].diff(),
                                   output_size=total)
    return node, torch.arange(total, device=dev) - st["page_off"][node]


def _plain_truncate(st, nodes, keep):
    V = st["parent"].numel()
    dev = st["parent"].device
    limit = torch.full((V,), 2**31 - 1, dtype=torch.int64, device=dev)
    limit[nodes.long()] = keep.long()
    node, q = _pages_of(st)
    page = st["page_table"].long()
    pos = st["slot_pos"][page.clamp(min=0)].long()                        # [logical page][P]
    s = q[:, None] * P + torch.arange(P, device=dev)
    here = (s < st["n_kept"].long()[node][:, None]) & (page >= 0)[:, None]
    stay = here & (pos < limit[node][:, None])
    c = torch.zeros(V, dtype=torch.int64, device=dev).index_add_(0, node, stay.sum(1))
    gone = (here & ~stay).nonzero()
    st["slot_pos"][page[gone[:, 0]], gone[:, 1]] = -1
    freed = ((q >= ((c + P - 1) // P)[node]) & (page >= 0)).nonzero().flatten()
    top = st["free_top"].long()
    st["free_stack"][top + torch.arange(freed.numel() - 1, -1, -1, device=dev)] = page[freed].int()
    st["page_table"][freed] = -1
    st["free_top"] += freed.numel()
    st["n_kept"].copy_(c)
    st["n_full"].copy_(torch.minimum(st["n_full"].long(), limit))


def _pop(st, first, last):
    """New pages first..last - 1 of each block, from the top of the free stack."""
    node, q = _pages_of(st)
    new = ((q >= first[node]) & (q < last[node])).nonzero().flatten()
    top = st["free_top"].long()
    st["page_table"][new] = st["free_stack"][top - 1 - torch.arange(new.numel(), device=new.device)]
    st["free_top"] -= new.numel()


def _plain_extend(st):
    dev = st["parent"].device
    nodes, cu = st["nodes"].long(), st["cu"].long()
    m = cu.diff()
    c0, n0 = st["n_kept"].long(), st["n_full"].long()
    grow = torch.zeros_like(c0).index_add_(0, nodes, m)
    _pop(st, (c0 + P - 1) // P, (c0 + grow + P - 1) // P)
    st["n_kept"].copy_(c0 + grow)
    st["n_full"].copy_(n0 + grow)
    up = st["chains"]
    above = torch.where((up >= 0) & (up != nodes[:, None]), (n0 + grow)[up.clamp(min=0)], 0).sum(1)
    t = torch.arange(st["n_tokens"], device=dev)
    e = torch.searchsorted(cu, t, right=True) - 1
    i, j = nodes[e], t - cu[e]
    s = c0[i] + j
    slots = st["page_table"][st["page_off"][i] + s // P].long() * P + s % P
    st["slot_pos"].view(-1)[slots] = (n0[i] + j).int()
    st["slots"].copy_(slots)
    st["positions"].copy_(above[e] + n0[i] + j)
    st["tokens"].copy_(st["tok_off"][i] + n0[i] + j)


def _plain_fork(st):
    dev = st["parent"].device
    src, dst = st["src"].long(), st["dst"].long()
    c, n = st["n_kept"].long()[src], st["n_full"].long()[src]
    need = torch.zeros(st["parent"].numel(), dtype=torch.int64, device=dev)
    need[dst] = (c + P - 1) // P
    _pop(st, torch.zeros_like(need), need)
    st["n_kept"][dst] = c.int()
    st["n_full"][dst] = n.int()

    def spread(count):
        e = torch.repeat_interleave(torch.arange(count.numel(), device=dev), count)
        return e, torch.arange(e.numel(), device=dev) - (count.cumsum(0) - count)[e]

    e, s = spread(c)
    a = st["page_table"][st["page_off"][src[e]] + s // P].long()
    b = st["page_table"][st["page_off"][dst[e]] + s // P].long()
    st["slot_pos"][b, s % P] = st["slot_pos"][a, s % P]
    st["k"][:, b, :, s % P] = st["k"][:, a, :, s % P]
    st["v"][:, b, :, s % P] = st["v"][:, a, :, s % P]
    e, p = spread(n)
    st["A"][st["tok_off"][dst[e]] + p] = st["A"][st["tok_off"][src[e]] + p]
    st["rows"][dst] = st["rows"][src]


def _split(case, qkv):
    H, D = case["heads"], case["dim"]
    Hq = H * case["group"]
    return qkv[:, :Hq * D], qkv[:, Hq * D:(Hq + H) * D], qkv[:, (Hq + H) * D:]


def _turn(case, x, w, cos, sin):
    """Norm over each head and rotation, in 32 bits."""
    if w is not None:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6) * w.float()
    rd = case["rotary"]
    if rd == 0:
        return x
    if case["interleaved"]:
        a, b = x[..., 0:rd:2], x[..., 1:rd:2]
        y = torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2)
    else:
        a, b = x[..., :rd // 2], x[..., rd // 2:rd]
        y = torch.cat((a * cos - b * sin, b * cos + a * sin), -1)
    return torch.cat((y, x[..., rd:]), -1)


def _plain_append(st, layer, i):
    case, dt = st["case"], _dt(st["case"])
    live = (st["slots"] >= 0).nonzero().flatten()
    q, k, v = (x[live].view(live.numel(), -1, case["dim"]) for x in _split(case, st["qkv"][i]))
    cos = sin = None
    if st["inv_freq"] is not None:
        angle = st["positions"][live].double()[:, None] * st["inv_freq"].double()
        cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    st["q_out"][live] = _turn(case, q.float(), st["q_norm"], cos, sin).to(dt)
    k = _turn(case, k.float(), st["k_norm"], cos, sin).to(dt)
    page, row = st["slots"][live] // P, st["slots"][live] % P
    st["k"][layer][page, :, row] = k
    st["v"][layer][page, :, row] = v
    if st["tokens"] is not None and "record_k" in st:
        st["record_k"][st["tokens"][live], layer] = k
        st["record_v"][st["tokens"][live], layer] = v


def _plain_visible(st):
    """The resident slots of all chains (page, row), and which of them each new token sees."""
    dev = st["parent"].device
    nodes, cu = st["nodes"].long(), st["cu"].long()
    V = st["parent"].numel()
    below = torch.zeros((nodes.numel(), V + 1), dtype=torch.bool, device=dev)
    below.scatter_(1, torch.where(st["chains"] >= 0, st["chains"], V), True)
    used = below[:, :V].any(0)
    c = st["n_kept"].long()
    count = torch.where(used, c, 0)
    block = torch.repeat_interleave(torch.arange(V, device=dev), count)
    s = torch.arange(block.numel(), device=dev) - (count.cumsum(0) - count)[block]
    t = torch.arange(st["n_tokens"], device=dev)
    e = torch.searchsorted(cu, t, right=True) - 1
    mine = c[nodes[e]] - cu[e + 1] + t                       # the slot of each new token
    sees = below[e][:, block] & ((block[None, :] != nodes[e][:, None]) | (s[None, :] <= mine[:, None]))
    return st["page_table"][st["page_off"][block] + s // P].long(), s % P, sees


def _plain_attend(st, layer, q, out, lse, page, row, sees):
    case = st["case"]
    H, G, D, T = case["heads"], case["group"], case["dim"], st["n_tokens"]
    k = st["k"][layer][page, :, row].float().permute(1, 2, 0).contiguous()      # [H][D][keys]
    v = st["v"][layer][page, :, row].float().transpose(0, 1).contiguous()       # [H][keys][D]
    z = torch.bmm(q.float().view(T, H, G, D).transpose(0, 1).reshape(H, T * G, D), k)
    z.mul_(1.0 / math.sqrt(D))
    z.view(H, T, G, -1).masked_fill_(~sees[:, None, :], -math.inf)
    m = z.amax(-1, keepdim=True)
    z.sub_(m).exp_()
    l = z.sum(-1, keepdim=True)
    o = torch.bmm(z, v) / l
    out.copy_(o.view(H, T, G, D).transpose(0, 1).reshape(T, H * G, D))
    lse.copy_((m + l.log()).view(H, T, G).transpose(0, 1).reshape(T, H * G))


# ---- one pass --------------------------------------------------------------------

def _kv(st):
    """The framework's handle of this state, and its workspaces, made once."""
    from paper_2605_22106_amd import _lib as L
    if "kv" not in st:
        c = st["case"]
        st["kv"] = L.KVState(st["parent"], st["n_full"], st["tok_off"], st["page_off"],
                             st["n_kept"], st["page_table"], st["k"], st["v"], st["slot_pos"],
                             st["free_stack"], st["free_top"], c["layers"], c["heads"],
                             c["group"], c["dim"], P, L.BF16 if c["dtype"] == "bf16" else L.F32,
                             st["num_tokens"])
        st["ws"] = torch.empty(L.arbor_workspace_size(st["kv"]), dtype=torch.uint8, device="cuda")
        if c["kind"] in ("attend", "grow"):
            n, t = st["nodes"].numel(), st["n_tokens"]
            st["plan"] = torch.empty(L.arbor_prefill_plan_size(st["kv"], n, t), dtype=torch.uint8,
                                     device="cuda")
            st["attn_ws"] = torch.empty(L.arbor_prefill_workspace_size(st["kv"], n, t),
                                        dtype=torch.uint8, device="cuda")
    return L, st["kv"]


def _append(st, layer, i):
    if not own:
        return _plain_append(st, layer, i)
    from paper_2605_22106_amd import _lib as L
    case = st["case"]
    if "pool" not in st:
        z = torch.zeros(1, dtype=torch.int32, device="cuda")
        st["pool"] = st["kv"] if "kv" in st else L.KVState(
            z, z, z.long(), z.long(), z, z, st["k"], st["v"], z, z, z, 1, case["heads"],
            case["group"], case["dim"], P, L.BF16 if case["dtype"] == "bf16" else L.F32,
            st["record_k"].shape[0] if "record_k" in st else 0)
    q, k, v = _split(case, st["qkv"][i])
    L.arbor_append(st["pool"], layer, q, k, v, st["slots"], st["positions"], st["q_out"],
                   st["status"], q_norm=st["q_norm"], k_norm=st["k_norm"], eps=1e-6,
                   inv_freq=st["inv_freq"], interleaved=case["interleaved"],
                   tokens=st["tokens"] if "record_k" in st else None,
                   record_k=st.get("record_k"), record_v=st.get("record_v"))


def _plan(st):
    if not own:
        return _plain_visible(st)
    L, kv = _kv(st)
    L.arbor_prefill_plan(kv, st["nodes"], st["cu"], st["n_tokens"], st["plan"], st["status"])
    return ()


def _attend(st, layer, q, plan):
    if not own:
        return _plain_attend(st, layer, q, st["out"][layer], st["lse"][layer], *plan)
    L, kv = _kv(st)
    L.arbor_tree_prefill_attn(kv, st["plan"], st["nodes"].numel(), layer, q, st["out"][layer],
                              st["lse"][layer], 0.0, st["status"], st["attn_ws"])


def _truncate(st, nodes):
    if not own:
        return _plain_truncate(st, nodes, st["keep"])
    L, kv = _kv(st)
    L.arbor_truncate(kv, nodes, st["keep"], st["status"], st["ws"])


def _extend(st):
    if not own:
        return _plain_extend(st)
    L, kv = _kv(st)
    L.arbor_extend(kv, st["nodes"], st["cu"], st["slots"], st["positions"], st["tokens"],
                   st["status"], st["ws"])


def _fork(st):
    if not own:
        return _plain_fork(st)
    L, kv = _kv(st)
    L.arbor_fork(kv, st["src"], st["dst"], st["status"], st["ws"], A=st["A"], rows_seen=st["rows"])


def _books(st):
    return {k: st[k] for k in ("n_full", "n_kept", "page_table", "slot_pos", "free_stack",
                               "free_top", "status")}


def run(st):
    kind = st["case"]["kind"]
    if kind == "append":
        _append(st, 0, 0)
        got = dict(q=st["q_out"], k=st["k"], v=st["v"], status=st["status"])
        if "record_k" in st:
            got.update(record_k=st["record_k"], record_v=st["record_v"])
        return got
    if kind == "beam":
        _truncate(st, st["dst"])
        _fork(st)
        return dict(_books(st), k=st["k"], v=st["v"], A=st["A"], rows=st["rows"])
    if kind == "draft":
        _truncate(st, st["nodes"])
        _extend(st)
        return dict(_books(st), slots=st["slots"], positions=st["positions"], tokens=st["tokens"])
    if kind == "attend":
        plan = _plan(st)
        for layer, q in enumerate(st["q"]):
            _attend(st, layer, q, plan)
        return dict(out=st["out"], lse=st["lse"], status=st["status"])
    _truncate(st, st["nodes"])
    _extend(st)
    plan = _plan(st)
    for layer in range(st["case"]["layers"]):
        _append(st, layer, layer)
        _attend(st, layer, st["q_out"], plan)
    return dict(_books(st), slots=st["slots"], positions=st["positions"], k=st["k"], v=st["v"],
                out=st["out"], lse=st["lse"])


# ---- what a pass cannot do without ---------------------------------------------

def _attend_work(case, t):
    H, G, D, e = case["heads"], case["group"], case["dim"], _size(case)
    pairs, union = 0, set()
    for i, m in zip(t["nodes"], t["m"]):
        up = _chain(t["parent"], i)
        union.update(up)
        above = sum(t["c"][x] for x in up[:-1])
        pairs += m * (above + t["c"][i] - m) + m * (m + 1) // 2
    T = sum(t["m"])
    return dict(bytes=case["layers"] * (2 * sum(t["c"][i] for i in union) * H * D * e +
                                        T * H * G * (2 * D * e + 4)),
                flops=4.0 * D * H * G * pairs * case["layers"])


def _append_work(case, tokens, layers):
    row = (case["heads"] * (case["group"] + 2)) * case["dim"]
    extra = 2 * case["heads"] * case["dim"] * _size(case) if case.get("record") else 0
    return dict(bytes=layers * tokens * (2 * row * _size(case) + extra + 12),
                flops=10.0 * layers * tokens * row)


def work(case):
    kind = case["kind"]
    if kind == "append":
        return _append_work(case, case["tokens"], 1)
    t = _tree(case)
    if kind == "attend":
        return _attend_work(case, t)
    if kind == "beam":
        pick = random.Random(case["shape"]).sample(t["deepest"], 2 * case["pairs"])
        order = sorted(pick, key=lambda i: (t["cap"][i], i))[:case["pairs"]]
        kept = sum(t["c"][i] for i in order)
        row = 4 * case["layers"] * case["heads"] * case["dim"] * _size(case)
        return dict(bytes=kept * (row + 12) + 8 * sum(t["n"][i] for i in order), flops=0.0)
    T = sum(t["m"])
    books = dict(bytes=T * 28.0 + len(t["nodes"]) * 80.0, flops=4.0 * T)
    if kind == "draft":
        return books
    a, b = _append_work(case, T, case["layers"]), _attend_work(case, t)
    return {k: books[k] + a[k] + b[k] for k in books}


# ---- the same in 64 bits ----------------------------------------------------------

def _exact_rope(case, x, w, pos, inv):
    """Row by row of the definition: heads normed, then rotated as complex numbers."""
    x = x.double()
    if w is not None:
        x = x / (x.square().sum(-1, keepdim=True) / x.shape[-1] + 1e-6).sqrt() * w.double()
    rd = case["rotary"]
    if rd:
        y = x[..., :rd]
        y = y.unflatten(-1, (rd // 2, 2)) if case["interleaved"] else \
            y.unflatten(-1, (2, rd // 2)).transpose(-1, -2)
        angle = pos.double()[:, None, None] * inv.double()
        y = torch.view_as_real(torch.view_as_complex(y.contiguous()) *
                               torch.polar(torch.ones_like(angle), angle))
        y = y.flatten(-2) if case["interleaved"] else y.transpose(-1, -2).flatten(-2)
        x = torch.cat((y, x[..., rd:]), -1)
    return x


def _exact_attend(case, t, layer, q, k, v, page_table, page_off):
    """Sequence by sequence over its own chain; k, v [L][pages][H][P][D] in fp64."""
    H, G, D = case["heads"], case["group"], case["dim"]
    out = torch.zeros((sum(t["m"]), H * G, D), dtype=torch.float64, device="cuda")
    lse = torch.zeros((sum(t["m"]), H * G), dtype=torch.float64, device="cuda")
    at = 0
    for i, m in zip(t["nodes"], t["m"]):
        ids = []
        for x in _chain(t["parent"], i):
            s = torch.arange(t["c"][x])
            ids.append(page_table[page_off[x] + s // P] * P + s % P)
        ids = torch.cat(ids).cuda()
        kk, vv = (y[layer][ids // P, :, ids % P].double() for y in (k, v))
        late = torch.arange(ids.numel(), device="cuda")[None] > \
            (ids.numel() - m + torch.arange(m, device="cuda"))[:, None]
        for h in range(H):
            z = q[at:at + m, h * G:(h + 1) * G].double().reshape(m * G, D) @ kk[:, h].T.contiguous()
            z = (z / math.sqrt(D)).view(m, G, -1).masked_fill_(late[:, None], -math.inf)
            big = torch.logsumexp(z, -1)
            lse[at:at + m, h * G:(h + 1) * G] = big
            out[at:at + m, h * G:(h + 1) * G] = (z.sub_(big[..., None]).exp_().view(m * G, -1) @
                                                vv[:, h].contiguous()).view(m, G, D)
        at += m
    return out, lse


def exact(case, seed):
    kind = case["kind"]
    if kind in ("beam", "draft"):
        return None                     # whole numbers and copied rows
    st = prepare(case, seed)
    dt = _dt(case)
    if kind == "append":
        T = case["tokens"]
        q, k, v = (x[:T].view(T, -1, case["dim"]) for x in _split(case, st["qkv"][0]))
        pos = st["positions"][:T]
        got = dict(q=st["q_out"].double(), k=st["k"].double(), v=st["v"].double(), status=None)
        got["q"][:T] = _exact_rope(case, q, st["q_norm"], pos, st["inv_freq"])
        k = _exact_rope(case, k, st["k_norm"], pos, st["inv_freq"])
        page, row = st["slots"][:T] // P, st["slots"][:T] % P
        got["k"][0, page, :, row] = k
        got["v"][0, page, :, row] = v.double()
        if case["record"]:
            got.update(record_k=st["record_k"].double(), record_v=st["record_v"].double())
            got["record_k"][st["tokens"][:T], 0] = k
            got["record_v"][st["tokens"][:T], 0] = v.double()
        return got
    t = _tree(case)
    table, off = st["page_table"].long().cpu(), st["page_off"].tolist()
    if kind == "attend":
        pairs = [_exact_attend(case, t, i, q, st["k"], st["v"], table, off)
                 for i, q in enumerate(st["q"])]
        return dict(out=[x for x, _ in pairs], lse=[x for _, x in pairs], status=None)
    # a step: the new tokens' rows first, held in the cache's type, then their attention;
    # the tokens taken back and reserved again get the pages that they had
    H, D = case["heads"], case["dim"]
    ids, pos = [], []
    for i, m in zip(t["nodes"], t["m"]):
        s = torch.arange(t["c"][i] - m, t["c"][i])
        ids.append(table[off[i] + s // P] * P + s % P)
        above = sum(t["n"][x] for x in _chain(t["parent"], i)[:-1])
        pos.append(above + torch.arange(t["n"][i] - m, t["n"][i]))
    ids, pos = torch.cat(ids).cuda(), torch.cat(pos).cuda()
    outs, lses = [], []
    for layer in range(case["layers"]):
        q, k, v = (x.view(x.shape[0], -1, D) for x in _split(case, st["qkv"][layer]))
        q = _exact_rope(case, q, st["q_norm"], pos, st["inv_freq"]).to(dt)
        k = _exact_rope(case, k, st["k_norm"], pos, st["inv_freq"]).to(dt)
        st["k"][layer][ids // P, :, ids % P] = k
        st["v"][layer][ids // P, :, ids % P] = v
        o, l = _exact_attend(case, t, layer, q, st["k"], st["v"], table, off)
        outs.append(o)
        lses.append(l)
    return dict(n_full=None, n_kept=None, page_table=None, slot_pos=None, free_stack=None,
                free_top=None, status=None, slots=None, positions=None, k=None, v=None,
                out=outs, lse=lses)
