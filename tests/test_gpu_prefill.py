"""arbor_prefill_plan and arbor_tree_prefill_attn against the oracle and 64-bit torch."""
import random

import numpy as np
import pytest
import torch

from oracle import arbor_oracle as O
from paper_2605_22106_amd import _lib as L
from tests.gpu_helpers import check_rc, status, to_gpu
from tests.grow_helpers import attention_bounds, cu_of, grow_state, ragged, reference
from tests.helpers import oracle_state

pytestmark = pytest.mark.gpu


def i32(x):
    return torch.tensor([int(y) for y in x], dtype=torch.int32, device="cuda")


class Prefill:
    """A plan and what its calls need."""

    def __init__(self, kv, nodes, m, pad=0):
        self.kv, self.nodes, self.cu = kv, i32(nodes), i32(cu_of(m))
        self.T = sum(m) + pad
        self.status = status()
        self.plan = torch.empty(L.arbor_prefill_plan_size(kv, len(nodes), self.T),
                                dtype=torch.uint8, device="cuda")
        self.ws = torch.empty(L.arbor_prefill_workspace_size(kv, len(nodes), self.T),
                              dtype=torch.uint8, device="cuda")
        self.make()

    def make(self):
        check_rc(L.arbor_prefill_plan(self.kv, self.nodes, self.cu, self.T, self.plan, self.status))

    def __call__(self, q, layer=0, lse=True, scale=0.0, out=None):
        out = torch.full_like(q, 7.0) if out is None else out
        l = torch.full(q.shape[:2], 7.0, device="cuda") if lse else None
        check_rc(L.arbor_tree_prefill_attn(self.kv, self.plan, self.nodes.numel(), layer, q, out, l,
                                           scale, self.status, self.ws))
        return out, l


def queries(kv, T, seed=0, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    q = torch.randn((T, kv.kv_heads * kv.q_per_kv, kv.head_dim), generator=g) * scale
    return q.to(kv.k.dtype).cuda()


def check(got, want, dtype, D):
    out, lse = got
    ref, rl, mass, big = (x if torch.is_tensor(x) else torch.tensor(x) for x in want)
    ref, rl, mass, big = (x.to(out.device) for x in (ref, rl, mass, big))
    tol, ltol = attention_bounds(dtype, D, ref, rl, mass, big)
    assert bool(torch.isfinite(out).all())
    worst = ((out.double() - ref).abs() / tol).max()
    assert worst <= 1, float(worst)
    if lse is not None:
        worst = ((lse.double() - rl).abs() / ltol).max()
        assert worst <= 1, float(worst)


TREE = [-1, 0, 0, 1, 1, 2, 2, 3, 4, 4]
SMALL = [  # dtype, d, kv heads, group, page size, nodes, new tokens
    ("f32", 64, 2, 1, 16, [7, 8, 9], [1, 1, 1]),
    ("f32", 128, 1, 4, 16, [0], [40]),
    ("bf16", 128, 2, 4, 16, [3, 5, 9], [1, 17, 40]),
    ("bf16", 64, 1, 8, 32, [7, 8, 9], [16, 0, 3]),
    ("bf16", 128, 1, 3, 16, [1, 3, 7, 9], [5, 33, 8, 2]),     # 3 and 7 lie below 1, 7 below 3
    ("f32", 64, 1, 7, 256, [5, 6], [19, 23]),
    ("bf16", 64, 3, 1, 16, [0, 2, 6], [37, 12, 1]),
    ("bf16", 128, 1, 128, 16, [4, 9], [3, 2]),
    ("f32", 128, 2, 5, 16, [9, 4, 4], [2, 9, 9]),             # any order, one block twice
]


@pytest.mark.parametrize("case", SMALL, ids=lambda c: "-".join(map(str, c[:5])))
@pytest.mark.parametrize("evicted", [False, True])
def test_small_against_the_oracle(case, evicted):
    dtype, d, H, G, P, nodes, m = case
    n = ragged(3, len(TREE), 41, 75)
    c = [random.Random(i).randint(2, x) if evicted else x for i, x in enumerate(n)]
    for i, x in zip(nodes, m):
        c[i] = max(c[i], 2 * x + 1)                # new tokens are resident
        n[i] = max(n[i], c[i])
    st = grow_state(TREE, n, c, kv_heads=H, q_per_kv=G, head_dim=d, dtype=dtype, page_size=P, seed=5)
    kv, pad = to_gpu(st), 3
    pf = Prefill(kv, nodes, m, pad)
    q = queries(kv, sum(m) + pad)
    q[sum(m):] = float("nan")
    for layer in (0, 1):
        out, lse = pf(q, layer)
        assert int(pf.status) == 0
        T = sum(m)
        assert bool((out[T:] == 7.0).all()) and bool((lse[T:] == 7.0).all())
        want = O.prefill_attn(oracle_state(st), nodes, cu_of(m), layer,
                              q[:T].float().cpu().numpy(), G)
        check((out[:T], lse[:T]), want, dtype, d)


LARGE = [  # dtype, d, heads, group, parent, resident, nodes, new tokens
    ("bf16", 128, 2, 4, [-1], [0], [0], [1500]),
    ("bf16", 128, 8, 8, [-1], [0], [0], [333]),
    ("bf16", 64, 4, 2, [-1], [0], [0], [2049]),
    ("f32", 128, 2, 4, [-1], [0], [0], [700]),
    ("f32", 64, 1, 1, [-1, 0], [900, 77], [1], [260]),
    ("bf16", 128, 8, 4, [-1] + [0] * 20, [9000] + ragged(1, 20, 0, 90), list(range(1, 21)),
     ragged(2, 20, 1, 9)),
    ("bf16", 128, 1, 4, [-1] + [0] * 70, [1200] + ragged(1, 70, 0, 40), list(range(1, 71)),
     [1] * 70),
    ("bf16", 128, 1, 1, [-1] + [0] * 200, [300] + ragged(1, 200, 0, 20), list(range(1, 201)),
     ragged(4, 200, 0, 3)),
    ("bf16", 64, 2, 1, list(range(-1, 63)), ragged(6, 64, 1, 30), [20, 40, 63], [50, 3, 130]),
    ("bf16", 128, 2, 4, [-1, 0, 0, 1, 1, 2], [5000, 400, 300, 0, 17, 1000], [3, 4, 5],
     [31, 600, 129]),
    ("bf16", 128, 2, 4, [-1], [40000], [0], [2]),
    ("f32", 64, 1, 2, [-1, 0], [30000, 3], [1], [5]),
]


@pytest.mark.parametrize("case", LARGE, ids=lambda c: f"{c[0]}-{c[1]}-{c[2]}x{c[3]}-{len(c[4])}-"
                                                      f"{sum(c[5])}-{sum(c[7])}")
def test_large_against_64_bits(case):
    dtype, d, H, G, parent, had, nodes, m = case
    n = list(had)
    for i, x in zip(nodes, m):
        n[i] += x
    st = grow_state(parent, n, kv_heads=H, q_per_kv=G, head_dim=d, dtype=dtype, seed=8, layers=1,
                    k_scale=1.5)
    kv = to_gpu(st)
    pf = Prefill(kv, nodes, m)
    q = queries(kv, sum(m))
    got = pf(q)
    assert int(pf.status) == 0
    dev = {k: v.cuda() if torch.is_tensor(v) else v for k, v in st.items()}
    check(got, reference(dev, parent, nodes, m, 0, q, G), dtype, d)
    again = pf(q)
    assert torch.equal(got[0], again[0]) and torch.equal(got[1], again[1])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_logits_that_grow_and_shrink_along_the_chain(dtype):
    """The reference max moves late, or the first keys outweigh all others; all logits far
    below zero; a scale of the caller's."""
    n = [400, 300]
    st = grow_state([-1, 0], n, kv_heads=1, q_per_kv=2, head_dim=64, dtype=dtype, layers=1, seed=2)
    kv = to_gpu(st)
    q = queries(kv, 20, seed=3)
    pf = Prefill(kv, [1], [20])
    dev = {k: v.cuda() if torch.is_tensor(v) else v for k, v in st.items()}
    direction = q.float().mean(dim=(0, 1))
    direction /= direction.norm()
    table = st["page_table"].long()
    first = int(table[0])                                   # pages of the root's first tokens
    last = int(table[int(st["page_off"][1]) + (n[1] - 1) // 16])     # and of the newest
    base = kv.k.clone()
    for page, by in ((first, 60.0), (last, 60.0), (first, -60.0)):
        kv.k.copy_(base)
        kv.k[0, page, 0] = (direction * by).to(kv.k.dtype)
        dev["k"] = kv.k
        for scale in (0.0, 0.5):
            check(pf(q, scale=scale), reference(dev, [-1, 0], [1], [20], 0, q, 2,
                                                scale=scale or None), dtype, 64)
    kv.k[0, :, 0] = (-50 * direction).to(kv.k.dtype)        # equal logits, all far below zero
    check(pf(q), reference(dev, [-1, 0], [1], [20], 0, q, 2), dtype, 64)


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 64), ("f32", 128)])
@pytest.mark.parametrize("what", ["inf", "nan"])
def test_what_is_not_seen_has_no_influence(dtype, d, what):
    """Infinite or NaN keys and values of later tokens and of other blocks in the same tile."""
    bad = float(what)
    n = [50, 40, 45, 61]
    parent, nodes, m = [-1, 0, 0, 0], [1, 2, 3], [7, 9, 20]
    st = grow_state(parent, n, kv_heads=2, q_per_kv=2, head_dim=d, dtype=dtype, layers=1, seed=4)
    kv = to_gpu(st)
    q = queries(kv, sum(m), seed=1)
    clean = Prefill(kv, nodes, m)(q)
    poison = {2: n[2] - 4, 3: n[3] - 11}              # a token of two of the blocks
    for i, slot in poison.items():
        page = int(st["page_table"][int(st["page_off"][i]) + slot // 16])
        kv.k[0, page, :, slot % 16, 3] = bad
        kv.v[0, page, :, slot % 16, 5:] = bad
    out, lse = Prefill(kv, nodes, m)(q)
    sees = torch.zeros(sum(m), dtype=torch.bool)
    at = 0
    for i, mm in zip(nodes, m):
        for j in range(mm):
            sees[at + j] = i in poison and n[i] - mm + j >= poison[i]
        at += mm
    # the last bits may differ: a unit with such values is summed key by key
    a, b = out[~sees].double(), clean[0][~sees].double()
    step = 2.0 ** -7 if dtype == "bf16" else 2.0 ** -20
    assert bool(torch.isfinite(a).all()) and bool(((a - b).abs() <= step * (b.abs() + 1.0)).all())
    assert bool(((lse[~sees] - clean[1][~sees]).abs() <= 1e-5).all())
    assert not bool(torch.isfinite(out[sees][..., 5:]).any())


def test_a_block_that_is_both_grown_and_an_ancestor():
    """The tokens of a parent are causal among themselves, and whole for its children."""
    parent, had, nodes, m = [-1, 0, 1, 1], [33, 10, 0, 4], [1, 2, 3], [20, 6, 9]
    n = [had[0], had[1] + 20, 6, 13]
    st = grow_state(parent, n, kv_heads=2, q_per_kv=1, head_dim=64, layers=1, seed=6)
    kv = to_gpu(st)
    q = queries(kv, 35)
    want = O.prefill_attn(oracle_state(st), nodes, cu_of(m), 0, q.cpu().numpy(), 1)
    check(Prefill(kv, nodes, m)(q), want, "f32", 64)


def test_device_refusals():
    st = grow_state(TREE, [20] * 10, kv_heads=1, layers=1)
    kv = to_gpu(st)
    q = queries(kv, 4)
    for nodes, cu in (([10], [0, 4]), ([-1], [0, 4]), ([1, 2], [0, 3, 2]), ([1], [1, 4]),
                      ([1], [0, 5]), ([1], [0, 21])):
        pf = Prefill(kv, [0] * len(nodes), [0] * len(nodes), 4 if cu[-1] < 20 else 21)
        pf.nodes, pf.cu, pf.status = i32(nodes), i32(cu), status()
        pf.make()
        assert int(pf.status) == L.EINVAL, (nodes, cu)
    # a plan that was never made, one of another call, a tree that lost its pages
    pf = Prefill(kv, [1], [4])
    size = pf.plan.numel()
    for plan in (torch.zeros_like(pf.plan), Prefill(kv, [1, 2], [2, 2]).plan[:size],
                 Prefill(kv, [1], [5]).plan[:size]):
        pf.plan, pf.status = plan, status()
        pf(q)
        assert int(pf.status) == L.EINVAL
    pf = Prefill(kv, [1], [4])
    kv.page_table.fill_(-1)
    pf(q)
    assert int(pf.status) == L.EINVAL


def test_too_deep():
    V = 66
    st = grow_state(list(range(-1, V - 1)), [3] * V, layers=1, kv_heads=1)
    kv = to_gpu(st)
    assert int(Prefill(kv, [63], [2]).status) == 0
    assert int(Prefill(kv, [64], [2]).status) == L.EUNSUPPORTED
    kv.parent[5] = 7
    assert int(Prefill(kv, [63], [2]).status) == L.EINVAL


def test_nothing_to_do():
    st = grow_state([-1], [20], layers=1)
    kv = to_gpu(st)
    pf = Prefill(kv, [0], [0])                         # no rows at all
    pf(queries(kv, 0))
    pf = Prefill(kv, [0, 0], [0, 0], 5)                # padding only
    out, lse = pf(queries(kv, 5))
    assert int(pf.status) == 0 and bool((out == 7.0).all()) and bool((lse == 7.0).all())
    none = torch.empty(0, dtype=torch.int32, device="cuda")
    assert L.arbor_prefill_plan(kv, none, i32([0]), 3, pf.plan, pf.status) == L.OK
