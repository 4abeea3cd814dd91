"""arbor_truncate_scored: tokens taken back leave no accumulated attention to those that get
their positions next."""
import random

import numpy as np
import pytest
import torch

from oracle import arbor_oracle as O
from paper_2605_22106_amd import _lib as L
from tests.grow_helpers import assert_same_books, cu_of, grow_state, ragged
from tests.helpers import oracle_state
from tests.test_grow_refusals import PTR, call, geom, pool, ref, tree

PARENT = [-1, 0, 0, 1, 1, 2, 3]


def i32(x):
    return torch.tensor([int(y) for y in x], dtype=torch.int32, device="cuda")


def test_the_oracle_clears_what_is_taken_back():
    n = ragged(1, len(PARENT), 5, 40)
    c = [random.Random(i).randint(0, x) for i, x in enumerate(n)]
    st = oracle_state(grow_state(PARENT, n, c, page_size=4))
    A = np.arange(1, int(st["tok_off"][-1]) + 1, dtype=np.float32)
    rows = np.arange(1, len(PARENT) + 1)
    nodes, keep = [1, 3, 4, 6], [0, 2, 1000, 0]
    new, A2, rows2, rc = O.truncate_scored(st, nodes, keep, A, rows)
    assert rc == O.OK
    assert_same_books(new, O.truncate(st, nodes, keep)[0])
    want = A.copy()
    for i, k in zip(nodes, keep):
        at = int(st["tok_off"][i])
        want[at + min(k, n[i]):at + n[i]] = 0       # not beyond n_i: nothing was there
    assert np.array_equal(A2, want) and list(rows2) == [1, 0, 3, 4, 5, 6, 0]


def test_host_refusals():
    def run(n=2, nodes=PTR, keep=PTR, A=PTR, rows=PTR, n_full=PTR, st=PTR):
        return call("arbor_truncate_scored", ref(geom()), ref(tree()), ref(pool()), n_full, nodes,
                    keep, n, A, rows, st, None, 0, None)
    for bad in (dict(nodes=None), dict(keep=None), dict(A=None), dict(rows=None), dict(n=-1),
                dict(n=11), dict(n_full=8), dict(st=None)):
        assert run(**bad) == L.EINVAL, bad
    assert run() == L.EWORKSPACE
    assert run(n=0, nodes=None, keep=None, A=None, rows=None) == L.OK


@pytest.mark.gpu
@pytest.mark.parametrize("blocks", [7, 1500])
def test_against_the_oracle(blocks):
    from tests.gpu_helpers import check_rc, gpu_to_oracle, status, to_gpu, workspace
    parent = [-1] + [(i - 1) // 2 for i in range(1, blocks)]
    n = ragged(2, blocks, 0, 40)
    n[3] = 3000
    c = [random.Random(i).randint(0, x) for i, x in enumerate(n)]
    st = grow_state(parent, n, c, layers=1, kv_heads=1)
    ost, kv = oracle_state(st), to_gpu(st)
    A = torch.rand(kv.num_tokens, device="cuda") + 1
    rows = torch.arange(1, blocks + 1, device="cuda")
    nodes = sorted(random.Random(4).sample(range(blocks), blocks * 3 // 4) + [3])
    nodes = sorted(set(nodes))
    keep = [random.Random(i).choice([0, 1, 15, 16, 4000]) for i in nodes]
    want, A2, rows2, _ = O.truncate_scored(ost, nodes, keep, A.cpu().numpy(), rows.cpu().numpy())
    s = status()
    check_rc(L.arbor_truncate_scored(kv, i32(nodes), i32(keep), A, rows, s, workspace(kv)))
    assert int(s) == 0
    assert_same_books(gpu_to_oracle(kv), want)
    assert np.array_equal(A.cpu().numpy(), A2) and np.array_equal(rows.cpu().numpy(), rows2)


@pytest.mark.gpu
def test_device_refusals_change_nothing():
    from tests.gpu_helpers import check_rc, gpu_to_oracle, status, to_gpu, workspace
    st = grow_state(PARENT, [20] * 7, layers=1, kv_heads=1)
    ost, kv = oracle_state(st), to_gpu(st)
    A, rows = torch.ones(kv.num_tokens, device="cuda"), torch.ones(7, dtype=torch.int64, device="cuda")

    def refused(nodes, keep, code, s=None):
        s = status() if s is None else s
        check_rc(L.arbor_truncate_scored(kv, i32(nodes), i32(keep), A, rows, s, workspace(kv)))
        assert int(s) == code and bool((A == 1).all()) and bool((rows == 1).all())
        assert_same_books(gpu_to_oracle(kv), ost)
    for nodes, keep in (([1, 1], [0, 0]), ([9], [0]), ([1, 2], [0, -1])):
        refused(nodes, keep, L.EINVAL)
    refused([1], [0], L.ENOPAGES, torch.tensor([L.ENOPAGES], dtype=torch.int32, device="cuda"))
    kv.n_full[6] = ost["n_full"][6] = 61                       # of a capacity of 60
    refused([2, 6], [0, 0], L.EINVAL)


@pytest.mark.gpu
def test_a_second_draft_starts_from_nothing():
    """Drafts are decoded with their attention accumulated, taken back, and others reserved in
    their place."""
    from tests.gpu_helpers import check_rc, status, to_gpu, workspace
    st = grow_state(PARENT, [20, 30, 9, 17, 4, 11, 6], layers=2, kv_heads=2, q_per_kv=2, extra_pages=9)
    kv = to_gpu(st)
    V, N, nodes, m = kv.num_nodes, kv.num_tokens, [4, 5, 6], [5, 33, 1]
    s, ws = status(), workspace(kv, n_slice=1, max_leaves=3, max_layers=2)
    A = torch.zeros(N, device="cuda")
    rows = torch.zeros(V, dtype=torch.int64, device="cuda")
    T = sum(m)
    slots, tok = (torch.empty(T, dtype=torch.int64, device="cuda") for _ in range(2))
    pos = torch.empty(T, dtype=torch.int32, device="cuda")
    x = torch.randn((T, 8 * 64), device="cuda")

    def draft():
        check_rc(L.arbor_extend(kv, i32(nodes), i32(cu_of(m)), slots, pos, tok, s, ws))
        for layer in range(2):
            check_rc(L.arbor_append(kv, layer, x[:, :256], x[:, 256:384], x[:, 384:], slots, pos,
                                    torch.empty((T, 4, 64), device="cuda"), s))

    def credit():
        q = torch.randn((3, 2, 4, 64), device="cuda")
        check_rc(L.arbor_tree_decode_attn_scored(kv, i32(nodes), 0, 2, q, torch.empty_like(q), None,
                                                 0.0, [1], 1, A, rows, s, ws))
    keep = kv.n_full[i32(nodes).long()].clone()
    draft()
    credit()
    old = A.clone()
    assert bool((A[tok[:4]] > 0).all()) and int(s) == 0       # (all but a block's newest token)
    check_rc(L.arbor_truncate_scored(kv, i32(nodes), keep, A, rows, s, ws))
    draft()
    assert int(s) == 0 and not bool(A[tok].any())
    rest = torch.ones(N, dtype=torch.bool, device="cuda")
    rest[tok] = False
    assert torch.equal(A[rest], old[rest])
    seen = rows.clone()
    check_rc(L.arbor_truncate_scored(kv, i32(nodes), i32([0] * 3), A, rows, s, ws))
    assert rows[nodes].tolist() == [0] * 3 and torch.equal(rows[:4], seen[:4])
