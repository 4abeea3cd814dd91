"""Pins of the oracle's operators that grow a tree: extend, truncate, fork, norm_rotate and
prefill_attn against closed forms, invariants and textbook routines."""
import math
import random

import numpy as np
import pytest
import torch

from oracle import arbor_oracle as O
from tests.grow_helpers import assert_same_books, cu_of, grow_state, ragged
from tests.helpers import oracle_state

PARENT = [-1, 0, 0, 1, 1, 2, 3]


def _state(seed=0, **kw):
    n = ragged(seed, len(PARENT), 1, 40)
    c = [random.Random(seed + i).randint(0, x) for i, x in enumerate(n)]
    return oracle_state(grow_state(PARENT, n, c, page_size=4, seed=seed, **kw))


def _pages_in_use(st):
    used = [int(p) for p in st["page_table"] if p >= 0]
    return sorted(used + [int(p) for p in st["free_stack"][:int(st["free_top"])]])


@pytest.mark.parametrize("seed", range(6))
def test_extend_reserves_and_truncate_undoes(seed):
    st = _state(seed)
    nodes, m = [2, 3, 6], ragged(seed + 9, 3, 0, 11)
    cu = np.array(cu_of(m))
    new, slots, pos, tok, rc = O.extend(st, nodes, cu, int(cu[-1]) + 3)
    assert rc == O.OK and _pages_in_use(new) == list(range(st["k"].shape[1]))
    assert len(set(slots[:cu[-1]])) == cu[-1]
    assert list(slots[cu[-1]:]) == [-1] * 3 and list(tok[cu[-1]:]) == [-1] * 3
    for e, i in enumerate(nodes):
        got = O.retained(new, i)
        assert [r[3] for r in got][len(got) - m[e]:] == list(range(st["n_full"][i],
                                                                   st["n_full"][i] + m[e]))
        assert [p * 4 + r for _, p, r, _ in got][len(got) - m[e]:] == list(slots[cu[e]:cu[e + 1]])
        # positions go on where the chain's tokens end, grown ancestors included
        above = sum(int(new["n_full"][x]) for x in O.chain(PARENT, i)[:-1])
        assert list(pos[cu[e]:cu[e + 1]]) == [above + int(st["n_full"][i]) + j for j in range(m[e])]
    back, rc = O.truncate(new, nodes, [int(st["n_full"][i]) for i in nodes])
    assert rc == O.OK
    assert_same_books(back, st)


def test_truncate_keeps_positions_below():
    st = _state(3)
    for kp in (0, 1, 7, 1000):
        new, _ = O.truncate(st, [0, 4], [kp, kp])
        for i in (0, 4):
            assert [r[3] for r in O.retained(new, i)] == [r[3] for r in O.retained(st, i)
                                                          if r[3] < kp]
            assert new["n_full"][i] == min(kp, st["n_full"][i])
        assert _pages_in_use(new) == _pages_in_use(st)


def test_fork_copies():
    st = _state(4, extra_pages=20)
    st, _ = O.truncate(st, [3, 4, 5], [0, 0, 0])
    # (capacities differ: what fits is what the sources hold)
    A, rows = np.arange(int(st["tok_off"][-1]), dtype=np.float32), np.arange(7)
    st["n_full"][2] = min(st["n_full"][2], 5)
    st, _ = O.truncate(st, [2], [5])
    new, A2, rows2, rc = O.fork(st, [2, 2, 3], [3, 4, 5], A, rows)
    assert rc == O.OK and _pages_in_use(new) == _pages_in_use(st)
    want = [r[3] for r in O.retained(st, 2)]
    for b in (3, 4):
        assert [r[3] for r in O.retained(new, b)] == want and rows2[b] == 2
        for (_, p, r, _), (_, q, s, _) in zip(O.retained(st, 2), O.retained(new, b)):
            assert np.array_equal(st["k"][:, p, :, r], new["k"][:, q, :, s])
        t2, tb, n = int(st["tok_off"][2]), int(st["tok_off"][b]), int(st["n_full"][2])
        assert np.array_equal(A2[tb:tb + n], A[t2:t2 + n])
    assert new["n_kept"][5] == 0 and rows2[5] == 3        # block 3 was empty before the call


def test_refusals():
    st = _state(5)
    room = int(st["tok_off"][1] - st["tok_off"][0] - st["n_full"][0])
    for nodes, cu in (([1, 1], [0, 1, 2]), ([2, 1], [0, 1, 2]), ([7], [0, 1]), ([-1], [0, 1]),
                      ([1, 2], [0, 2, 1]), ([1], [1, 2]), ([1], [0, 9]), ([0], [0, room + 1])):
        n = 8 if cu[-1] <= 9 else cu[-1]
        assert O.extend(st, nodes, np.array(cu), n)[-1] == O.EINVAL
    st["free_top"] = np.int64(0)
    assert O.extend(st, [1], np.array([0, 20]), 20)[-1] == O.ENOPAGES
    assert O.truncate(st, [1], [-1])[-1] == O.EINVAL
    assert O.fork(st, [1], [2])[-1] == O.EINVAL


def test_norm_rotate_closed_forms():
    rng = np.random.default_rng(0)
    x = rng.normal(size=(5, 3, 16))
    inv = np.array([1.0, 0.1, 0.01, 0.001])
    # position 0 turns nothing; a norm of a constant head is the weight
    assert np.array_equal(O.norm_rotate(x, None, 0.0, np.zeros(5), inv, False)[0], x)
    y, _ = O.norm_rotate(np.full((1, 1, 16), 3.0), np.arange(16.0), 0.0, [0], None, False)
    assert np.allclose(y[0, 0], np.arange(16.0), rtol=1e-15)
    # lengths of pairs stay, elements beyond the rotary part stay
    for inter in (False, True):
        y, _ = O.norm_rotate(x, None, 0.0, np.arange(5) * 1000.0, inv, inter)
        assert np.allclose((y ** 2).sum(-1), (x ** 2).sum(-1)) and np.array_equal(y[..., 8:], x[..., 8:])
    # products of two heads depend on the difference of their positions alone
    q, k = x[:1], x[1:2]
    dot = lambda a, b: (O.norm_rotate(q, None, 0, [a], inv, True)[0] *  # noqa: E731
                        O.norm_rotate(k, None, 0, [b], inv, True)[0]).sum()
    assert math.isclose(dot(7, 3), dot(1007, 1003), rel_tol=1e-9)
    # a complex product, by hand
    y, _ = O.norm_rotate(np.array([[[1.0, 0.0]]]), None, 0, [2], np.array([0.25]), False)
    assert np.allclose(y[0, 0], [math.cos(0.5), math.sin(0.5)])


@pytest.mark.parametrize("seed", range(3))
def test_prefill_attn_is_the_dense_causal_softmax(seed):
    st = _state(seed, kv_heads=2, head_dim=8)
    c = st["n_kept"]
    nodes = [i for i in (0, 4, 6) if c[i] > 0]
    m = [min(int(c[i]), 1 + 2 * seed) for i in nodes]
    rng = np.random.default_rng(seed)
    q = rng.normal(size=(sum(m), 4, 8))
    out, lse, mass, big = O.prefill_attn(st, nodes, cu_of(m), 1, q, 2)
    at = 0
    for i, mm in zip(nodes, m):
        rows = [r for x in O.chain(PARENT, i) for r in O.retained(st, x)]
        k = np.stack([st["k"][1][p, :, r] for _, p, r, _ in rows])
        v = np.stack([st["v"][1][p, :, r] for _, p, r, _ in rows])
        n = len(rows)
        mask = torch.arange(n)[None] <= (n - mm + torch.arange(mm))[:, None]
        t = lambda x: torch.tensor(x).double().transpose(0, 1)  # noqa: E731
        want = torch.nn.functional.scaled_dot_product_attention(
            t(q[at:at + mm]), t(k).repeat_interleave(2, 0), t(v).repeat_interleave(2, 0),
            attn_mask=mask)
        assert np.allclose(out[at:at + mm], want.transpose(0, 1).numpy(), rtol=1e-12, atol=1e-12)
        at += mm
    assert np.all(mass >= np.abs(out) - 1e-12) and np.all(np.isfinite(lse)) and np.all(big > 0)


def test_prefill_attn_of_one_token_is_the_decode():
    st = _state(1, kv_heads=2, head_dim=8)
    leaf = 6 if st["n_kept"][6] else 3
    q = np.random.default_rng(1).normal(size=(1, 4, 8))
    out, lse, _, _ = O.prefill_attn(st, [leaf], [0, 1], 0, q, 2)
    o, l = O.tree_decode_attn(st, [leaf], 0, 1, q[:, None], 2)
    assert np.allclose(out[0], o[0, 0], rtol=1e-6) and np.allclose(lse[0], l[0, 0], rtol=1e-6)
