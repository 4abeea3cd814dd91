"""What a token may not see, and the queries of other tokens, leave every bit of its output and
LSE as they were."""
import pytest
import torch

from tests.gpu_helpers import to_gpu
from tests.grow_helpers import grow_state, ragged
from tests.test_gpu_prefill import Prefill, queries

pytestmark = pytest.mark.gpu

TYPES = [("bf16", 128), ("bf16", 64), ("f32", 64), ("f32", 128)]
CASES = {                                   # parent, tokens, blocks that grow, by how much
    "one tile": ([-1, 0, 0, 0], [50, 40, 45, 61], [1, 2, 3], [7, 9, 20]),
    "parts": ([-1, 0, 0, 0], [6000, 40, 45, 61], [1, 2, 3], [7, 9, 20]),
    "tiles": ([-1, 0, 0, 1], [300, 400, 290, 333], [1, 2, 3], [150, 200, 290]),
    "leaves": ([-1] + [0] * 40, [1500] + ragged(1, 40, 20, 90), list(range(1, 41)),
               ragged(2, 40, 1, 9)),
}


def sees(nodes, n, m, parent, poison):
    """Whether each new token sees a slot of `poison` ({block: slot})."""
    got = []
    for i, mm in zip(nodes, m):
        up, x = set(), parent[i]
        while x >= 0:
            up.add(x)
            x = parent[x]
        for j in range(mm):
            own = n[i] - mm + j
            got.append(any(b in up or (b == i and s <= own) for b, s in poison.items()))
    return torch.tensor(got, device="cuda")


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("case", CASES)
@pytest.mark.parametrize("value", [float("inf"), float("-inf"), float("nan"), 3e4])
def test_hidden_keys_and_values(dtype, d, case, value):
    parent, n, nodes, m = CASES[case]
    st = grow_state(parent, n, kv_heads=2, q_per_kv=2, head_dim=d, dtype=dtype, layers=1, seed=4)
    kv = to_gpu(st)
    q = queries(kv, sum(m), seed=1)
    pf = Prefill(kv, nodes, m)
    clean, lse = pf(q)
    poison = {i: n[i] - max(1, mm // 2) for i, mm in list(zip(nodes, m))[1:3]}
    for i, slot in poison.items():
        page = int(st["page_table"][int(st["page_off"][i]) + slot // 16])
        kv.k[0, page, :, slot % 16, 3] = value
        kv.v[0, page, :, slot % 16, 5:9] = value
    out, lse2 = pf(q)
    blind = ~sees(nodes, n, m, parent, poison)
    assert bool(blind.any()) and not bool(blind.all())
    assert torch.equal(out[blind], clean[blind]) and torch.equal(lse2[blind], lse[blind])
    if value != 3e4:
        assert not bool(torch.isfinite(out[~blind][..., 5:9]).any())


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("case", CASES)
@pytest.mark.parametrize("factor", [100.0, float("nan"), float("inf"), 0.0])
def test_other_queries(dtype, d, case, factor):
    parent, n, nodes, m = CASES[case]
    st = grow_state(parent, n, kv_heads=2, q_per_kv=3, head_dim=d, dtype=dtype, layers=1, seed=5)
    kv = to_gpu(st)
    q = queries(kv, sum(m), seed=2)
    pf = Prefill(kv, nodes, m)
    clean, lse = pf(q)
    other = torch.zeros(q.shape[:2], dtype=torch.bool, device="cuda")
    other[1::3], other[:, 1] = True, True             # some tokens, and one head of all
    q2 = q.clone()
    q2[other] *= factor
    out, lse2 = pf(q2)
    assert torch.equal(out[~other], clean[~other]) and torch.equal(lse2[~other], lse[~other])
