"""One block's few tokens in a buffer made for many (a captured step): the split over a long
prompt goes by the tokens that are there."""
import pytest
import torch

from tests.gpu_helpers import to_gpu
from tests.grow_helpers import grow_state, reference
from tests.test_gpu_prefill import Prefill, check, queries

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("live,rows", [(8, 4096), (300, 9000), (4096, 4096), (1, 70000)])
def test_one_block_in_a_long_buffer(live, rows):
    parent, n = [-1, 0], [20000, live + 5]
    st = grow_state(parent, n, kv_heads=8, q_per_kv=4, head_dim=128, dtype="bf16", layers=1)
    kv = to_gpu(st)
    pf, alone = Prefill(kv, [1], [live], rows - live), Prefill(kv, [1], [live])
    q = queries(kv, rows)
    out, lse = pf(q)
    assert int(pf.status) == 0
    assert bool((out[live:] == 7.0).all()) and bool((lse[live:] == 7.0).all())
    dev = {k: v.cuda() if torch.is_tensor(v) else v for k, v in st.items()}
    check((out[:live], lse[:live]), reference(dev, parent, [1], [live], 0, q[:live], 4), "bf16", 128)
    want = alone(q[:live])
    assert torch.equal(out[:live], want[0]) and torch.equal(lse[:live], want[1])
    # the plan's header: magic, then nine counts of which the last are tiles, units and tiles
    # that are cut
    counts = [p.plan[8:44].view(torch.int32)[6:].tolist() for p in (pf, alone)]
    assert counts[0] == counts[1] and (counts[0][2] > 0) == (live < 4096)
