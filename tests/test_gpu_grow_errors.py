"""Errors that one workgroup raises while others of the same launch start: what they leave
behind is whole."""
import pytest
import torch

from paper_2605_22106_amd import _lib as L
from tests.gpu_helpers import check_rc, status, to_gpu, workspace
from tests.grow_helpers import grow_state, ragged
from tests.test_gpu_grow import append_case, split
from tests.test_gpu_prefill import Prefill, queries

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tokens,rotary,record", [(2900, 128, False), (9000, 128, True),
                                                  (5000, 64, True), (5000, 0, False)])
def test_a_bad_slot_leaves_other_tokens_whole(tokens, rotary, record):
    """The token with the bad slot is left out; each other token is written whole, queries, keys,
    values and record, or is left out too."""
    heads, group, d = 2, 4, 128
    kv, x, slots, pos = append_case("bf16", d, heads, group, tokens, 0, layers=1)
    q, k, v = split(x, heads, group, d)
    inv = torch.rand(rotary // 2, device="cuda") if rotary else None
    places = kv.num_pages * kv.page_size
    page, row = slots // kv.page_size, slots % kv.page_size
    bad = [0, tokens // 2]
    got = []
    for sl in (slots, slots.index_fill(0, torch.tensor(bad, device="cuda"), places + 5)):
        kv.k.fill_(7.0)
        kv.v.fill_(7.0)
        out = torch.full((tokens, heads * group, d), 7.0, dtype=torch.bfloat16, device="cuda")
        rec = [torch.full((kv.num_tokens, 1, heads, d), 7.0, dtype=torch.bfloat16, device="cuda")
               for _ in range(2)] if record else (None, None)
        tok = torch.arange(tokens, device="cuda") if record else None
        s = status()
        check_rc(L.arbor_append(kv, 0, q, k, v, sl, pos, out, s, inv_freq=inv, tokens=tok,
                                record_k=rec[0], record_v=rec[1]))
        parts = [out, kv.k[0][page, :, row], kv.v[0][page, :, row]]
        parts += [r[:tokens, 0] for r in rec if r is not None]
        got.append(torch.cat([p.reshape(tokens, -1) for p in parts], 1).clone())
        assert int(s) == (L.OK if sl is slots else L.EINVAL)
    clean, hit = got
    written = (hit == clean).all(1)
    untouched = (hit == 7.0).all(1)
    assert bool(untouched[bad].all()) and bool((written | untouched).all())


@pytest.mark.parametrize("lost", [1.0, 0.02])
@pytest.mark.parametrize("dtype,head_dim", [("bf16", 128), ("f32", 64)])
def test_a_stale_plan_of_many_tiles_is_refused(dtype, head_dim, lost):
    """Some or all pages of the tree have gone since the plan was made: hundreds of workgroups
    find so, thousands start meanwhile.  The error is raised and the pool stays as it was."""
    parent = [-1] + [0] * 60
    n = [4000] + ragged(3, 60, 200, 900)
    st = grow_state(parent, n, kv_heads=4, q_per_kv=8, head_dim=head_dim, dtype=dtype, layers=1)
    kv = to_gpu(st)
    m = [x - 3 for x in n[1:]]
    pf = Prefill(kv, list(range(1, 61)), m)
    q = queries(kv, sum(m))
    gone = torch.rand(kv.page_table.numel(), generator=torch.Generator().manual_seed(1)) < lost
    kv.page_table[gone.cuda()] = -1
    before = [x.clone() for x in (kv.k, kv.v, kv.slot_pos)]
    for _ in range(3):
        pf.status.zero_()
        pf(q)
        assert int(pf.status) == L.EINVAL
    for x, y in zip((kv.k, kv.v, kv.slot_pos), before):
        assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))


@pytest.mark.parametrize("blocks", [5, 5000])
def test_a_block_with_more_tokens_than_pages(blocks):
    """A malformed tree: the plan refuses it, so no entry of the page table beyond the block's
    is read.  As an ancestor, as the block itself, as the last block."""
    parent = [-1] + [0] * (blocks - 1)
    for node, bad, count in ((1, 0, 20 + 40 + 16), (2, 2, 80), (blocks - 1, blocks - 1, 1 << 30),
                             (1, 0, -1)):
        st = grow_state(parent, [20] * blocks, kv_heads=1, layers=1)
        kv = to_gpu(st)
        kv.n_kept[bad] = count
        pf = Prefill(kv, [node], [4])
        assert int(pf.status) == L.EINVAL, (node, bad)
        pf.status.zero_()
        pf(queries(kv, 4))                       # a plan that was refused is none
        assert int(pf.status) == L.EINVAL


@pytest.mark.parametrize("top", [-1, 1, 1000])
def test_a_stack_top_outside_the_stack(top):
    """extend and fork pop no page from beyond the free stack."""
    st = grow_state([-1, 0, 0, 0], [20, 33, 0, 0], kv_heads=1, layers=1, extra_pages=0)
    kv = to_gpu(st)
    kv.free_top.fill_(kv.num_pages + top if top > 0 else top)
    before = [x.clone() for x in (kv.n_full, kv.n_kept, kv.page_table, kv.slot_pos, kv.free_top)]
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    slots, pos = torch.zeros(20, dtype=torch.int64, device="cuda"), i32(*[0] * 20)
    for call in (lambda s: L.arbor_extend(kv, i32(1), i32(0, 20), slots, pos, None, s, workspace(kv)),
                 lambda s: L.arbor_fork(kv, i32(1), i32(2), s, workspace(kv))):
        s = status()
        check_rc(call(s))
        assert int(s) == L.ECORRUPT
        for x, y in zip((kv.n_full, kv.n_kept, kv.page_table, kv.slot_pos, kv.free_top), before):
            assert torch.equal(x, y)


def test_a_fork_of_more_tokens_than_the_capacity():
    st = grow_state([-1, 0, 0], [20, 0, 60], spare=[40, 500, 0], kv_heads=1, layers=1)
    kv = to_gpu(st)
    kv.n_full[2] = 61                                 # the last block: its A would end beyond N
    A = torch.ones(kv.num_tokens, device="cuda")
    s = status()
    one, two = (torch.tensor([x], dtype=torch.int32, device="cuda") for x in (1, 2))
    check_rc(L.arbor_fork(kv, two, one, s, workspace(kv), A=A))
    assert int(s) == L.EINVAL and int(kv.n_kept[1]) == 0 and bool((A == 1).all())
