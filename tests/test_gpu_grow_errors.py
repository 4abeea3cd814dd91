"""Errors that one workgroup raises while others of the same launch start: what they leave
behind is whole."""
import pytest
import torch

from paper_2605_22106_amd import _lib as L
from tests.gpu_helpers import check_rc, status
from tests.test_gpu_grow import append_case, split

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tokens,rotary,record", [(5000, 128, False), (9000, 128, True),
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
