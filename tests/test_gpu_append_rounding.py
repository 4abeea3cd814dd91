"""Every bf16 that arbor_append writes is the 64-bit value, rounded: where fp32 leaves open
which of two neighbours that is, also where the terms of a rotation cancel."""
import pytest
import torch

from paper_2605_22106_amd import _lib as L
from tests.gpu_helpers import check_rc, status
from tests.test_gpu_grow import append_case, split

pytestmark = pytest.mark.gpu

EPS = 2.0 ** -17                             # the same number in 32 and 64 bits


def exact(x, w, pos, inv, interleaved):
    """Norm and rotation of heads x [T][heads][d] in 64 bits."""
    x = x.double()
    if w is not None:
        x = x / (x.square().mean(-1, keepdim=True) + EPS).sqrt() * w.double()
    if inv is None:
        return x
    rd = 2 * inv.numel()
    a, b = x[..., :rd // 2], x[..., rd // 2:rd]
    if interleaved:
        a, b = x[..., 0:rd:2], x[..., 1:rd:2]
    ang = pos.double()[:, None, None] * inv.double()
    c, s = ang.cos(), ang.sin()
    y = x.clone()
    u, v = a * c - b * s, b * c + a * s
    if interleaved:
        y[..., 0:rd:2], y[..., 1:rd:2] = u, v
    else:
        y[..., :rd // 2], y[..., rd // 2:rd] = u, v
    return y


@pytest.mark.parametrize("d,tokens,rotary,interleaved,norm", [
    (128, 3000, 128, False, True), (128, 9000, 128, False, True), (128, 9000, 128, True, True),
    (64, 8500, 64, False, True), (64, 2000, 64, True, False), (128, 3000, 64, False, True),
    (64, 3000, 32, False, False), (128, 2500, 0, False, True)])
def test_bf16_results_are_the_64_bit_values_rounded(d, tokens, rotary, interleaved, norm):
    heads, group = 2, 8
    kv, x, slots, pos = append_case("bf16", d, heads, group, tokens, 0, layers=1)
    # near positions: both sides are within 1e-12 of the definition, and of these millions of
    # results hardly one lies so near the middle of two bf16 (5e-10 each)
    pos %= 4096
    q, k, v = split(x, heads, group, d)
    g = torch.Generator().manual_seed(5)
    wq, wk = ((torch.rand(d, generator=g) + 0.5).bfloat16().cuda() for _ in range(2)) if norm \
        else (None, None)
    inv = (10000.0 ** (-torch.arange(0, rotary, 2).double() / rotary)).float().cuda() if rotary \
        else None
    out = torch.empty((tokens, heads * group, d), dtype=torch.bfloat16, device="cuda")
    s = status()
    check_rc(L.arbor_append(kv, 0, q, k, v, slots, pos, out, s, q_norm=wq, k_norm=wk, eps=EPS,
                            inv_freq=inv, interleaved=interleaved))
    assert int(s) == 0
    page, row = slots // kv.page_size, slots % kv.page_size
    for got, src, w in ((out, q, wq), (kv.k[0][page, :, row], k, wk)):
        want = exact(src.reshape(tokens, -1, d), w, pos, inv, interleaved).float().bfloat16()
        wrong = int((got != want).sum())
        assert wrong == 0, f"{wrong} of {want.numel()} elements"
