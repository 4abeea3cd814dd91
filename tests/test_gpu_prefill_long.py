"""A block so long that its slots need more than 23 bits."""
import math

import pytest
import torch

from paper_2605_22106_amd import _lib as L
from tests.test_gpu_prefill import Prefill, queries

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_tokens_beyond_eight_million_are_causal(dtype):
    """The newest 40 tokens of a block of 8,389,648, whose other keys and values are zero: a
    weight of 1 each, far less than those of the keys that a token must not see."""
    old, new, d = 8 * 1024 * 1024 + 1000, 40, 64
    n = old + new
    pages = -(-n // 16)
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    k, v = (torch.zeros((1, pages, 1, 16, d), dtype=dtype, device="cuda") for _ in range(2))
    kv = L.KVState(i32(-1), i32(n), torch.tensor([0, n], device="cuda"),
                   torch.tensor([0, pages], device="cuda"), i32(n),
                   torch.arange(pages, dtype=torch.int32, device="cuda"), k, v,
                   torch.arange(pages * 16, dtype=torch.int32, device="cuda").view(pages, 16),
                   torch.zeros(pages, dtype=torch.int32, device="cuda"), i32(0), 1, 1, 2, d, 16,
                   L.BF16 if dtype is torch.bfloat16 else L.F32, n)
    g = torch.Generator().manual_seed(1)
    q = queries(kv, new)
    # token t's key meets the queries with 4 more than token t - 1's, from 20 on
    q[..., 0] = 8.0
    kk = 0.1 * torch.randn((new, d), generator=g)
    kk[:, 0] = 20.0 + 4.0 * torch.arange(new)
    vv = torch.randn((new, d), generator=g)
    k.view(-1, d)[old:n], v.view(-1, d)[old:n] = kk.to(dtype).cuda(), vv.to(dtype).cuda()
    pf = Prefill(kv, [0], [new])
    out, lse = pf(q)
    assert int(pf.status) == 0
    z = q.double().reshape(new * 2, d) @ k.view(-1, d)[old:n].double().T.contiguous() / math.sqrt(d)
    z = z.view(new, 2, new).masked_fill(
        torch.ones((new, new), dtype=torch.bool, device="cuda").triu(1)[:, None], -math.inf)
    top = z.amax(-1, keepdim=True)
    w = (z - top).exp()
    total = w.sum(-1, keepdim=True) + old * (-top).exp()
    want = (w.view(-1, new) @ v.view(-1, d)[old:n].double()).view(new, 2, d) / total
    # a logit's error, at most (d + 4) 2^-24 of scale * sum |q k|, is its weight's and the LSE's;
    # bf16 rounds each weight and the output, half a step each
    big = (q.double().abs().reshape(new * 2, d) @ k.view(-1, d)[old:n].double().abs().T.contiguous()
           / math.sqrt(d)).view(new, 2, new).amax(-1)
    off = (d + 4) * 2.0 ** -24 * big + 2.0 ** -21 * (1 + lse.double().abs())
    half = 2.0 ** -8 if dtype is torch.bfloat16 else 0.0
    tol = (2 * off + 2 * half)[..., None] * v.abs().max().double()
    assert bool(((out.double() - want).abs() <= tol).all())
    assert bool(((lse.double() - (top + total.log())[..., 0]).abs() <= off).all())
