"""States with room to grow for the tests of extend, truncate, fork, append and the prefill
attention: blocks with spare capacity, a part of their tokens evicted, shuffled pages, and
NaN in every row of the pool that holds no token."""
from __future__ import annotations

import random

import numpy as np
import torch


def grow_state(parent, n, c=None, spare=40, *, layers=2, kv_heads=2, q_per_kv=2, head_dim=64,
               dtype="f32", page_size=16, seed=0, extra_pages=3, k_scale=1.0):
    """c[i] of block i's n[i] tokens resident at random positions, the newest ones of a block
    among them; capacity n[i] + spare (a number, or one for each block)."""
    g, r = torch.Generator().manual_seed(seed), random.Random(seed)
    V, P = len(parent), page_size
    c = list(n) if c is None else list(c)
    cap = [x + (spare if isinstance(spare, int) else spare[i]) for i, x in enumerate(n)]
    off = lambda v: torch.tensor([0] + list(np.cumsum(v)), dtype=torch.int64)  # noqa: E731
    tok_off, page_off = off(cap), off([-(-x // P) for x in cap])
    pages = int(page_off[-1]) + extra_pages
    free = list(range(pages))
    r.shuffle(free)
    page_table = torch.full((int(page_off[-1]),), -1, dtype=torch.int32)
    slot_pos = torch.full((pages, P), -1, dtype=torch.int32)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    shape = (layers, pages, kv_heads, P, head_dim)
    k = (torch.randn(shape, generator=g) * k_scale).to(dt)
    v = torch.randn(shape, generator=g).to(dt)
    used = torch.zeros((pages, P), dtype=torch.bool)
    for i in range(V):
        # the newest half of what stays is the block's end, the rest lies anywhere before
        tail = c[i] - c[i] // 2
        pos = sorted(r.sample(range(n[i] - tail), c[i] - tail)) + list(range(n[i] - tail, n[i]))
        for q in range(-(-c[i] // P)):
            page_table[int(page_off[i]) + q] = free.pop()
        for s, p in enumerate(pos):
            page = int(page_table[int(page_off[i]) + s // P])
            slot_pos[page, s % P] = p
            used[page, s % P] = True
    for x in (k, v):
        x.permute(1, 3, 0, 2, 4)[~used] = float("nan")
    free_stack = torch.full((pages,), -1, dtype=torch.int32)
    free_stack[:len(free)] = torch.tensor(free, dtype=torch.int32)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32)  # noqa: E731
    return dict(parent=i32(parent), n_full=i32(n), tok_off=tok_off, page_off=page_off,
                n_kept=i32(c), page_table=page_table, slot_pos=slot_pos, free_stack=free_stack,
                free_top=i32([len(free)]), k=k, v=v, num_pages=pages, page_size=P, layers=layers,
                kv_heads=kv_heads, q_per_kv=q_per_kv, head_dim=head_dim, dtype=dtype,
                num_tokens=int(tok_off[-1]))


BOOKS = ("n_full", "n_kept", "page_table", "slot_pos", "free_top")


def assert_same_books(a: dict, b: dict):
    """Equal bookkeeping of two oracle-form states, the live part of the free stack too."""
    for key in BOOKS:
        assert np.array_equal(np.asarray(a[key]).reshape(-1), np.asarray(b[key]).reshape(-1)), key
    top = int(a["free_top"])
    assert np.array_equal(a["free_stack"][:top], b["free_stack"][:top])


def ragged(seed, count, lo, hi):
    r = random.Random(seed)
    return [r.randint(lo, hi) for _ in range(count)]


def cu_of(m):
    return [0] + [int(x) for x in np.cumsum(m)]


def reference(st, parent, nodes, m, layer, q, G, scale=None):
    """The definition in 64 bits for sizes beyond the oracle's loops: sequence by sequence,
    torch fp64 on q's device.  out, lse, sum p |v|, and a bound on scale * sum |q_x k_x|."""
    dev, P = q.device, st["page_size"]
    T, Hq, D = q.shape
    H = Hq // G
    scale = D ** -0.5 if scale is None else scale
    out = torch.zeros((T, Hq, D), dtype=torch.float64, device=dev)
    mass = torch.zeros_like(out)
    lse = torch.zeros((T, Hq), dtype=torch.float64, device=dev)
    big = torch.zeros_like(lse)
    table, off, c = st["page_table"].long(), st["page_off"].tolist(), st["n_kept"].tolist()
    at = 0
    for i, mm in zip(nodes, m):
        if mm == 0:
            continue
        up, x = [], i
        while x >= 0:
            up.append(x)
            x = parent[x]
        ids = torch.cat([table[off[x] + torch.arange(c[x], device=dev) // P] * P +
                         torch.arange(c[x], device=dev) % P for x in up[::-1]])
        k, v = (y[layer][ids // P, :, ids % P].double() for y in (st["k"], st["v"]))
        late = torch.arange(ids.numel(), device=dev)[None] > (
            ids.numel() - mm + torch.arange(mm, device=dev))[:, None]
        for h in range(H):
            qq = q[at:at + mm, h * G:(h + 1) * G].double().reshape(mm * G, D)
            z = (qq @ k[:, h].T.contiguous() * scale).view(mm, G, -1)
            z = z.masked_fill(late[:, None], -float("inf"))
            s = torch.logsumexp(z, -1)
            p = (z - s[..., None]).exp().view(mm * G, -1)
            sl = (slice(at, at + mm), slice(h * G, (h + 1) * G))
            lse[sl] = s
            out[sl] = (p @ v[:, h].contiguous()).view(mm, G, D)
            mass[sl] = (p @ v[:, h].abs().contiguous()).view(mm, G, D)
            big[sl] = scale * (qq.abs() @ k[:, h].abs().T.contiguous()).amax(-1).view(mm, G)
        at += mm
    return out, lse, mass, big


def attention_bounds(dtype, D, out, lse, mass, big):
    """How far fp32 arithmetic may be off, element by element.  A logit is a sum of D
    products: off by at most D 2^-24 of scale * sum |q k| (big), and its scaling and
    exponential by 4 2^-24 of |logit| <= big and 2^-22; the same again for the denominator.
    bf16 rounds each weight and the output, half a step (2^-8) each."""
    e = (2 * (D + 4) * 2.0 ** -24) * big + 2.0 ** -20
    half = 2.0 ** -8 if dtype == "bf16" else 0.0
    tol = mass * (e[..., None] + half) + abs(out) * (half + 2.0 ** -22)
    return tol, (D + 4) * 2.0 ** -24 * big + 2.0 ** -21 * (1 + abs(lse))
