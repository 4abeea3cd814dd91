"""Host-side refusals of extend, truncate, fork, append and the prefill attention: decided
before anything is enqueued, so no GPU is needed."""
import ctypes

import pytest
import torch

from paper_2605_22106_amd import _lib as L

PTR = 4096          # stands for any aligned device pointer; never read


def geom(**kw):
    d = dict(num_layers=4, num_kv_heads=8, q_per_kv=4, head_dim=128, page_size=16, dtype=L.BF16,
             num_pages=100)
    d.update(kw)
    return L.Geom(**d)


def tree(n_full=PTR, nodes=10, tokens=1000):
    return L.TreeS(nodes, tokens, PTR, n_full, PTR, PTR, PTR, PTR)


def pool(k=PTR):
    return L.PoolS(k, PTR, PTR, PTR, PTR)


def ref(x):
    return None if x is None else ctypes.byref(x)


def call(name, *args):
    return getattr(L.load(), name)(*args)


def extend(g=None, t=None, p=None, n_full=PTR, nodes=PTR, n_seq=2, cu=PTR, n=5, slots=PTR, pos=PTR,
           st=PTR, ws=None, size=0):
    return call("arbor_extend", ref(g or geom()), ref(t or tree()), ref(p or pool()), n_full, nodes,
                n_seq, cu, n, slots, pos, None, st, ws, size, None)


def test_extend():
    for bad in (dict(n_full=8192), dict(nodes=None), dict(cu=None), dict(slots=None), dict(pos=None),
                dict(st=None), dict(n_seq=-1), dict(n_seq=11), dict(n=-1), dict(p=pool(None)),
                dict(t=tree(None), n_full=None)):
        assert extend(**bad) == L.EINVAL, bad
    assert extend(g=geom(head_dim=96)) == L.EUNSUPPORTED
    assert extend(g=geom(page_size=24)) == L.EUNSUPPORTED
    assert extend() == L.EWORKSPACE and extend(ws=PTR, size=64) == L.EWORKSPACE
    assert extend(n=0) == L.OK


def test_truncate_and_fork():
    def run(name, a=PTR, b=PTR, n=2, n_full=PTR, st=PTR, more=()):
        return call(name, ref(geom()), ref(tree()), ref(pool()), n_full, a, b, n, *more, st, None, 0,
                    None)
    for name, more in (("arbor_truncate", ()), ("arbor_fork", (None, None))):
        for bad in (dict(a=None), dict(b=None), dict(n=-1), dict(n=11), dict(n_full=8), dict(st=None)):
            assert run(name, more=more, **bad) == L.EINVAL, (name, bad)
        assert run(name, more=more) == L.EWORKSPACE
        assert run(name, more=more, n=0, a=None, b=None) == L.OK


def append(layer=0, n=3, g=None, st=PTR, **kw):
    d = dict(q=PTR, k=PTR, v=PTR, q_stride=6144, k_stride=6144, v_stride=6144, q_norm=None,
             k_norm=None, inv_freq=PTR, slots=PTR, positions=PTR, tokens=None, record_k=None,
             record_v=None, q_out=2 * PTR, eps=1e-6, rotary_dim=128, interleaved=0)
    d.update(kw)
    return call("arbor_append", ref(g or geom()), ref(tree()), ref(pool()), layer,
                ref(L.Append(**d)), n, st, None)


def test_append():
    for bad in (dict(layer=-1), dict(layer=4), dict(n=-1), dict(st=None), dict(q=None), dict(k=None),
                dict(v=None), dict(q_out=None), dict(slots=None), dict(positions=None),
                dict(q_stride=4088), dict(k_stride=1016), dict(v_stride=0), dict(interleaved=2),
                dict(rotary_dim=-8), dict(inv_freq=None), dict(eps=-1.0), dict(eps=float("nan")),
                dict(record_k=PTR), dict(record_v=PTR, tokens=PTR),
                dict(record_k=PTR, record_v=PTR), dict(q_out=PTR)):
        assert append(**bad) == L.EINVAL, bad
    for bad in (dict(rotary_dim=12), dict(rotary_dim=136), dict(q=PTR + 8), dict(q_out=PTR + 2),
                dict(k_stride=6145), dict(q_norm=PTR + 4), dict(g=geom(head_dim=80))):
        assert append(**bad) == L.EUNSUPPORTED, bad
    assert append(n=0) == L.OK


def test_prefill():
    def plan(g=None, nodes=PTR, n_seq=2, cu=PTR, n=5, buf=PTR, size=0, st=PTR):
        return call("arbor_prefill_plan", ref(g or geom()), ref(tree()), nodes, n_seq, cu, n, buf,
                    size, st, None)

    def attn(g=None, buf=PTR, size=1 << 30, n_seq=2, n=5, layer=0, q=PTR, out=PTR, st=PTR, ws=PTR,
             ws_size=0):
        return call("arbor_tree_prefill_attn", ref(g or geom()), ref(tree()), ref(pool()), buf, size,
                    n_seq, n, layer, q, out, None, 0.0, st, ws, ws_size, None)

    for bad in (dict(nodes=None), dict(cu=None), dict(n_seq=-1), dict(n=-1), dict(buf=None),
                dict(buf=PTR + 16), dict(st=None)):
        assert plan(**bad) == L.EINVAL, bad
    for bad in (dict(buf=None), dict(buf=PTR + 16), dict(layer=-1), dict(layer=4), dict(q=None),
                dict(out=None), dict(st=None), dict(ws=None), dict(n=-1)):
        assert attn(**bad) == L.EINVAL, bad
    for f in (plan, attn):
        assert f(g=geom(q_per_kv=129)) == L.EUNSUPPORTED
        assert f(g=geom(head_dim=256)) == L.EUNSUPPORTED
    assert attn(q=PTR + 8) == L.EUNSUPPORTED
    assert plan() == L.EWORKSPACE and attn(size=100) == L.EWORKSPACE and attn() == L.EWORKSPACE
    assert plan(n=0) == L.OK and attn(n=0, q=None, out=None, ws=None) == L.OK
    assert plan(n_seq=0, nodes=None, cu=None) == L.OK


@pytest.mark.parametrize("group", [1, 3, 8, 128])
def test_sizes_grow_with_the_call(group):
    lib = L.load()
    g = geom(q_per_kv=group)
    sizes = [lib.arbor_prefill_plan_size(ref(g), s, t) for s, t in ((1, 1), (1, 100), (50, 100),
                                                                   (50, 9000), (4000, 9000))]
    assert sizes == sorted(sizes) and sizes[0] > 0 and len(set(sizes)) == 5
    w = [lib.arbor_prefill_workspace_size(ref(g), s, t) for s, t in ((1, 0), (1, 1), (1, 100),
                                                                    (9, 9000))]
    assert w == sorted(w) and w[0] > 0
    assert lib.arbor_prefill_plan_size(ref(geom(q_per_kv=129)), 1, 1) == 0
    assert lib.arbor_prefill_workspace_size(ref(g), -1, 1) == 0


def test_tiles_never_exceed_their_bound():
    """The cut of packed tokens into tiles, followed on the CPU over many batches: no more
    tiles than the plan has room for (two neighbours hold more than one tile may, or a run of
    64 blocks ended), which the plan's size is made for."""
    import random
    r = random.Random(1)
    for _ in range(3000):
        tq = r.choice([1, 2, 16, 25, 32, 42, 128])
        m = [r.choice([0, 0, 1, r.randint(0, 5), r.randint(0, 3 * tq)])
             for _ in range(r.choice([1, 5, 70, 300]))]
        tiles, e, off = 0, 0, 0
        while e < len(m):
            first = m[e] - off
            if first == 0:
                e, off = e + 1, 0
            elif first > tq:
                tiles, off = tiles + first // tq, off + first // tq * tq
            else:
                total, n = 0, 0
                while e + n < len(m) and n < 64 and total + m[e + n] - (off if n == 0 else 0) <= tq:
                    total += m[e + n] - (off if n == 0 else 0)
                    n += 1
                tiles, e, off = tiles + 1, e + n, 0
        assert tiles <= min(sum(m), 2 * (sum(m) // tq) + len(m) // 64 + 2)


def test_the_binding_checks_shapes_types_and_places():
    cpu = torch.zeros(3, dtype=torch.int32)
    for f in (lambda: L._is(cpu, "x", torch.int64, 3), lambda: L._is(cpu, "x", torch.int32, 4),
              lambda: L._is(cpu, "x", torch.int32, 3), lambda: L._packed(cpu, cpu),
              lambda: L._rows(torch.zeros(2, 8), "q", torch.bfloat16, 2, 8),
              lambda: L._rows(torch.zeros(2, 8), "q", torch.float32, 3, 8),
              lambda: L._rows(torch.zeros(2, 8), "q", torch.float32, 2, 9),
              lambda: L._rows(torch.zeros(2, 8), "q", torch.float32, 2, 8)):
        with pytest.raises(ValueError):
            f()
