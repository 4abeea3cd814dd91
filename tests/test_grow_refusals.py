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


def test_tiles_by_links_keep_the_bound_and_hold_every_token():
    """The plan's own cut: a block's whole tiles, then its rest with the blocks that fit."""
    import bisect
    import random
    r = random.Random(2)
    for _ in range(3000):
        tq = r.choice([1, 2, 16, 25, 32, 42, 128])
        m = [r.choice([0, 0, 1, tq, r.randint(0, 5), r.randint(0, 3 * tq)])
             for _ in range(r.choice([1, 5, 70, 300]))]
        cu = [0]
        for x in m:
            cu.append(cu[-1] + x)
        tiles, e = [], 0
        while e < len(m):
            full = m[e] // tq
            tiles += [(cu[e] + x * tq, tq, 1) for x in range(full)]
            t, nxt = cu[e] + full * tq, e + 1
            if t < cu[e + 1]:
                hi = min(len(m), e + 64)
                nxt = bisect.bisect_right(cu, t + tq, e + 1, hi + 1) - 1
                tiles.append((t, cu[nxt] - t, nxt - e))
            e = nxt
        at = 0
        for t, n, blocks in tiles:
            assert t == at and 0 < n <= tq and 1 <= blocks <= 64
            at += n
        assert at == cu[-1]
        assert len(tiles) <= min(sum(m), 2 * (sum(m) // tq) + len(m) // 64 + 2)


def test_the_binding_checks_shapes_types_and_places():
    cpu = torch.zeros(3, dtype=torch.int32)
    rows = torch.zeros(2, 8)
    for f in (lambda: L._is(cpu, "x", torch.int64, (3,), -1),
              lambda: L._is(cpu, "x", torch.int32, (4,), -1),
              lambda: L._is(cpu, "x", torch.int32, (3,), -1),
              lambda: L._is(cpu, "x", torch.int32, (3,), 0),
              lambda: L._packed(cpu, cpu, 0), lambda: L._bytes(cpu, "x", 0),
              lambda: L._rows(rows, "q", torch.bfloat16, 2, 8, -1),
              lambda: L._rows(rows, "q", torch.float32, 3, 8, -1),
              lambda: L._rows(rows, "q", torch.float32, 2, 9, -1),
              lambda: L._rows(rows, "q", torch.float32, 2, 8, 0),
              lambda: L._record(rows, "r", torch.float32, (2, 9)),
              lambda: L._record(rows, "r", torch.float32, (2, 8))):
        with pytest.raises(ValueError):
            f()


def test_descriptors_follow_the_state(monkeypatch):
    """What a KVState's tensors are is read again when a field is set or a tensor is moved."""
    monkeypatch.setattr(L, "_dev", lambda t, name: None if t is None else t.data_ptr())
    monkeypatch.setattr(torch.cuda, "current_device", lambda: -1)     # CPU tensors here
    z = lambda n: torch.zeros(n, dtype=torch.int32)  # noqa: E731
    kv = L.KVState(z(4), z(4), z(5), z(5), z(4), z(9), torch.zeros(1, 9, 2, 16, 64),
                   torch.zeros(1, 9, 2, 16, 64), z(9), z(9), z(1), 1, 2, 4, 64, 16, L.F32, 100)
    tree = lambda: L._descriptors(kv)[2]._obj  # noqa: E731
    geom = lambda: L._descriptors(kv)[1]._obj  # noqa: E731
    assert L._descriptors(kv) == L._descriptors(kv) and tree() is tree()
    assert tree().num_nodes == 4 and L._descriptors(kv)[4] == kv.n_full.data_ptr()
    buf = z(20)
    kv.parent = buf[:4]
    assert tree().parent == buf.data_ptr() and tree().num_nodes == 4
    kv.parent = buf[:7]                                  # the same memory, more blocks
    assert tree().num_nodes == 7
    kv.q_per_kv, kv.num_tokens = 8, 300
    assert geom().q_per_kv == 8 and tree().num_tokens == 300
    kv.n_kept.data = z(64)
    assert tree().n_kept == kv.n_kept.data_ptr()
    copy = kv.clone()
    assert L._descriptors(copy)[2]._obj.parent == copy.parent.data_ptr() != tree().parent
    kv.k.resize_(1, 5, 2, 16, 64)
    assert geom().num_pages == 5
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    with pytest.raises(ValueError):
        L._descriptors(kv)


def test_append_struct_layout(tmp_path):
    """The binding's arbor_append_t has the C compiler's size and offsets."""
    import os
    import subprocess
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    names = [f[0] for f in L.Append._fields_]
    src = tmp_path / "layout.c"
    src.write_text("#include <stdio.h>\n#include <stddef.h>\n#include \"arbor.h\"\nint main(void) {"
                   'printf("%zu\\n", sizeof(arbor_append_t));' +
                   "".join(f'printf("%zu\\n", offsetof(arbor_append_t, {n}));' for n in names) +
                   "return 0; }\n")
    exe = tmp_path / "layout"
    subprocess.run(["gcc", "-D__HIP_PLATFORM_AMD__", "-I", os.path.join(root, "include"), "-I",
                    "/opt/rocm/include", str(src), "-o", str(exe)], check=True)
    got = [int(x) for x in subprocess.run([str(exe)], check=True, capture_output=True,
                                          text=True).stdout.split()]
    assert got == [ctypes.sizeof(L.Append)] + [getattr(L.Append, n).offset for n in names]
