"""A tree without blocks: its arrays may be null, so the prefill calls refuse it on the host."""
from paper_2605_22106_amd import _lib as L
from tests.test_grow_refusals import PTR, call, geom, pool, ref


def test_no_blocks():
    none = L.TreeS(0, 0, None, None, None, None, None, None)

    def plan(n_seq, n):
        return call("arbor_prefill_plan", ref(geom()), ref(none), PTR, n_seq, PTR, n, PTR, 1 << 30,
                    PTR, None)

    def attn(n_seq, n):
        return call("arbor_tree_prefill_attn", ref(geom()), ref(none), ref(pool()), PTR, 1 << 30,
                    n_seq, n, 0, PTR, PTR, None, 0.0, PTR, PTR, 1 << 30, None)
    for f in (plan, attn):
        assert f(1, 4) == L.EINVAL
        assert f(0, 4) == L.OK and f(1, 0) == L.OK
