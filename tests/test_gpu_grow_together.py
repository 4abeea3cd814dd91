"""The operators that grow a tree as a program runs them: thoughts that grow, are scored and
thinned out, restored, decoded, dropped and forked; the same step captured, on two streams,
and with two plans; and the sizes at which the plan and the append change their launches."""
import numpy as np
import pytest
import torch

from oracle import arbor_oracle as O
from paper_2605_22106_amd import _lib as L
from tests.gpu_helpers import assert_same_pool, check_rc, gpu_to_oracle, status, to_gpu, workspace
from tests.grow_helpers import assert_same_books, cu_of, grow_state, ragged, reference
from tests.helpers import np_float, oracle_state
from tests.test_gpu_grow import append_case, split
from tests.test_gpu_prefill import Prefill, check, queries

pytestmark = pytest.mark.gpu

PARAMS = dict(alpha_max=float("inf"), gamma=2.0, lambda_d=0.1, lambda_delta=0.5, eta=0.8,
              r_min=0.05, k_min=2, l_tail=4, theta=(1.0, 1.0, 1.0), select_mode=0,
              score_self_window=0)
EPS = 1e-5


def i32(x):
    return torch.tensor([int(y) for y in x], dtype=torch.int32, device="cuda")


class Step:
    """truncate, extend, plan, then append and attention of each layer, on buffers of its own."""

    def __init__(self, kv, nodes, m, keep=None, record=None, seed=0, pad=0):
        g = torch.Generator().manual_seed(seed)
        self.kv, self.nodes, self.m, self.cu = kv, i32(nodes), m, i32(cu_of(m))
        self.T = T = sum(m) + pad
        self.keep = None if keep is None else i32(keep)
        Hq, H, d, dt = kv.kv_heads * kv.q_per_kv, kv.kv_heads, kv.head_dim, kv.k.dtype
        self.x = [torch.randn((T, (Hq + 2 * H) * d), generator=g).to(dt).cuda()
                  for _ in range(kv.layers)]
        self.wq, self.wk = ((torch.rand(d, generator=g) + 0.5).to(dt).cuda() for _ in range(2))
        self.inv = (10000.0 ** (-torch.arange(0, d, 2).double() / d)).float().cuda()
        self.record, self.status = record, status()
        self.slots, self.tokens = (torch.empty(T, dtype=torch.int64, device="cuda")
                                   for _ in range(2))
        self.pos = torch.empty(T, dtype=torch.int32, device="cuda")
        self.q = torch.zeros((kv.layers, T, Hq, d), dtype=dt, device="cuda")
        self.out, self.lse = torch.zeros_like(self.q), torch.zeros((kv.layers, T, Hq), device="cuda")
        self.plan = torch.empty(L.arbor_prefill_plan_size(kv, len(nodes), T), dtype=torch.uint8,
                                device="cuda")
        self.ws = torch.empty(L.arbor_prefill_workspace_size(kv, len(nodes), T),
                              dtype=torch.uint8, device="cuda")
        self.ws2 = workspace(kv)

    def split(self, layer):
        return split(self.x[layer], self.kv.kv_heads, self.kv.q_per_kv, self.kv.head_dim)

    def __call__(self):
        kv, s = self.kv, self.status
        if self.keep is not None:
            check_rc(L.arbor_truncate(kv, self.nodes, self.keep, s, self.ws2))
        check_rc(L.arbor_extend(kv, self.nodes, self.cu, self.slots, self.pos, self.tokens, s,
                                self.ws2))
        check_rc(L.arbor_prefill_plan(kv, self.nodes, self.cu, self.T, self.plan, s))
        rk, rv = self.record or (None, None)
        for layer in range(kv.layers):
            q, k, v = self.split(layer)
            check_rc(L.arbor_append(kv, layer, q, k, v, self.slots, self.pos, self.q[layer], s,
                                    q_norm=self.wq, k_norm=self.wk, eps=EPS, inv_freq=self.inv,
                                    tokens=self.tokens if rk is not None else None, record_k=rk,
                                    record_v=rv))
            check_rc(L.arbor_tree_prefill_attn(kv, self.plan, self.nodes.numel(), layer,
                                               self.q[layer], self.out[layer], self.lse[layer], 0.0,
                                               s, self.ws))

    def results(self):
        torch.cuda.synchronize()
        kv = self.kv
        return [t.clone() for t in (self.slots, self.pos, self.tokens, self.q, self.out, self.lse,
                                    self.status, kv.n_full, kv.n_kept, kv.page_table, kv.slot_pos,
                                    kv.free_stack, kv.free_top, kv.k.view(torch.int16),
                                    kv.v.view(torch.int16))]


def same(a, b):
    return all(torch.equal(x, y) for x, y in zip(a, b))


PARENT = [-1, 0, 0, 1, 1, 2, 3, 5, 2]        # 6, 7 and 8 are empty at first


def small_state(seed=0, dtype="bf16", d=128, G=4):
    n = [90, 40, 33, 50, 21, 64, 0, 0, 0]
    c = [60, 25, 33, 50, 20, 40, 0, 0, 0]
    return grow_state(PARENT, n, c, spare=150, kv_heads=2, q_per_kv=G, head_dim=d, dtype=dtype,
                      seed=seed, extra_pages=60)


@pytest.mark.parametrize("dtype,d,G", [("bf16", 128, 4), ("f32", 64, 3)])
def test_a_search_that_grows_and_thins_out(dtype, d, G):
    """Two rounds: blocks grow, what they have is thinned out, restored, decoded; one is
    dropped and becomes a copy.  All bookkeeping as the oracle's, all values within bounds."""
    st = small_state(dtype=dtype, d=d, G=G)
    kv, ost, N = to_gpu(st), oracle_state(st), st["num_tokens"]
    Hq, V, Ln = kv.kv_heads * G, kv.num_nodes, kv.layers
    gen = torch.Generator().manual_seed(3)
    rec = [(torch.randn((N, Ln, kv.kv_heads, d), generator=gen)).to(kv.k.dtype).pin_memory()
           for _ in range(2)]
    A = torch.rand(N, generator=gen).cuda()
    rows_seen = torch.arange(V, device="cuda", dtype=torch.int64)
    rng, ws = np.random.default_rng(5), workspace(kv, max_leaves=4, max_layers=Ln)
    for rnd, (nodes, m) in enumerate([([3, 4, 6, 7, 8], [5, 17, 1, 40, 16]),
                                      ([4, 6, 7, 8], [2, 33, 1, 9])]):
        step = Step(kv, nodes, m, record=rec, seed=rnd, pad=2)
        step()
        torch.cuda.synchronize()
        assert int(step.status) == 0
        ost, slots, pos, tokens, so = O.extend(ost, nodes, cu_of(m), step.T)
        assert so == O.OK and np.array_equal(step.slots.cpu().numpy(), slots)
        assert np.array_equal(step.tokens.cpu().numpy(), tokens)
        live, T = slots >= 0, sum(m)
        assert np.array_equal(step.pos.cpu().numpy()[live], pos[live])
        assert_same_books(gpu_to_oracle(kv), ost)
        page, row = slots[live] // kv.page_size, slots[live] % kv.page_size
        g = gpu_to_oracle(kv)
        for layer in range(Ln):
            q, k, v = (np_float(t)[live].reshape(T, -1, d) for t in step.split(layer))
            for got, x, w in ((np_float(step.q[layer])[live], q, step.wq),
                              (g["k"][layer][page, :, row], k, step.wk)):
                want, normed = O.norm_rotate(x, np_float(w), EPS, pos[live],
                                             step.inv.cpu().numpy(), False)
                # as in the test of the append alone, for positions below 1,000
                pair = 2 * np.abs(normed).max(-1, keepdims=True)
                tol = pair * ((d / 2 + 6) * 2.0 ** -24 + 2.0 ** -22 + 2.0 ** -41)
                tol = tol + np.abs(want) * (2.0 ** -8 if dtype == "bf16" else 2.0 ** -24)
                assert np.all(np.abs(got - want) <= tol)
            assert np.array_equal(g["v"][layer][page, :, row], v)
            for r, x in zip(rec, (g["k"], g["v"])):
                assert np.array_equal(np_float(r)[tokens[live], layer], x[layer][page, :, row])
        ost["k"], ost["v"] = g["k"], g["v"]        # (the same bits from here on)
        for layer in range(Ln):
            want = O.prefill_attn(ost, nodes, cu_of(m), layer, np_float(step.q[layer])[:T], G)
            check((step.out[layer][:T], step.lse[layer][:T]), want, dtype, d)
        # an event thins the tree out, and one leaf's path is restored from the record
        s = rng.random(V).astype(np.float32)
        budget = int(0.6 * ost["n_kept"].sum())
        k_o, _, _, so = O.allocate(np.array(PARENT), ost["n_full"], ost["n_kept"], np.array([7]), budget, s,
                                   PARAMS)
        k, onp = torch.empty(V, dtype=torch.int32, device="cuda"), torch.empty(
            V, dtype=torch.uint8, device="cuda")
        check_rc(L.arbor_allocate(kv, i32([7]), budget, torch.tensor(s, device="cuda"), PARAMS, k,
                                  torch.empty_like(k), onp, step.status, ws))
        assert int(step.status) == so and np.array_equal(k.cpu().numpy(), k_o)
        sel_o, _ = O.select(ost, A.cpu().numpy(), k_o, PARAMS["l_tail"])
        ost = O.compact(ost, k_o, sel_o)
        step.status.zero_()
        check_rc(L.arbor_select_compact(kv, A, k, PARAMS, torch.empty(N, dtype=torch.int32,
                                                                      device="cuda"),
                                        step.status, ws))
        assert_same_pool(gpu_to_oracle(kv), ost)
        path = np.zeros(V, dtype=np.uint8)
        path[O.chain(np.array(PARENT), 6)] = 1
        ost, so = O.rehydrate(ost, path, np_float(rec[0]), np_float(rec[1]))
        check_rc(L.arbor_rehydrate(kv, torch.tensor(path, device="cuda"), rec[0], rec[1],
                                   step.status, ws))
        assert so == O.OK and int(step.status) == 0
        assert_same_pool(gpu_to_oracle(kv), ost)
        # single tokens: the tree's own decode over what has grown
        leaves, qd = [6, 7, 4], torch.randn((3, Ln, Hq, d), generator=gen).to(kv.k.dtype)
        out, lse = (torch.empty(x, device="cuda") for x in ((3, Ln, Hq, d), (3, Ln, Hq)))
        check_rc(L.arbor_tree_decode_attn(kv, i32(leaves), 0, Ln, qd.cuda(), out, lse, 0.0,
                                          step.status, ws))
        o_o, l_o = O.tree_decode_attn(ost, leaves, 0, Ln, np_float(qd), G)
        assert np.max(np.abs(out.cpu().numpy() - o_o)) <= 2e-3
        assert np.max(np.abs(lse.cpu().numpy() - l_o)) <= 2e-3
        # a block that lost is emptied and becomes a copy of one that won
        check_rc(L.arbor_truncate(kv, i32([8]), i32([0]), step.status, ws))
        check_rc(L.arbor_fork(kv, i32([6]), i32([8]), step.status, ws, A=A, rows_seen=rows_seen))
        ost, so = O.truncate(ost, [8], [0])
        assert so == O.OK
        ost, a_o, r_o, so = O.fork(ost, [6], [8], None, None)
        assert so == O.OK and int(step.status) == 0
        assert_same_pool(gpu_to_oracle(kv), ost)
        assert_same_books(gpu_to_oracle(kv), ost)
        n6, t6, t8 = int(ost["n_full"][6]), int(kv.tok_off[6]), int(kv.tok_off[8])
        assert torch.equal(A[t8:t8 + n6], A[t6:t6 + n6]) and int(rows_seen[8]) == 6
        for r in rec:                              # (the program copies the record's rows)
            r[t8:t8 + n6] = r[t6:t6 + n6].clone()


def drafts(seed=0):
    """A step that takes its own drafts back first, so that each run does the same."""
    kv = to_gpu(small_state(seed))
    step = Step(kv, [3, 4, 6, 7], [9, 1, 30, 64], seed=seed)
    step()
    keep = kv.n_full[step.nodes.long()].cpu() - torch.tensor(step.m)
    step.keep = i32(keep)
    return step


def test_a_captured_step_replayed():
    step = drafts()
    step()
    eager = step.results()
    assert int(step.status) == 0
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(4):
        for t in (step.out, step.lse, step.q, step.slots, step.ws, step.plan, step.ws2):
            t.fill_(3)
        torch.randn(1 << 20, device="cuda").sum().item()
        graph.replay()
        assert same(step.results(), eager)


def test_two_graphs_with_buffers_of_their_own():
    a, b = drafts(0), drafts(1)
    a(), b()
    want = a.results(), b.results()
    graphs = []
    for s in (a, b):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            s()
        graphs.append(g)
    for _ in range(3):
        for g in graphs + graphs[::-1]:
            g.replay()
    assert same(a.results(), want[0]) and same(b.results(), want[1])


def test_on_another_stream_and_runs_alike():
    step = drafts()
    step()
    want = step.results()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(3):
            step()
    torch.cuda.current_stream().wait_stream(side)
    assert same(step.results(), want)


def test_one_plan_read_on_two_streams():
    """Two layers' attention at once: one plan, a workspace each."""
    parent, had, m = [-1] + [0] * 6, [4000] + [0] * 6, ragged(5, 6, 1, 60)
    n = [4000] + m
    kv = to_gpu(grow_state(parent, n, kv_heads=2, q_per_kv=4, head_dim=128, dtype="bf16"))
    pf, other = Prefill(kv, list(range(1, 7)), m), Prefill(kv, list(range(1, 7)), m)
    other.plan = pf.plan
    q = queries(kv, sum(m))
    want = [pf(q, layer) for layer in (0, 1)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    outs = [torch.empty_like(q) for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(4):
        with torch.cuda.stream(side):
            got1 = other(q, 1, out=outs[1])
        got0 = pf(q, 0, out=outs[0])
    torch.cuda.synchronize()
    for got, w in zip((got0, got1), want):
        assert torch.equal(got[0], w[0]) and torch.equal(got[1], w[1])


def test_out_may_be_q():
    kv = to_gpu(grow_state([-1, 0], [3000, 70], kv_heads=2, q_per_kv=4, head_dim=128,
                           dtype="bf16", layers=1))
    pf, q = Prefill(kv, [0, 1], [200, 70]), None
    q = queries(kv, 270)
    want = pf(q)[0]
    assert torch.equal(pf(q, out=q)[0], want)


PLANS = [  # parent, tokens that were there, nodes, new tokens, group, dtype: what the plan needs
    ([-1], [0], [0], [2500], 8, "bf16"),                              # many tiles, one block
    ([-1] + [0] * 4200, [20] + [0] * 4200, list(range(1, 4201)),      # more blocks than LDS holds
     [x % 2 for x in range(4200)], 1, "bf16"),
    ([-1] + [0] * 4999, [33] + [1] * 4999, [7, 4998], [3, 40], 4, "f32"),        # a wide tree
    ([-1] + [0] * 63, [50] + [0] * 63, list(range(1, 64)), [1] * 63, 128, "bf16"),   # 63 tiles
    ([-1] + [0] * 64, [50] + [0] * 64, list(range(1, 65)), ragged(2, 64, 0, 30), 16, "f32"),
    (list(range(-1, 63)), [3] * 64, list(range(64)), [1] * 64, 1, "bf16"),   # each below the last
]


@pytest.mark.parametrize("case", PLANS, ids=lambda c: f"{len(c[0])}-{len(c[2])}-{sum(c[3])}-{c[4]}")
def test_plans_of_each_kind(case):
    parent, had, nodes, m, G, dtype = case
    n = list(had)
    for i, x in zip(nodes, m):
        n[i] += x
    st = grow_state(parent, n, spare=0, kv_heads=1, q_per_kv=G, head_dim=64, dtype=dtype, seed=4,
                    layers=1)
    kv = to_gpu(st)
    pf, q = Prefill(kv, nodes, m), queries(kv, sum(m))
    got = pf(q)
    assert int(pf.status) == 0
    dev = {k: v.cuda() if torch.is_tensor(v) else v for k, v in st.items()}
    check(got, reference(dev, parent, nodes, m, 0, q, G), dtype, 64)


def test_a_plan_of_another_tree():
    """As many blocks, but a page table of another length: refused before anything is read."""
    a, b = (to_gpu(grow_state([-1, 0], n, spare=0, kv_heads=1, layers=1))
            for n in ([400, 30], [40, 30]))
    pf, q = Prefill(a, [1], [30]), queries(b, 30)
    pf.kv, pf.status = b, status()
    out, _ = pf(q)
    assert int(pf.status) == L.EINVAL and bool((out == 7.0).all())


@pytest.mark.parametrize("had,T,G", [(0, 1100, 8), (777, 1024, 8), (300, 67, 128), (0, 8200, 1)])
def test_one_block_of_many_tiles(had, T, G):
    """Twice as many tiles as the chip holds for a KV head: a call without parts."""
    heads = 16 if G < 128 else 64
    st = grow_state([-1, 0], [had, T], spare=0, kv_heads=heads, q_per_kv=G, head_dim=64,
                    dtype="bf16", seed=6, layers=1)
    kv = to_gpu(st)
    pf, q = Prefill(kv, [1], [T]), queries(kv, T)
    pf.ws.fill_(255)                               # (NaN, if parts were read)
    got = pf(q)
    assert int(pf.status) == 0
    dev = {k: v.cuda() if torch.is_tensor(v) else v for k, v in st.items()}
    if T * G < 10000:
        check(got, reference(dev, [-1, 0], [1], [T], 0, q, G), "bf16", 64)
        return
    # the last tokens alone are the reference's; more of them would not fit its matrices
    last = 40
    want = reference(dev, [-1, 0], [1], [last], 0, q[T - last:], G)
    check(tuple(x[T - last:] for x in got), want, "bf16", 64)


@pytest.mark.parametrize("T", [8191, 8192, 8700])
@pytest.mark.parametrize("inter", [False, True])
def test_append_of_many_tokens(T, inter):
    """The same rows whether a wave takes a token or four do: those of short calls."""
    kv, x, slots, pos = append_case("bf16", 64, 2, 3, T, 20)
    q, k, v = split(x, 2, 3, 64)
    kw = dict(q_norm=torch.rand(64, device="cuda").bfloat16(), eps=EPS,
              inv_freq=torch.rand(32, device="cuda"), interleaved=inter)
    out = torch.full((T + 20, 6, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    short, part = kv.clone(), out.clone()
    check_rc(L.arbor_append(kv, 1, q, k, v, slots, pos, out, status(), **kw))
    for a in range(0, T + 20, 1000):
        b = slice(a, a + 1000)
        check_rc(L.arbor_append(short, 1, q[b], k[b], v[b], slots[b], pos[b], part[b], status(),
                                **kw))
    assert torch.equal(out, part)
    for y, z in ((kv.k, short.k), (kv.v, short.v)):
        assert torch.equal(y.view(torch.int16), z.view(torch.int16))


def test_timing_of_the_attention():
    step = drafts()
    a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    a.record(), b.record()
    torch.cuda.synchronize()
    want = step.results()
    check_rc(L.arbor_tree_prefill_attn(step.kv, step.plan, step.nodes.numel(), 1, step.q[1],
                                       step.out[1], step.lse[1], 0.0, step.status, step.ws,
                                       timing=L.timing(L.KERNEL_PREFILL_ATTN, a, b)))
    assert same(step.results(), want)
    assert 0.0 < a.elapsed_time(b) < 1000.0


def test_blocks_to_come_are_scored():
    """Score over a tree with spare capacity and blocks that hold nothing yet, against the
    oracle."""
    st = small_state(seed=7)
    for x in ("k", "v"):                           # rows that hold nothing are not read
        assert bool(torch.isnan(st[x]).any())
    kv, ost, V, N, W = to_gpu(st), oracle_state(st), 9, st["num_tokens"], 8
    Hq, gen = 8, torch.Generator().manual_seed(2)
    obs, sl = [3, 4, 5], [0, 1]
    qw = torch.randn((3, 2, Hq, W, 128), generator=gen).bfloat16()
    vs, us = torch.rand(V, generator=gen), torch.rand(V, generator=gen)
    A, rows = torch.zeros(N, device="cuda"), torch.zeros(V, dtype=torch.int64, device="cuda")
    a, s, stt = torch.empty(V, device="cuda"), torch.empty(V, device="cuda"), status()
    check_rc(L.arbor_score(kv, i32(obs), qw.cuda(), W, sl, vs.cuda(), us.cuda(), A, rows, a, s,
                           PARAMS, stt, workspace(kv, max_observers=3, window=W, n_slice=2)))
    Ao, ro, ao, so = O.score(ost, obs, np_float(qw), W, sl, 4, vs.numpy(), us.numpy(),
                             np.zeros(N, np.float32), np.zeros(V, np.int64), theta=PARAMS["theta"],
                             self_window=0)
    assert int(stt) == 0 and np.array_equal(rows.cpu().numpy(), ro)
    full = st["n_full"].numpy() > 0
    for got, want in ((A.cpu().numpy(), Ao), (a.cpu().numpy()[full], ao[full]),
                      (s.cpu().numpy()[full], so[full])):
        assert np.all(np.abs(got - want) <= 1e-4 * np.abs(want) + 1e-30)
    assert bool(torch.isfinite(a).all()) and bool(torch.isfinite(s).all())


def test_rows_beyond_four_gib():
    """Append, attention and forks where the pool's byte offsets pass 32 bits: the same bits
    as in a small pool."""
    st = grow_state([-1, 0, 0], [300, 40, 0], spare=300, kv_heads=8, q_per_kv=4, head_dim=128,
                    dtype="bf16", layers=1, extra_pages=8)
    small = to_gpu(st)
    far, pages = 150_000, st["num_pages"]          # 32 KiB a page of K: 4.9 GB before these
    st2 = dict(st, num_pages=far + pages)
    for x in ("k", "v"):
        st2[x] = torch.empty((1, 1, 8, 16, 128), dtype=torch.bfloat16)
    for x in ("page_table", "free_stack"):
        st2[x] = torch.where(st[x] >= 0, st[x] + far, st[x])
    st2["slot_pos"] = torch.cat((torch.full((far, 16), -1, dtype=torch.int32), st["slot_pos"]))
    st2["free_stack"] = torch.cat((st2["free_stack"], torch.full((far,), -1, dtype=torch.int32)))
    big = to_gpu(st2)
    for x in ("k", "v"):
        y = torch.empty((1, far + pages, 8, 16, 128), dtype=torch.bfloat16, device="cuda")
        y[:, far:] = getattr(small, x)
        setattr(big, x, y)
    a, b = (Step(kv, [0, 1], [70, 33]) for kv in (small, big))
    for s in (a, b):
        s()
        check_rc(L.arbor_fork(s.kv, i32([1]), i32([2]), s.status, s.ws2))
    assert int(a.status) == int(b.status) == 0
    assert torch.equal(a.q, b.q) and torch.equal(a.out, b.out) and torch.equal(a.lse, b.lse)
    assert torch.equal(a.slots + 16 * far, b.slots)
    for x, y in ((small.k, big.k), (small.v, big.v)):
        assert torch.equal(x.view(torch.int16), y[:, far:].view(torch.int16))
