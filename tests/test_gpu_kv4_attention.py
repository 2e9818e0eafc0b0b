"""seq_tree_kv4_attention against the definition in 64 bits, where it can go wrong."""
import numpy as np
import pytest
import torch

from paper_2402_12374_b200 import binding as B
from tests import kv4_util as U

pytestmark = pytest.mark.gpu
ROOM = 0  # tokens that a page table has room for, at least


@pytest.fixture(autouse=True, params=["tight", "roomy"])
def room(request):
    """The lengths' bound chooses the kernel: with room for 40000 tokens no cluster takes the few rows, nor small trees."""
    global ROOM
    ROOM = 40000 if request.param == "roomy" else 0
    return request.param


class Case:
    """Requests with the given prefix lengths over a shuffled pool; everything behind a prefix's last token is 0xFF (NaN scales)."""

    def __init__(self, lengths, n, Hq, Hkv, page, dt, seed=0, mask="common", layers=1, layer=0, max_len=None):
        rng = np.random.default_rng(seed)
        self.lengths, self.n, self.Hq, self.Hkv, self.page, self.dt = list(lengths), n, Hq, Hkv, page, dt
        R = len(lengths)
        self.count = [-(-max(L, 0) // page) for L in lengths]
        most = max(1, max(self.count), -(-ROOM // page))
        pages = sum(self.count) + 2
        self.pool = U.random_pool(pages, layers, Hkv, page, rng)
        self.table = np.full((R, most), 10 ** 6, dtype=np.int32)  # (what is behind the last page is not read)
        ids = rng.permutation(pages)
        at = 0
        for r, c in enumerate(self.count):
            self.table[r, :c] = ids[at:at + c]
            at += c
            if lengths[r] > 0:
                for t in range(lengths[r], c * page):
                    for h in range(Hkv):
                        for x, w in zip(U.place(page, Hkv, h, t), (64, 64, 4, 4)):
                            self.pool[self.table[r, c - 1], layer, x:x + w] = 0xFF
        g = torch.Generator().manual_seed(seed)
        self.q = torch.randn(R, n, Hq, 128, generator=g).to(dt)
        self.kt, self.vt = torch.randn(R, n, Hkv, 128, generator=g).to(dt), torch.randn(R, n, Hkv, 128, generator=g).to(dt)
        if mask == "chain":
            self.seen, self.mask = [np.tril(np.ones((n, n), dtype=bool))] * R, None
        elif mask == "common":
            _, s = U.tree(n, rng)
            self.seen, self.mask = [s] * R, torch.from_numpy(U.mask_words(s)).cuda()
        else:
            self.seen = [U.tree(n, rng)[1] for _ in range(R)]
            self.mask = torch.from_numpy(U.mask_words(np.stack(self.seen))).cuda()
        self.layer = layer
        self.pool_dev = torch.from_numpy(self.pool).reshape(pages, layers, Hkv, page * 136).cuda()
        self.max_len = max_len

    def call(self, q=None, **kw):
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")
        R = len(self.lengths)
        lse = torch.full((R, self.Hq, self.n), 7.0, device="cuda")
        args = dict(mask_bits=self.mask, max_len=self.max_len, lse=lse, dev_status=self.status)
        args.update(kw)
        return B.KV4AttentionCall((self.q if q is None else q).cuda(), self.kt.cuda(), self.vt.cuda(), self.pool_dev[:, self.layer],
                                  torch.from_numpy(self.table).cuda(), torch.tensor(self.lengths, dtype=torch.int32, device="cuda"), **args)

    def reference(self, r, **kw):
        k, v = U.prefix_rows(self.pool, self.layer, self.table[r], self.lengths[r], self.Hkv, self.page)
        return U.attention(self.q[r], self.kt[r], self.vt[r], k, v, self.seen[r], **kw)

    def check(self, exact_keys=False, status=0, **kw):
        call = self.call(**kw)
        out = call.run()
        torch.cuda.synchronize()
        assert int(self.status) == status
        for r, L in enumerate(self.lengths):
            if L >= 0:
                ref = self.reference(r, scale=kw.get("softmax_scale"), window=kw.get("window", 0), sinks=kw.get("sinks", 0))
                U.check_attention(out[r], call.lse[r], ref, self.dt, exact_keys)
        return out, call


BOTH = pytest.mark.parametrize("dt", [torch.float16, torch.bfloat16])


@BOTH
@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("L", [0, 1, 15, 16, 17, 31, 33, 127, 128, 129, 300])
def test_one_token_of_grouped_heads(L, page, dt):
    Case([L], 1, 8, 1, page, dt, seed=L).check()


@BOTH
@pytest.mark.parametrize("n,Hq,Hkv", [(1, 4, 4), (2, 8, 2), (8, 2, 2), (16, 1, 1), (5, 6, 2), (7, 10, 2), (3, 40, 8), (33, 2, 1), (64, 4, 4), (100, 10, 2),
                                      (200, 8, 1), (65, 16, 2), (1024, 1, 1), (700, 2, 1)])
def test_trees_and_groups(n, Hq, Hkv, dt):
    Case([77, 200], n, Hq, Hkv, 32, dt, seed=n, mask="each").check(exact_keys=dt == torch.float16)


@pytest.mark.parametrize("n,Hq", [(1, 2), (1, 130), (40, 3), (130, 1), (129, 4)])
def test_chain_without_a_mask(n, Hq):
    Case([50, 0], n, Hq, 1, 16, torch.float16, seed=3, mask="chain").check()


@BOTH
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 3), (16, 0), (40, 4), (100, 33), (127, 1), (128, 0), (129, 300), (5000, 2), (1 << 30, 1 << 30)])
@pytest.mark.parametrize("n,Hq", [(1, 8), (12, 1), (40, 4)])
def test_window_and_sinks(window, sinks, n, Hq, dt):
    Case([0, 5, 300, 431], n, Hq, 1, 16, dt, seed=window, mask="each").check(exact_keys=dt == torch.float16, window=window, sinks=sinks)


def test_window_inside_a_deep_tree():
    """A chain deeper than the window: ancestors drop out too, but for the sinks, which can lie in the tree."""
    for L, sinks in ((3, 0), (3, 6), (0, 2), (100, 4)):
        for Hq in (1, 4):
            Case([L], 60, Hq, 1, 16, torch.float16, seed=L, mask="chain").check(window=10, sinks=sinks)


@pytest.mark.parametrize("n,Hq", [(1, 8), (24, 4)])
def test_idle_slots_are_left_as_they_are(n, Hq):
    c = Case([40, -1, 0, -5, 90], n, Hq, 1, 16, torch.bfloat16)
    out = torch.full_like(c.q, 3.0).cuda()
    _, call = c.check(out=out)
    for r in (1, 3):
        assert (out[r] == 3.0).all() and (call.lse[r] == 7.0).all()


def test_every_slot_idle():
    c = Case([-1, -1], 1, 8, 1, 16, torch.float16)
    out = torch.full_like(c.q, 3.0).cuda()
    c.check(out=out)
    assert (out == 3.0).all()


@pytest.mark.parametrize("n,Hq", [(1, 8), (40, 4)])
def test_many_ragged_requests(n, Hq):
    """More units than ranges, ranges that cut units, and units cut into several."""
    rng = np.random.default_rng(1)
    Case(list(rng.integers(-1, 500, 60)), n, 2 * Hq, 2, 32, torch.bfloat16, seed=5).check()


@pytest.mark.parametrize("n,Hq", [(1, 4), (50, 4)])
def test_a_long_prefix_of_one_request(n, Hq):
    Case([6001], n, Hq, 1, 64, torch.float16, seed=5).check(exact_keys=True)


@BOTH
@pytest.mark.parametrize("n,Hq", [(1, 8), (40, 4)])
def test_the_largest_magnitudes_stay_finite(n, Hq, dt):
    """Rows up to +-65504, whose 4-bit forms reach past the largest half, before the window; rows below 6e4 inside."""
    c = Case([300], n, Hq, 1, 16, dt, seed=12, mask="each")
    rng = np.random.default_rng(5)
    for t in range(300):
        for kv in range(2):
            x = rng.uniform(-1, 1, 128) * (65504 if t < 150 else 1.0 if kv == 0 else 6e4)
            if t < 150:
                x[:2] = (65504, -65504) if t % 2 else (65504, 65000)
                x = np.clip(x, 65000, 65504) if t % 4 == 0 else x
            U.store(c.pool, c.table[0, t // 16], 0, 0, 16, t, kv, *U.quantise(x))
    c.pool_dev = torch.from_numpy(c.pool).reshape(c.pool.shape[0], 1, 1, -1).cuda()
    c.check(window=100)


@BOTH
@pytest.mark.parametrize("n,Hq", [(1, 8), (40, 4)])
def test_scales_of_many_magnitudes(n, Hq, dt):
    """Values from 1e-3 to 1e4 among the keys and values, large ones where a window hides them, rows of one number (scale 0)."""
    c = Case([300, 200], n, Hq, 1, 16, dt, seed=12, mask="each")
    rng = np.random.default_rng(5)
    for r, L in enumerate(c.lengths):
        for t in range(L):
            for kv in range(2):
                size = 10.0 ** rng.uniform(-3, -1) if t < L // 2 else 10.0 ** rng.uniform(-1, 1 if kv == 0 else 4)
                x = rng.standard_normal(128) * size + size if t % 7 else np.full(128, size)
                U.store(c.pool, c.table[r, t // 16], 0, 0, 16, t, kv, *U.quantise(x))
    c.pool_dev = torch.from_numpy(c.pool).reshape(c.pool.shape[0], 1, 1, -1).cuda()
    c.q = c.q * 0.1
    c.check()
    c.check(window=64, sinks=30)


def test_same_call_same_bits_and_any_workspace_contents():
    for n, lengths in ((1, [900, 30, 411]), (1, [900, 30, 411] * 40), (40, [900, 30, 411])):
        c = Case(lengths, n, 8, 2, 16, torch.bfloat16)
        call = c.call()
        a = call.run().clone()
        if call.workspace is not None:
            call.workspace.fill_(0xFF)
        call.out.zero_()
        assert torch.equal(a, call.run())


def test_a_request_alone_and_in_a_batch():
    """What a request gets does not depend on its neighbours beyond rounding: both are within rounding of the definition."""
    c = Case([333, 20], 3, 4, 2, 16, torch.float16)
    c.check()
    d = Case([333], 3, 4, 2, 16, torch.float16)
    d.check()


@pytest.mark.parametrize("n,Hq", [(2, 4), (50, 4)])
def test_strides_and_layers(n, Hq):
    """q, out and the tree's rows inside larger arrays, one layer of a pool of three."""
    c = Case([70, 130], n, Hq, 2, 16, torch.float16, layers=3, layer=1, seed=2)
    R = 2
    big_q = torch.full((R, n + 1, Hq + 3, 136), float("nan"), dtype=c.dt, device="cuda")
    big_t = torch.full((2, R + 1, Hq, n, 2, 128), float("nan"), dtype=c.dt, device="cuda")
    big_o = torch.full((R, Hq, n + 2, 256), 5.0, dtype=c.dt, device="cuda")
    q, out = big_q[:, :n, :Hq, 8:], big_o[:, :, :n, 64:192].transpose(1, 2)
    kt, vt = big_t[0, 1:, 0], big_t[1, 1:, 0]
    q.copy_(c.q), kt.copy_(c.kt), vt.copy_(c.vt)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    B.seq_tree_kv4_attention(q, kt, vt, c.pool_dev[:, 1], torch.from_numpy(c.table).cuda(), torch.tensor(c.lengths, dtype=torch.int32, device="cuda"),
                             mask_bits=c.mask, out=out, dev_status=status)
    assert int(status) == 0
    for r in range(R):
        U.check_attention(out[r], None, c.reference(r), c.dt, False)
    assert (big_o[..., :64] == 5).all() and (big_o[..., 192:] == 5).all() and (big_o[:, :, n:] == 5).all()


@BOTH
@pytest.mark.parametrize("n,Hq", [(6, 2), (40, 4)])
def test_rows_that_a_node_does_not_see_may_hold_anything(n, Hq, dt):
    c = Case([45], n, Hq, 1, 16, dt, seed=8)
    star = np.eye(n, dtype=bool)
    star[:, 0] = True
    c.seen, c.mask = [star], torch.from_numpy(U.mask_words(star)).cuda()
    clean, _ = c.check()
    bad = {2: float("nan"), 3: float("inf"), n - 1: -float("inf")}
    for j, x in bad.items():
        c.kt[0, j, 0, 5] = x
        c.vt[0, j, 0, 7] = x
    out = c.call().run()
    for i in range(n):
        if i in bad:
            assert torch.isnan(out[0, i]).all(), i
        else:
            assert torch.equal(out[0, i], clean[0, i]), i


@BOTH
@pytest.mark.parametrize("n,Hq", [(1, 8), (20, 4)])
def test_a_row_of_q_that_is_not_finite_stays_alone(n, Hq, dt):
    c = Case([45], n, Hq, 1, 16, dt, seed=8)
    clean = c.call().run().clone()
    c.q[0, n - 1, 1, 3] = float("nan")
    out = c.call().run()
    assert torch.isnan(out[0, n - 1, 1]).all()
    keep = torch.ones(n, Hq, dtype=torch.bool)
    keep[n - 1, 1] = False
    assert torch.equal(out[0][keep], clean[0][keep])


@pytest.mark.parametrize("size", [1e-30, 1e-4, 300.0])
@pytest.mark.parametrize("n", [1, 40])
def test_magnitudes_of_q(n, size):
    """bfloat16 rows are scaled into half precision by a power of two: no magnitude is lost."""
    c = Case([45], n, 4, 1, 16, torch.bfloat16, seed=8)
    c.q = (c.q.float() * size).to(torch.bfloat16)
    c.kt = (c.kt.float() * 0.3).to(torch.bfloat16)
    c.q[0, 0, 0] = 0
    c.check(softmax_scale=0.1 / max(size, 1e-2))


def test_scores_that_rise_by_far():
    """Reference maxima move many times: keys that grow along the prefix, and a last key far above all others."""
    for n, Hq in ((1, 8), (40, 4)):
        c = Case([700], n, Hq, 1, 16, torch.float16, seed=4)
        c.q = torch.ones_like(c.q)
        for t in range(700):
            x = np.random.default_rng(t).standard_normal(128) + 0.02 * t
            nib, s, m = U.quantise(x)
            U.store(c.pool, c.table[0, t // 16], 0, 0, 16, t, 0, nib, s, m)
        c.pool_dev = torch.from_numpy(c.pool).reshape(c.pool.shape[0], 1, 1, -1).cuda()
        c.check()


def test_bad_pages_and_lengths_are_reported():
    for n in (1, 40):
        for page in (16, 64):
            c = Case([100, 64], n, 8, 1, page, torch.float16, seed=4)
            c.table[1, 0] = -1
            out, _ = None, None
            call = c.call()
            got = call.run().clone()
            assert int(c.status) == B.SEQ_DEV_BAD_PAGE
            c.table[1, 0] = 0
            assert torch.equal(got, c.call().run())
            c.table[0, 100 // page] = c.pool.shape[0]  # one behind the last
            c.call().run()
            assert int(c.status) == B.SEQ_DEV_BAD_PAGE
        c = Case([100], n, 8, 1, 16, torch.float16, seed=4)
        call = c.call(max_len=60)
        got = call.run().clone()
        assert int(c.status) == B.SEQ_DEV_BAD_LENGTH
        c.lengths = [60]
        assert torch.equal(got, c.call(max_len=60).run())
        c = Case([100] + [45] * 299, n, 8, 2, 16, torch.float16, seed=4)
        call = c.call(max_len=60)
        got = call.run().clone()
        assert call.workspace_bytes_needed > 0 and int(c.status) == B.SEQ_DEV_BAD_LENGTH
        c.lengths[0] = 60
        assert torch.equal(got, c.call(max_len=60).run())


def test_graph_replayed_while_prefixes_grow_on_another_stream():
    for n, Hq in ((1, 8), (24, 4)):
        c = Case([200, 90], n, Hq, 1, 16, torch.bfloat16, seed=6)
        lengths = torch.tensor([150, 20], dtype=torch.int32, device="cuda")
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream):
            call = B.KV4AttentionCall(c.q.cuda(), c.kt.cuda(), c.vt.cuda(), c.pool_dev[:, 0], torch.from_numpy(c.table).cuda(), lengths, mask_bits=c.mask,
                                      dev_status=status)
            call.run()
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call.run()
        for now in ([150, 20], [200, 90], [1, -1], [0, 33]):
            lengths.copy_(torch.tensor(now, dtype=torch.int32))
            graph.replay()
            torch.cuda.synchronize()
            for r, L in enumerate(now):
                if L >= 0:
                    k, v = U.prefix_rows(c.pool, 0, c.table[r], L, 1, 16)
                    U.check_attention(call.out[r], None, U.attention(c.q[r], c.kt[r], c.vt[r], k, v, c.seen[r]), c.dt, False)
        assert int(status) == 0


def test_offsets_beyond_32_bits():
    """Pages more than 2^32 bytes into the pool."""
    page, heads = 128, 8
    part = page * 136
    pages = (1 << 32) // (heads * part) + 40
    pool = torch.zeros((pages, heads, part), dtype=torch.uint8, device="cuda")
    for n in (1, 40):
        c = Case([300], n, 8, 8, page, torch.float16, seed=9)
        far = pages - c.pool.shape[0]
        pool[far:] = c.pool_dev[:, 0]
        out = B.seq_tree_kv4_attention(c.q.cuda(), c.kt.cuda(), c.vt.cuda(), pool, torch.from_numpy(c.table + far).cuda(),
                                       torch.tensor([300], dtype=torch.int32, device="cuda"), mask_bits=c.mask)
        U.check_attention(out[0], None, c.reference(0), c.dt, False)


def test_workspace_that_is_too_small_is_refused(room):
    for lengths, n in (([45] * 300, 1), ([45], 400)):
        c = Case(lengths, n, 16, 2, 16, torch.float16)
        need = c.call().workspace_bytes_needed
        assert need > 0
        call = c.call(workspace=torch.empty(need - 16, dtype=torch.uint8, device="cuda"))
        with pytest.raises(B.SeqTreeError, match="WORKSPACE"):
            call.run()
    if room == "tight":
        assert Case([45], 1, 8, 1, 16, torch.float16).call().workspace is None  # a cluster a unit: none is needed


def test_memory_of_a_call_on_another_stream_is_not_handed_out(room):
    """The workspace and out of a call on a stream of its own outlive the call object until that stream is through."""
    c = Case([300, 20, 411] * 12, 1, 8, 2, 16, torch.float16, seed=3) if room == "roomy" else Case([300, 20] * 30, 20, 8, 2, 16, torch.float16, seed=3)
    want = c.call().run().clone()
    q, kt, vt, pool, table = c.q.cuda(), c.kt.cuda(), c.vt.cuda(), c.pool_dev[:, 0], torch.from_numpy(c.table).cuda()
    lengths = torch.tensor(c.lengths, dtype=torch.int32, device="cuda")
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(50_000_000)
    call = B.KV4AttentionCall(q, kt, vt, pool, table, lengths, mask_bits=c.mask)
    need, held = call.workspace_bytes_needed, set(t.data_ptr() for t in (call.out, call.workspace) if t is not None)
    out = call.run(stream=side)
    del call
    others = [torch.empty(max(need, 1), dtype=torch.uint8, device="cuda") for _ in range(4)]
    assert need > 0 and not held & set(t.data_ptr() for t in others)
    side.synchronize()
    assert torch.equal(out, want)


def test_tensors_of_another_device_are_refused(monkeypatch):
    """The launch goes to the current device."""
    c = Case([45], 1, 8, 1, 16, torch.float16)
    call = c.call()
    one = torch.zeros(1, dtype=torch.int32, device="cuda")
    rows = torch.zeros(1, 1, 2, 1, 128, dtype=torch.float16, device="cuda")
    table = torch.from_numpy(c.table).cuda()
    refs = torch.zeros(c.pool.shape[0], dtype=torch.int32, device="cuda")
    monkeypatch.setattr(B, "_raw_device", lambda: 1)
    for f in (call.run, c.call, lambda: B.seq_tree_kv4_append(rows, rows, c.pool_dev, table, one), lambda: B.seq_tree_kv4_read(c.pool_dev, table, rows, rows),
              lambda: B.seq_tree_pages_resize(table, one, refs, one, 16), lambda: B.seq_tree_pages_compact(c.pool_dev, table, one, refs),
              lambda: B.seq_tree_pages_fork(c.pool_dev, table, one, refs, one, one, 16)):
        with pytest.raises(ValueError, match="current device"):
            f()
