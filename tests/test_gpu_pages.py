"""seq_tree_pages_resize, _fork, _compact against their definitions, slot by slot."""
import numpy as np
import pytest
import torch

from paper_2402_12374_b200 import binding as B
from tests import kv4_util as U

pytestmark = pytest.mark.gpu


def state(slots, most, pages, page_size, seed, fill=0.5, shared=True):
    """A sound state: some slots empty, some with a beginning in common."""
    rng = np.random.default_rng(seed)
    count = rng.integers(0, most + 1, slots) * (rng.random(slots) < 0.8)
    while count.sum() > fill * pages:
        count = count * 3 // 4
    table = np.full((slots, most), -1, dtype=np.int32)
    ids = rng.permutation(pages)
    at = 0
    for r in range(slots):
        table[r, :count[r]] = ids[at:at + count[r]]
        at += count[r]
    if shared:
        for r in range(0, slots, 3):
            o = int(rng.integers(0, slots))
            m = int(min(count[r], count[o]) // 2)
            table[r, :m] = table[o, :m]
    refs = np.bincount(table[table >= 0], minlength=pages).astype(np.int32)
    lengths = np.where(count > 0, count * page_size - rng.integers(0, page_size, slots), 0)
    return table, count.astype(np.int32), refs, lengths.astype(np.int32), rng


def dev(*xs):
    return [torch.from_numpy(np.array(x)).cuda() for x in xs]


def status():
    return torch.zeros(1, dtype=torch.int32, device="cuda")


SHAPES = [(1, 1, 1), (1, 5, 7), (16, 40, 300), (33, 7, 64), (256, 100, 20000), (2048, 3, 4001), (5, 3000, 9000), (700, 300, 150001)]


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("slots,most,pages", SHAPES)
def test_resize(slots, most, pages, in_place):
    for seed, fill in ((1, 0.5), (2, 0.95)):
        table, count, refs, lengths, rng = state(slots, most, pages, 16, seed, fill)
        tokens = rng.integers(-1, most * 16 + 1, slots).astype(np.int32)
        want = U.resize(table, count, refs, tokens, 16)
        t, c, f, tok = dev(table, count, refs, tokens)
        outs = (t, c, f) if in_place else [torch.full_like(x, 77) for x in (t, c, f)]
        kw = {} if in_place else dict(table_out=outs[0], count_out=outs[1], refs_out=outs[2])
        st = status()
        B.seq_tree_pages_resize(t, c, f, tok, 16, dev_status=st, **kw)
        assert int(st) == (B.SEQ_DEV_NO_PAGES if want[3] else 0)
        for got, ref in zip(outs, want):
            assert np.array_equal(got.cpu().numpy(), ref)
        if not in_place:
            assert np.array_equal(t.cpu().numpy(), table) and np.array_equal(f.cpu().numpy(), refs)


def test_resize_frees_everything_and_fills_a_pool_to_the_last_page():
    table, count, refs, _, _ = state(20, 30, 400, 16, 3)
    t, c, f = dev(table, count, refs)
    st = status()
    B.seq_tree_pages_resize(t, c, f, torch.zeros(20, dtype=torch.int32, device="cuda"), 16, dev_status=st)
    assert int(st) == 0 and (t == -1).all() and (c == 0).all() and (f == 0).all()
    B.seq_tree_pages_resize(t, c, f, torch.full((20,), 20 * 16, dtype=torch.int32, device="cuda"), 16, dev_status=st)
    assert int(st) == 0 and (c == 20).all() and (f == 1).all()
    assert torch.equal(t[:, :20].flatten(), torch.arange(400, dtype=torch.int32, device="cuda"))
    B.seq_tree_pages_resize(t, c, f, torch.full((20,), 20 * 16 + 1, dtype=torch.int32, device="cuda"), 16, dev_status=st)
    assert int(st) == B.SEQ_DEV_NO_PAGES and (c == 20).all() and (t[:, 20:] == -1).all()


def test_resize_reports_what_contradicts_itself():
    table, count, refs, _, _ = state(8, 10, 60, 16, 4, shared=False)
    count[:] = [3, 3, 3, 3, 0, 0, 0, 0]
    table[:] = -1
    table[:4, :3] = np.arange(12).reshape(4, 3)
    refs[:] = 0
    refs[:12] = 1
    # a count that cannot be, a size that cannot be
    c2 = count.copy()
    c2[1] = 11
    t, c, f, tok = dev(table, c2, refs, np.array([0, 0, 161, -1, 16, 0, 0, 0], dtype=np.int32))
    st = status()
    B.seq_tree_pages_resize(t, c, f, tok, 16, dev_status=st)
    assert int(st) == B.SEQ_DEV_BAD_SLOT
    assert c.tolist() == [0, 11, 3, 3, 1, 0, 0, 0] and t[4, 0] == 0 and t[1].tolist() == table[1].tolist()
    # a page outside the pool, a reference too many given up
    table2, refs2 = table.copy(), refs.copy()
    table2[0, 1], refs2[4] = 60, 0
    t, c, f, tok = dev(table2, count, refs2, np.array([0, 0, -1, -1, -1, -1, -1, -1], dtype=np.int32))
    st = status()
    B.seq_tree_pages_resize(t, c, f, tok, 16, dev_status=st)
    assert int(st) == B.SEQ_DEV_BAD_PAGE | B.SEQ_DEV_BAD_SLOT
    assert c.tolist() == [0, 0, 3, 3, 0, 0, 0, 0] and f[:6].tolist() == [0, 1, 0, 0, 0, 0]


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("slots,most,pages", SHAPES[:-1])
def test_fork(slots, most, pages, in_place):
    for seed in (1, 2, 3):
        page_size = [16, 1, 7][seed - 1]
        table, count, refs, lengths, rng = state(slots, most, pages, page_size, seed, 0.5 if seed < 3 else 0.97)
        source = np.where((count == 0) & (rng.random(slots) < 0.8), rng.integers(0, slots, slots), -1).astype(np.int32)
        pool = rng.integers(0, 256, (pages, 3, 16), dtype=np.uint8)
        want = U.fork(pool, table, count, refs, lengths, source, page_size)
        p, t, c, f, n, s = dev(pool, table, count, refs, lengths, source)
        outs = (t, c, f, n) if in_place else [torch.full_like(x, 77) for x in (t, c, f, n)]
        kw = {} if in_place else dict(table_out=outs[0], count_out=outs[1], refs_out=outs[2], lengths_out=outs[3])
        st = status()
        B.seq_tree_pages_fork(p, t, c, f, n, s, page_size, dev_status=st, **kw)
        assert int(st) == (B.SEQ_DEV_BAD_SLOT if want[5] else 0) | (B.SEQ_DEV_NO_PAGES if want[6] else 0)
        for got, ref in zip((p, *outs), want):
            assert np.array_equal(got.cpu().numpy(), ref)


def test_fork_reports_what_it_cannot_do():
    table = np.full((6, 4), -1, dtype=np.int32)
    table[0, :3], table[1, :1] = [4, 2, 9], [0]
    count, lengths = np.array([3, 1, 0, 0, 0, 0], dtype=np.int32), np.array([40, 17, 5, 0, -1, 0], dtype=np.int32)
    refs = np.bincount(table[table >= 0], minlength=12).astype(np.int32)
    pool = np.arange(12 * 64, dtype=np.uint8).reshape(12, 64)
    for r, s in ((2, 6), (2, 2), (1, 0), (2, 1), (3, 4), (3, 2)):  # no such slot, itself, not empty, longer than its pages (twice), idle
        source = np.full(6, -1, dtype=np.int32)
        source[r] = s
        p, t, c, f, n, src = dev(pool, table, count, refs, lengths, source)
        st = status()
        B.seq_tree_pages_fork(p, t, c, f, n, src, 16, dev_status=st)
        assert int(st) == B.SEQ_DEV_BAD_SLOT, (r, s)
        for got, was in ((p, pool), (t, table), (c, count), (f, refs), (n, lengths)):
            assert np.array_equal(got.cpu().numpy(), was)
    # a fork of an empty slot is empty, also of one that is itself being forked
    source = np.array([-1, -1, -1, 0, -1, 3], dtype=np.int32)
    p, t, c, f, n, src = dev(pool, table, count, refs, lengths, source)
    st = status()
    B.seq_tree_pages_fork(p, t, c, f, n, src, 16, dev_status=st)
    assert int(st) == 0 and c.tolist() == [3, 1, 0, 3, 0, 0] and n.tolist() == [40, 17, 5, 40, -1, 0] and t[3].tolist() == [4, 2, 1, -1]
    assert torch.equal(p[1], p[9])


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("slots,most,pages", SHAPES)
def test_compact(slots, most, pages, in_place):
    for seed, fill in ((1, 0.5), (2, 0.97), (3, 0.05)):
        table, count, refs, _, rng = state(slots, most, pages, 16, seed, fill)
        pool = rng.integers(0, 256, (pages, 16), dtype=np.uint8)
        want = U.compact(pool, table, count, refs)
        p, t, c, f = dev(pool, table, count, refs)
        outs = (t, f) if in_place else [torch.full_like(x, 77) for x in (t, f)]
        kw = {} if in_place else dict(table_out=outs[0], refs_out=outs[1])
        st, live = status(), torch.full((1,), -1, dtype=torch.int32, device="cuda")
        B.seq_tree_pages_compact(p, t, c, f, live=live, dev_status=st, **kw)
        assert int(st) == 0 and int(live) == want[3]
        assert np.array_equal(p.cpu().numpy()[:want[3]], want[0][:want[3]])
        assert np.array_equal(outs[0].cpu().numpy(), want[1]) and np.array_equal(outs[1].cpu().numpy(), want[2])


@pytest.mark.parametrize("page_bytes", [16, 48, 32768, 32784, 100000 // 16 * 16])
def test_pages_of_any_size_type_and_planes(page_bytes):
    """Contents: several planes with gaps between them, pages that end inside a piece, what lies between pages stays."""
    table, count, refs, lengths, rng = state(9, 6, 40, 16, 5)
    big = torch.from_numpy(rng.integers(0, 256, (3, 41, page_bytes + 32), dtype=np.uint8)).cuda()
    pool = big[:, :40, 16:16 + page_bytes]
    want = U.compact(pool.transpose(0, 1).cpu().numpy(), table, count, refs)
    before = big.clone()
    t, c, f = dev(table, count, refs)
    B.seq_tree_pages_compact(pool, t, c, f, planes=True)
    live = want[3]
    assert np.array_equal(pool.transpose(0, 1).cpu().numpy()[:live], want[0][:live])
    before[:, :40, 16:16 + page_bytes] = pool
    assert torch.equal(before, big)
    # the same pages as a pool of halves, forked
    table, count, refs, lengths, rng = state(9, 6, 40, 16, 6)
    source = np.where(count == 0, int(np.argmax(lengths)), -1).astype(np.int32)
    pool16 = torch.from_numpy(rng.standard_normal((40, page_bytes // 2)).astype(np.float16)).cuda()
    want = U.fork(pool16.cpu().numpy(), table, count, refs, lengths, source, 16)
    t, c, f, n, s = dev(table, count, refs, lengths, source)
    B.seq_tree_pages_fork(pool16, t, c, f, n, s, 16)
    assert np.array_equal(pool16.cpu().numpy(), want[0]) and np.array_equal(t.cpu().numpy(), want[1])


def test_compact_reports_tables_that_name_no_page():
    table = np.array([[3, 9, -1], [1, 0, -1]], dtype=np.int32)
    count, refs = np.array([2, 1], dtype=np.int32), np.array([0, 1, 0, 1], dtype=np.int32)
    pool = np.arange(4 * 16, dtype=np.uint8).reshape(4, 16)
    p, t, c, f = dev(pool, table, count, refs)
    st = status()
    B.seq_tree_pages_compact(p, t, c, f, dev_status=st)
    assert int(st) == B.SEQ_DEV_BAD_PAGE and t.tolist() == [[0, -1, -1], [1, 0, -1]] and f.tolist() == [1, 1, 0, 0]
    st = status()
    p, t, c, f = dev(pool, np.array([[3, 2], [1, -1]], dtype=np.int32), np.array([2, 5], dtype=np.int32), refs)
    B.seq_tree_pages_compact(p, t, c, f, dev_status=st)
    assert int(st) == B.SEQ_DEV_BAD_SLOT and t.tolist() == [[0, -1], [1, -1]]  # page 2 is held but free; a count of 5


def test_a_serving_loop_in_one_graph():
    """Grow, append, attend, commit: two requests, one forked from the other half way, replayed from one CUDA graph."""
    page, heads, dt = 16, 2, torch.float16
    slots, most, pages, n = 3, 12, 30, 4
    g = torch.Generator(device="cuda").manual_seed(0)
    pool = torch.zeros((pages, 1, heads, page * 136), dtype=torch.uint8, device="cuda")
    i32 = dict(dtype=torch.int32, device="cuda")
    table, count, refs, lengths = torch.full((slots, most), -1, **i32), torch.zeros(slots, **i32), torch.zeros(pages, **i32), torch.zeros(slots, **i32)
    st = status()
    prompt = [torch.randn((1, slots, 40, heads, 128), device="cuda", generator=g).to(dt) for _ in range(2)]
    have = torch.tensor([37, 21, 0], **i32)
    B.seq_tree_pages_resize(table, count, refs, have, page, dev_status=st)
    new = torch.zeros(slots, **i32)
    B.seq_tree_kv4_append(*prompt, pool, table, lengths, count=have, new_lengths=new, dev_status=st)
    lengths.copy_(new)
    B.seq_tree_pages_fork(pool, table, count, refs, lengths, torch.tensor([-1, -1, 0], **i32), page, dev_status=st)
    assert int(st) == 0 and lengths.tolist() == [37, 21, 37] and refs.sum() == 8 and count.tolist() == [3, 2, 3]
    rows = [[x[0, r, :m].cpu() for x in prompt] for r, m in ((0, 37), (1, 21), (0, 37))]

    q = torch.empty((slots, n, 4, 128), dtype=dt, device="cuda")
    k, v = torch.empty((1, slots, n, heads, 128), dtype=dt, device="cuda"), torch.empty((1, slots, n, heads, 128), dtype=dt, device="cuda")
    path, path_len = torch.zeros((slots, n), **i32), torch.zeros(slots, **i32)
    attend = B.KV4AttentionCall(q, k[0], v[0], pool[:, 0], table, lengths, dev_status=st)  # a chain

    def step():
        B.seq_tree_pages_resize(table, count, refs, lengths + n, page, dev_status=st)
        attend.run()
        B.seq_tree_kv4_append(k, v, pool, table, lengths, count=path_len, path=path, new_lengths=new, dev_status=st)
        lengths.copy_(new)

    def refill():
        for x in (q, k, v):
            x.copy_(torch.randn(x.shape, device="cuda", generator=g))
        path_len.copy_(torch.randint(1, n + 1, (slots,), device="cuda", generator=g))
        path.copy_(torch.arange(n, device="cuda", dtype=torch.int32))

    saved = [x.clone() for x in (table, count, refs, lengths, pool)]
    refill()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        step()
    torch.cuda.current_stream().wait_stream(stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for x, s in zip((table, count, refs, lengths, pool), saved):
        x.copy_(s)
    for _ in range(6):
        refill()
        before = lengths.tolist()
        graph.replay()
        torch.cuda.synchronize()
        assert int(st) == 0
        for r in range(slots):
            stored = [np.stack([U.quantise(x.double().numpy())[0].astype(float) - 8]) for x in rows[r]]
            vals = []
            for x in rows[r]:
                nib, s, m = U.quantise(x.double().numpy())
                vals.append((s[..., None].astype(float) * (nib.astype(float) - 8) + m[..., None]).transpose(1, 0, 2))
            assert before[r] == len(rows[r][0]) and stored[0].shape[1] == before[r]
            ref = U.attention(q[r].cpu(), k[0, r].cpu(), v[0, r].cpu(), vals[0], vals[1], np.tril(np.ones((n, n), dtype=bool)))
            U.check_attention(attend.out[r], None, ref, dt, False)
            m = int(path_len[r])
            rows[r] = [torch.cat([rows[r][0], k[0, r, :m].cpu()]), torch.cat([rows[r][1], v[0, r, :m].cpu()])]
        assert lengths.tolist() == [len(x[0]) for x in rows]
    held = table[table >= 0]
    assert torch.equal(torch.bincount(held.long(), minlength=pages).int(), refs)


@pytest.mark.parametrize("handle", [False, True])
def test_a_workspace_on_another_stream_is_that_streams_own(handle):
    """The current stream still writes to memory of the workspace's size that it has given back: a call on another stream does not get it."""
    table, count, refs, lengths, rng = state(33, 40, 30000, 16, 3)
    tokens = rng.integers(-1, 40 * 16 + 1, 33).astype(np.int32)
    source = np.where(count == 0, int(np.argmax(lengths)), -1).astype(np.int32)
    pool = rng.integers(0, 256, (30000, 16), dtype=np.uint8)
    want_resize, want_fork, want_compact = (U.resize(table, count, refs, tokens, 16), U.fork(pool, table, count, refs, lengths, source, 16),
                                            U.compact(pool, table, count, refs))
    side = torch.cuda.Stream()
    on = side.cuda_stream if handle else side
    # (kernels are loaded at their first launch, which waits for the device)
    p, t, c, f, n, tok, src = dev(pool, table, count, refs, lengths, tokens, source)
    B.seq_tree_pages_fork(p, t, c, f, n, src, 16)
    B.seq_tree_pages_compact(p, t, c, f)
    B.seq_tree_pages_resize(t, c, f, tok, 16)
    for call in ("resize", "fork", "compact"):
        p, t, c, f, n, tok, src = dev(pool, table, count, refs, lengths, tokens, source)
        torch.cuda.synchronize()
        torch.cuda.empty_cache()
        before = torch.empty(1 + 3 * 30000, dtype=torch.int32, device="cuda")
        before.fill_(0)  # (what is asked for behind the wait has been loaded)
        torch.cuda._sleep(1_000_000_000)
        before.fill_(7)
        through = torch.cuda.Event()
        through.record()
        del before
        if call == "resize":
            B.seq_tree_pages_resize(t, c, f, tok, 16, stream=on)
        elif call == "fork":
            B.seq_tree_pages_fork(p, t, c, f, n, src, 16, stream=on)
        else:
            B.seq_tree_pages_compact(p, t, c, f, stream=on)
        side.synchronize()
        assert not through.query()  # (it did not wait for the current stream either)
        torch.cuda.synchronize()
        want = {"resize": (t, want_resize[0], f, want_resize[2]), "fork": (t, want_fork[1], f, want_fork[3]), "compact": (t, want_compact[1], f, want_compact[2])}[call]
        assert np.array_equal(want[0].cpu().numpy(), want[1]) and np.array_equal(want[2].cpu().numpy(), want[3])


def both_ways(call, arrays, outs):
    """``call(arrays, outputs)`` in place and into other arrays: the same status and the same results, which are returned."""
    results = []
    for in_place in (True, False):
        on = dict(zip(arrays, dev(*arrays.values())))
        to = {x: on[x] if in_place else torch.full_like(on[x], 77) for x in outs}
        st = status()
        call(on, to if not in_place else {}, st)
        results.append([int(st)] + [to[x].cpu().numpy() for x in outs] + ([on["pool"].cpu().numpy()] if "pool" in on else []))
    for a, b in zip(*results):
        assert np.array_equal(a, b), (a, b)
    return results[0]


def resize_call(on, to, st):
    kw = {x + "_out": y for x, y in to.items()}
    B.seq_tree_pages_resize(on["table"], on["count"], on["refs"], on["tokens"], 16, dev_status=st, **kw)


def fork_call(on, to, st):
    kw = {x + "_out": y for x, y in to.items()}
    B.seq_tree_pages_fork(on["pool"], on["table"], on["count"], on["refs"], on["lengths"], on["source"], 16, dev_status=st, **kw)


def compact_call(on, to, st):
    kw = {x + "_out": y for x, y in to.items()}
    B.seq_tree_pages_compact(on["pool"], on["table"], on["count"], on["refs"], dev_status=st, **kw)


def i32(x):
    return np.array(x, dtype=np.int32)


@pytest.mark.parametrize("wrong", [-1, -(1 << 31), 4, 1 << 30])
def test_a_slot_whose_count_cannot_be_is_left_alone(wrong):
    """Slot 1 takes no part in the calls; its row has something behind what a sound slot would have."""
    table, refs = i32([[5, -1, -1], [2, 9, 8], [-1, -1, -1]]), i32([0, 0, 1, 0, 0, 1, 0])
    count, pool = i32([1, wrong, 0]), np.arange(7 * 16, dtype=np.uint8).reshape(7, 16)
    got = both_ways(resize_call, dict(table=table, count=count, refs=refs, tokens=i32([17, 0, 1])), ("table", "count", "refs"))
    assert got[0] == B.SEQ_DEV_BAD_SLOT and got[1].tolist() == [[5, 0, -1], [2, 9, 8], [1, -1, -1]] and got[2].tolist() == [2, wrong, 1]
    assert got[3].tolist() == [1, 1, 1, 0, 0, 1, 0]
    got = both_ways(fork_call, dict(pool=pool, table=table, count=count, refs=refs, lengths=i32([16, 40, 0]), source=i32([-1, -1, 0])),
                    ("table", "count", "refs", "lengths"))
    assert got[0] == B.SEQ_DEV_BAD_SLOT and got[1].tolist() == [[5, -1, -1], [2, 9, 8], [5, -1, -1]] and got[2].tolist() == [1, wrong, 1]
    assert got[3].tolist() == [0, 0, 1, 0, 0, 2, 0] and got[4].tolist() == [16, 40, 16]
    got = both_ways(compact_call, dict(pool=pool, table=table, count=count, refs=refs), ("table", "refs"))
    assert got[0] == B.SEQ_DEV_BAD_SLOT and got[1].tolist() == [[1, -1, -1], [2, 9, 8], [-1, -1, -1]] and got[2].tolist() == [1, 1, 0, 0, 0, 0, 0]


def test_fork_counts_a_negative_reference_as_none():
    table, count, lengths = i32([[3, 4], [-1, -1], [-1, -1]]), i32([2, 0, 0]), i32([20, 0, 0])
    pool = np.arange(6 * 16, dtype=np.uint8).reshape(6, 16)
    # page 0: free but for its count; page 5 as well, and nobody gets it
    got = both_ways(fork_call, dict(pool=pool, table=table, count=count, refs=i32([-3, 1, 1, 1, 1, -1]), lengths=lengths, source=i32([-1, 0, -1])),
                    ("table", "count", "refs", "lengths"))
    assert got[0] == B.SEQ_DEV_BAD_SLOT and got[1].tolist() == [[3, 4], [3, 0], [-1, -1]] and got[3].tolist() == [1, 1, 1, 2, 1, 0]
    assert np.array_equal(got[5][0], pool[4])
    got = both_ways(fork_call, dict(pool=pool, table=table, count=count, refs=i32([0, 1, 1, 1, 1, -1]), lengths=lengths, source=i32([-1, -1, -1])),
                    ("table", "count", "refs", "lengths"))
    assert got[0] == B.SEQ_DEV_BAD_SLOT and got[3].tolist() == [0, 1, 1, 1, 1, 0] and got[1].tolist() == table.tolist()


@pytest.mark.parametrize("held", [0, -1])
def test_fork_of_pages_that_count_as_free(held):
    table, count, lengths, source = i32([[3, 4], [-1, -1], [-1, -1]]), i32([2, 0, 0]), i32([20, 0, 0]), i32([-1, 0, 0])
    pool = np.arange(6 * 16, dtype=np.uint8).reshape(6, 16)
    # the full page: shared by two from 0 on, and by what it is handed out to
    for refs, own in (([1, 0, 1, held, 1, 1], [1, 3]), ([1, 1, 1, held, 1, 1], [3, None])):
        got = both_ways(fork_call, dict(pool=pool, table=table, count=count, refs=i32(refs), lengths=lengths, source=source), ("table", "count", "refs", "lengths"))
        short = own[1] is None
        assert got[0] == B.SEQ_DEV_BAD_SLOT | (B.SEQ_DEV_NO_PAGES if short else 0)
        assert got[1].tolist() == [[3, 4], [3, own[0]], [-1, -1] if short else [3, own[1]]]
        assert got[3][3] == (2 if short else 3) and np.array_equal(got[5][own[0]], pool[4])
    # the open page: its contents may be another's, so they are not copied
    got = both_ways(fork_call, dict(pool=pool, table=table, count=count, refs=i32([0, 0, 1, 1, held, 1]), lengths=lengths, source=source),
                    ("table", "count", "refs", "lengths"))
    assert got[0] == B.SEQ_DEV_BAD_SLOT and got[1].tolist() == [[3, 4], [3, 0], [3, 1]] and got[3].tolist() == [1, 1, 1, 3, 0, 1]
    assert np.array_equal(got[5], pool)


def test_fork_of_a_row_that_names_no_page():
    table, count, lengths, source = i32([[6, 2, -7], [-1, -1, -1]]), i32([3, 0]), i32([40, 0]), i32([-1, 0])
    pool = np.arange(6 * 16, dtype=np.uint8).reshape(6, 16)
    got = both_ways(fork_call, dict(pool=pool, table=table, count=count, refs=i32([0, 0, 1, 0, 0, 0]), lengths=lengths, source=source),
                    ("table", "count", "refs", "lengths"))
    assert got[0] == B.SEQ_DEV_BAD_PAGE and got[1].tolist() == [[6, 2, -7], [-1, 2, 0]] and got[2].tolist() == [3, 3]
    assert got[3].tolist() == [1, 0, 2, 0, 0, 0] and got[4].tolist() == [40, 40] and np.array_equal(got[5], pool)
