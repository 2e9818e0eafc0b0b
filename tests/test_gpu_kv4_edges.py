"""seq_tree_kv4_attention where its kernels hand things over: ranges that open or end with a piece of a unit."""
import numpy as np
import pytest
import torch

from paper_2402_12374_b200 import binding as B
from tests import kv4_util as U
from tests import test_gpu_kv4_attention as T
from tests.test_gpu_kv4_attention import Case

pytestmark = pytest.mark.gpu
BOTH = pytest.mark.parametrize("dt", [torch.float16, torch.bfloat16])


@BOTH
@pytest.mark.parametrize("R,seed", [(60, 0), (100, 1), (150, 2)])
def test_ranges_that_open_with_the_last_step_of_a_unit(R, seed, dt):
    """Many ragged units over all SMs: between 9 and 16 of the ranges begin with one step and go on with the next unit.  The two
    groups of threads that share a row of q have channels of different magnitudes, so that each needs what the other found."""
    lengths = np.random.default_rng(seed).integers(100, 700, R)
    c = Case(list(lengths), 20, 8, 2, 16, dt, seed=seed)
    piece = torch.arange(128) // 8 % 2
    size = 2.0 ** torch.randint(-6, 1, (R, 20, 8, 2), generator=torch.Generator().manual_seed(seed))
    c.q = (c.q.float() * size[..., piece]).to(dt)
    out, call = c.check(exact_keys=dt == torch.float16)
    assert call.workspace is not None  # ranges, not clusters
    out, lse = out.clone(), call.lse.clone()
    for _ in range(20):
        assert torch.equal(call.run(), out) and torch.equal(call.lse, lse)


@pytest.fixture(params=["tight", "roomy"])
def room(request, monkeypatch):
    """With room for 40000 tokens no cluster takes the few rows, nor small trees."""
    monkeypatch.setattr(T, "ROOM", 40000 if request.param == "roomy" else 0)


@pytest.mark.parametrize("which", ["k", "v"])
@pytest.mark.parametrize("sign", [1.0, -1.0, 0.0])
@pytest.mark.parametrize("n,Hq,dt", [(6, 2, torch.float16), (6, 2, torch.bfloat16), (14, 1, torch.bfloat16), (40, 4, torch.float16), (40, 4, torch.bfloat16),
                                     (150, 2, torch.float16), (150, 2, torch.bfloat16)])
def test_a_row_of_the_tree_beyond_half_precision(n, Hq, dt, sign, which, room):
    """Keys alone and values alone: whoever sees such a row becomes NaN, whatever the sign of the score it would have; nobody else changes."""
    c = Case([45], n, Hq, 1, 16, dt, seed=8)
    star = np.eye(n, dtype=bool)
    star[:, 0] = True
    star[n - 1, 1] = True  # (a node that sees a bad row of another one)
    c.seen, c.mask = [star], torch.from_numpy(U.mask_words(star)).cuda()
    c.q[..., 5] = sign
    clean = c.call().run().clone()
    assert torch.isfinite(clean).all()
    rows = c.kt if which == "k" else c.vt
    bad = {1: 1e5, 2: float("nan"), 3: float("inf"), n - 2: -float("inf")}  # (1e5: an infinity in half precision)
    for j, x in bad.items():
        rows[0, j, 0, 5] = x
    call = c.call()
    out = call.run()
    assert int(c.status) == 0
    for i in range(n):
        if i in bad or i == n - 1:
            assert torch.isnan(out[0, i]).all() and torch.isnan(call.lse[0, :, i]).all(), i
        else:
            assert torch.equal(out[0, i], clean[0, i]) and torch.isfinite(call.lse[0, :, i]).all(), i


@pytest.mark.parametrize("given", [True, False])
@pytest.mark.parametrize("n,times", [(1, 30), (1, 110), (20, 30)])  # clusters (no workspace), ranges, tiles
def test_memory_of_a_call_on_another_current_stream_is_not_handed_out(n, times, given):
    """What a call owns outlives the call object until the stream of its runs is through, however that stream was chosen."""
    c = Case([300, 20, 411] * times, n, 8, 2, 16, torch.float16, seed=3)
    want = c.call().run().clone()
    call = c.call()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    need, held = call.workspace_bytes_needed, {t.data_ptr() for t in (call.out, call.workspace) if t is not None}
    with torch.cuda.stream(side):
        torch.cuda._sleep(1_000_000_000)
        out = call.run() if not given else None
    if given:
        out = call.run(stream=side.cuda_stream)
    del call
    others = [torch.empty(max(need, 1), dtype=torch.uint8, device="cuda") for _ in range(4)]
    others += [torch.empty_like(out) for _ in range(4)]
    assert (need > 0) == (len(held) == 2) and not held & {t.data_ptr() for t in others}
    side.synchronize()
    assert torch.equal(out, want)


@pytest.mark.parametrize("how", ["current", "given", "function", "out given"])
@pytest.mark.parametrize("n,times", [(1, 110), (20, 30)])
def test_memory_that_a_call_takes_over_is_not_used_before_its_last_user_is_through(n, times, how):
    """out (and the workspace) lie where another tensor was that the stream of the call's making still writes to; the run is elsewhere."""
    c = Case([300, 20, 411] * times, n, 8, 2, 16, torch.float16, seed=3)
    call = c.call()
    want, need = call.run().clone(), call.workspace_bytes_needed
    del call
    q, kt, vt, pool, table = c.q.cuda(), c.kt.cuda(), c.vt.cuda(), c.pool_dev[:, 0], torch.from_numpy(c.table).cuda()
    lengths = torch.tensor(c.lengths, dtype=torch.int32, device="cuda")
    mine = torch.full_like(q, 5.0) if how == "out given" else None
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    before = [torch.empty_like(q), torch.empty(need, dtype=torch.uint8, device="cuda")]
    places = {t.data_ptr() for t in before}
    for t in before:
        t.fill_(0)  # (what is asked for behind the wait has been loaded)
    torch.cuda._sleep(1_000_000_000)
    for t in before:
        t.fill_(77)
    through = torch.cuda.Event()
    through.record()
    del t, before
    kw = dict(mask_bits=c.mask)
    if how in ("current", "given"):
        call = B.KV4AttentionCall(q, kt, vt, pool, table, lengths, **kw)
        assert {call.out.data_ptr(), call.workspace.data_ptr()} & places
        if how == "current":
            with torch.cuda.stream(side):
                out = call.run()
        else:
            out = call.run(stream=side)
    else:
        out = B.seq_tree_kv4_attention(q, kt, vt, pool, table, lengths, out=mine, stream=side, **kw)
        assert mine is not None or out.data_ptr() in places
    side.synchronize()
    assert how != "out given" or not through.query()  # nothing of the call's is that stream's: it did not wait
    torch.cuda.synchronize()
    assert torch.equal(out, want)


@BOTH
@pytest.mark.parametrize("n,Hq", [(1, 8), (14, 1), (40, 4)])
@pytest.mark.parametrize("scale", [1e-45, 1e-38, 1e-30])
def test_a_scale_that_makes_all_scores_alike(scale, n, Hq, dt, room):
    """Hidden keys stay hidden: their -inf is not multiplied by a scale of zero."""
    c = Case([45, 0, 300], n, Hq, 1, 16, dt, seed=3, mask="each")
    c.check(softmax_scale=scale)
    c.check(softmax_scale=scale, window=20, sinks=3)


@pytest.mark.parametrize("n,Hq", [(1, 8), (14, 1), (40, 4)])
@pytest.mark.parametrize("size,scale", [(1e36, 1e-37), (1e30, 1e-31), (1e-28, 1e27)])
def test_rows_of_q_at_the_ends_of_bfloat16s_range(size, scale, n, Hq, room):
    c = Case([45, 300], n, Hq, 1, 16, torch.bfloat16, seed=8, mask="each")
    c.q = (c.q.double() * size).to(torch.bfloat16)
    c.check(softmax_scale=scale)


@BOTH
@pytest.mark.parametrize("n,Hq", [(1, 8), (14, 1), (40, 4), (100, 2)])
@pytest.mark.parametrize("scale", [1e3, 1e7, 1e15, 1e30])
@pytest.mark.parametrize("sign", [1, -1])
def test_scores_far_from_zero(sign, scale, n, Hq, dt, room):
    """One key is so far above the others that it alone counts, and its score is up to 1e33 from zero: a row's own node, whose key is
    larger than all others, or smaller where q is negative."""
    c = Case([0, 33, 700], n, Hq, 1, 16, dt, seed=8, mask="chain")
    for r, L in enumerate(c.lengths):
        for t in range(L):
            U.store(c.pool, c.table[r, t // 16], 0, 0, 16, t, 0, *U.quantise(np.full(128, 8.0)))
    c.pool_dev = torch.from_numpy(c.pool).reshape(c.pool.shape[0], 1, 1, -1).cuda()
    c.q[:] = sign
    i = torch.arange(n).reshape(1, n, 1, 1)
    c.kt[:] = 8.5 + i / 16 if sign > 0 else 7.5 - i / 32  # (exact in both types; steps of 1/32: scores are 4 * scale apart)
    call = c.call(softmax_scale=scale)
    out = call.run()
    torch.cuda.synchronize()
    assert int(c.status) == 0
    # its probability over the sum of itself: P's rounding to half precision and the output's
    v = c.vt.double()
    assert ((out.double().cpu() - v).abs() <= (U.EPS2[dt] + 1.01 * U.HALF) * v.abs() + 2.0 ** -24).all()
    # half a step each: the scale as fp32, log2(e), their product, the score, the logarithm of the sum added, ln(2), the result
    want = 128 * scale * sign * c.kt[:, :, 0, 0].double()[:, None]
    assert ((call.lse.double().cpu() - want).abs() <= 7.01 * 2.0 ** -24 * want.abs()).all()


@pytest.mark.parametrize("n,Hq", [(1, 8), (14, 1), (40, 4)])
def test_the_largest_rows_of_half_precision(n, Hq, room):
    """q, keys and values near the largest half: scores beyond 1e8."""
    c = Case([45, 300], n, Hq, 1, 16, torch.float16, seed=8, mask="each")
    rng = np.random.default_rng(5)
    for r, L in enumerate(c.lengths):
        for t in range(L):
            U.store(c.pool, c.table[r, t // 16], 0, 0, 16, t, 0, *U.quantise(rng.uniform(-6e4, 6e4, 128)))
    c.pool_dev = torch.from_numpy(c.pool).reshape(c.pool.shape[0], 1, 1, -1).cuda()
    c.q, c.kt = (c.q * 1e4).clamp(-6e4, 6e4), (c.kt * 1e4).clamp(-6e4, 6e4)
    out, _ = c.check()
    for r, L in enumerate(c.lengths):  # the key with the largest score, where that is no matter of rounding
        k, v = U.prefix_rows(c.pool, 0, c.table[r], L, 1, 16)
        k, v = torch.cat([torch.as_tensor(k[0]), c.kt[r, :, 0].double()]), torch.cat([torch.as_tensor(v[0]), c.vt[r, :, 0].double()])
        s = torch.einsum("nhc,jc->nhj", c.q[r].double(), k).masked_fill(~torch.cat([torch.ones(n, L, dtype=torch.bool), torch.as_tensor(c.seen[r])], 1)[:, None], -torch.inf)
        top = s.topk(2, -1)
        sure = top.values[..., 0] - top.values[..., 1] > 1e-4 * s.abs().nan_to_num(posinf=0).amax(-1)
        assert sure.double().mean() > 0.9
        got, want = out[r].double().cpu()[sure], v[top.indices[..., 0]][sure]
        assert ((got - want).abs() <= 3 * U.HALF * (want.abs() + 8)).all()  # (out's rounding, and scale * 1's: codes up to 8 scales, |value| + |mid| <= 8)


@BOTH
@pytest.mark.parametrize("L", [200, 300, 420, 560, 700])
def test_last_segments_that_end_with_either_groups_tile(L, dt):
    """A unit a range or nearly so: the group of threads that does not have the last key tile is through before that tile's product, and
    takes the rows' sums and reference as the other one leaves them."""
    c = Case([L] * 30, 40, 8, 2, 16, dt, seed=L)
    c.kt *= 3  # (the tree's tile, the last one, has the largest scores)
    out, call = c.check()
    assert call.workspace is not None
    out, lse = out.clone(), call.lse.clone()
    for _ in range(20):
        assert torch.equal(call.run(), out) and torch.equal(call.lse, lse)


@pytest.mark.parametrize("lengths,n,Hq,Hkv,window,dt,seed", [([-1, 1651], 620, 15, 3, 667, torch.bfloat16, 21), ([1200, 900], 500, 12, 3, 300, torch.float16, 2),
                                                          ([3000], 768, 16, 2, 0, torch.bfloat16, 3), ([3000], 768, 16, 2, 0, torch.float16, 4)])
def test_many_tiles_of_rows_a_range(lengths, n, Hq, Hkv, window, dt, seed):
    """The scores of the next tile of rows are computed, and its buffers go round, while the last one's results are still being written."""
    c = Case(lengths, n, Hq, Hkv, 128, dt, seed=seed, mask="each")
    out, call = c.check(window=window, sinks=3 if window else 0)
    out, lse = out.clone(), call.lse.clone()
    live = [r for r, L in enumerate(lengths) if L >= 0]
    for _ in range(10):
        assert torch.equal(call.run()[live], out[live]) and torch.equal(call.lse[live], lse[live])
    assert int(c.status) == 0
