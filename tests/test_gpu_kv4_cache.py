"""seq_tree_kv4_append and seq_tree_kv4_read against the format's definition."""
import numpy as np
import pytest
import torch

from paper_2402_12374_b200 import binding as B
from tests import kv4_util as U

pytestmark = pytest.mark.gpu


def make(lengths, rows, layers, Hkv, page, dt, seed=0, count=None, path=None, spare=1):
    rng = np.random.default_rng(seed)
    R = len(lengths)
    most = max(1, max(-(-(max(L, 0) + rows) // page) for L in lengths))
    pages = R * most + spare
    table = rng.permutation(pages)[:R * most].reshape(R, most).astype(np.int32)
    pool = rng.integers(0, 256, (pages, layers, Hkv * page * 136), dtype=np.uint8)
    g = torch.Generator().manual_seed(seed)
    k, v = (torch.randn(layers, R, rows, Hkv, 128, generator=g).mul_(2.0).to(dt) for _ in range(2))
    return table, pool, k, v


def expect(pool, table, k, v, lengths, count, path, page):
    pool = pool.copy()
    layers, R, rows, Hkv, _ = k.shape
    for r in range(R):
        if lengths[r] < 0:
            continue
        for i in range(count[r]):
            t, node = lengths[r] + i, i if path is None else path[r][i]
            for which, x in ((0, k), (1, v)):
                nib, s, m = U.quantise(x[:, r, node].double().numpy())
                for l in range(layers):
                    for h in range(Hkv):
                        U.store(pool, table[r, t // page], l, h, page, t, which, nib[l, h], s[l, h], m[l, h])
    return pool


def run(pool, table, k, v, lengths, page, count=None, path=None):
    layers, R, rows, Hkv, _ = k.shape
    dev = torch.from_numpy(pool).reshape(pool.shape[0], layers, Hkv, page * 136).cuda()
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    new = torch.full((R,), -9, dtype=torch.int32, device="cuda")
    i32 = lambda x: None if x is None else torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    B.seq_tree_kv4_append(k.cuda(), v.cuda(), dev, torch.from_numpy(table).cuda(), i32(lengths), count=i32(count), path=i32(path), new_lengths=new,
                          dev_status=status)
    return dev.reshape(pool.shape).cpu().numpy(), new.tolist(), int(status), dev


BOTH = pytest.mark.parametrize("dt", [torch.float16, torch.bfloat16])


@BOTH
@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("lengths,rows,layers,Hkv", [([0], 1, 1, 1), ([5, 0, 15], 3, 2, 3), ([100], 40, 1, 8), ([31, 16], 17, 3, 9)])
def test_every_byte_of_the_pool(lengths, rows, layers, Hkv, page, dt):
    table, pool, k, v = make(lengths, rows, layers, Hkv, page, dt, seed=rows)
    got, new, status, _ = run(pool, table, k, v, lengths, page)
    assert status == 0 and new == [L + rows for L in lengths]
    assert np.array_equal(got, expect(pool, table, k, v, lengths, [rows] * len(lengths), None, page))


@BOTH
def test_counts_paths_and_idle_slots(dt):
    lengths, count = [7, 30, -1, 0, 64], [3, 0, 5, 20, 1]
    rows, page = 20, 16
    rng = np.random.default_rng(0)
    path = [list(rng.integers(0, rows, rows)) for _ in lengths]  # any order, repeats
    path[0][3:] = [10 ** 6] * (rows - 3)                         # what lies behind the count is not looked at
    table, pool, k, v = make(lengths, rows, 2, 4, page, dt)
    for p in (None, path):
        got, new, status, _ = run(pool, table, k, v, lengths, page, count, p)
        assert status == 0 and new == [10, 30, -1, 20, 65]
        assert np.array_equal(got, expect(pool, table, k, v, lengths, count, p, page))


@BOTH
def test_rows_that_are_hard_to_round(dt):
    """Constant rows, rows with a large mean, exact middles between codes, tiny and large magnitudes, negative zeros."""
    rows = []
    rng = np.random.default_rng(1)
    rows.append(np.zeros(128))
    rows.append(np.full(128, -0.0))
    rows.append(np.full(128, 3.25))
    rows.append(np.full(128, 65504.0 if dt == torch.float16 else 65280.0))
    rows.append(np.where(np.arange(128) % 2, -65504.0 if dt == torch.float16 else -65280.0, 65504.0 if dt == torch.float16 else 65280.0))
    rows.append(np.arange(128) % 31 / 2.0)                # every half step between 0 and 15
    rows.append((np.arange(128) % 31 / 2.0 - 7) * 2.0 ** -9)
    rows.append(rng.standard_normal(128) * 1e-7)
    rows.append(rng.standard_normal(128) * 1e-4)
    rows.append(1000 + rng.standard_normal(128))
    rows.append(2000.0 + np.arange(128) % 4)              # the mid's rounding is several codes
    rows.append(-30000.0 - 16 * (np.arange(128) % 3))
    rows.append(rng.standard_normal(128) * 2e4 if dt == torch.float16 else rng.standard_normal(128) * 1e4)
    rows += [np.round(rng.standard_normal(128) * 4) / 8 for _ in range(40)]
    x = torch.tensor(np.stack(rows)).to(dt).reshape(1, 1, len(rows), 1, 128)
    table, pool, _, _ = make([3], len(rows), 1, 1, 16, dt)
    got, _, status, _ = run(pool, table, x, x.flip(2), [3], 16)
    assert status == 0
    assert np.array_equal(got, expect(pool, table, x, x.flip(2), [3], [len(rows)], None, 16))


@pytest.mark.parametrize("x", [float("nan"), float("inf"), -float("inf"), 1e30])
def test_rows_that_are_not_finite_are_zeros(x):
    table, pool, k, v = make([3], 6, 1, 2, 16, torch.bfloat16)
    k[0, 0, 2, 1, 127] = x
    v[0, 0, 5, 0, 0] = x
    got, new, status, _ = run(pool, table, k, v, [3], 16)
    assert status == B.SEQ_DEV_NONFINITE and new == [9]
    assert np.array_equal(got, expect(pool, table, k, v, [3], [6], None, 16))
    assert (U.fetch(got, table[0, 0], 0, 1, 16, 5, 0) == 0).all()


def test_bad_requests_are_left_alone():
    lengths = [7, 8, 9]
    table, pool, k, v = make(lengths, 6, 1, 2, 16, torch.float16)
    path = [[0, 1, 2, 3, 4, 5]] * 3
    for count, p, bit in (([2, 7, 1], None, B.SEQ_DEV_BAD_PATH), ([2, -1, 1], None, B.SEQ_DEV_BAD_PATH),
                          ([2, 3, 1], [path[0], [0, 6, 1, 0, 0, 0], path[0]], B.SEQ_DEV_BAD_PATH),
                          ([2, 3, 1], [path[0], [0, 1, -1, 0, 0, 0], path[0]], B.SEQ_DEV_BAD_PATH)):
        got, new, status, _ = run(pool, table, k, v, lengths, 16, count, p)
        assert status == bit and new == [9, 8, 10]
        assert np.array_equal(got, expect(pool, table, k, v, lengths, [2, 0, 1], p, 16))
    reach = table.shape[1] * 16
    got, new, status, _ = run(pool, table, k, v, [7, reach - 2, 9], 16, [2, 3, 1])
    assert status == B.SEQ_DEV_BAD_LENGTH and new == [9, reach - 2, 10]
    assert np.array_equal(got, expect(pool, table, k, v, lengths, [2, 0, 1], None, 16))
    table, pool, k, v = make([7, 12, 9], 6, 1, 2, 16, torch.float16)  # (a table of two pages each)
    bad = table.copy()
    bad[1, 0] = pool.shape[0]
    got, new, status, _ = run(pool, bad, k, v, [7, 12, 9], 16, [2, 6, 1])  # tokens 12..15 have no page, 16, 17 do
    assert status == B.SEQ_DEV_BAD_PAGE and new == [9, 18, 10]
    want = expect(pool, table, k, v, [7, 12, 9], [2, 6, 1], None, 16)
    want[table[1, 0]] = pool[table[1, 0]]
    assert np.array_equal(got, want)


@BOTH
@pytest.mark.parametrize("page", [16, 64])
def test_read_gives_what_is_stored_rounded_once(page, dt):
    lengths, rows = [5, 40, 0], 33
    table, pool, k, v = make(lengths, rows, 2, 3, page, dt)
    got, _, _, dev = run(pool, table, k, v, lengths, page)
    ko, vo = (torch.full((2, 3, rows, 3, 128), 9.0, dtype=dt, device="cuda") for _ in range(2))
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    start, count = torch.tensor([5, -1, 3], dtype=torch.int32, device="cuda"), torch.tensor([33, 20, 7], dtype=torch.int32, device="cuda")
    B.seq_tree_kv4_read(dev, torch.from_numpy(table).cuda(), ko, vo, start=start, count=count, dev_status=status)
    assert int(status) == 0
    for which, o in ((0, ko.cpu()), (1, vo.cpu())):
        want = torch.full_like(o, 9.0)
        for r, s, m in ((0, 5, 33), (2, 3, 7)):
            for i in range(m):
                for l in range(2):
                    for h in range(3):
                        x = U.fetch(got, table[r, (s + i) // page], l, h, page, s + i, which)
                        want[l, r, i, h] = torch.tensor(x).float().to(dt)
        assert torch.equal(o, want)


def test_read_without_start_and_its_refusals():
    table, pool, k, v = make([0], 20, 1, 2, 16, torch.float16)
    got, _, _, dev = run(pool, table, k, v, [0], 16)
    ko, vo = torch.zeros_like(k[0]).cuda(), torch.zeros_like(v[0]).cuda()
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    B.seq_tree_kv4_read(dev, torch.from_numpy(table).cuda(), ko, vo, dev_status=status)
    assert int(status) == 0
    # half a code step: the row's width / 15 / 2, and half a step of its scale and mid, of which codes are up to 8
    width = (k[0].float().amax(-1) - k[0].float().amin(-1))[..., None]
    tol = width / 30 * (1 + 1e-2) + 20 * U.HALF * k[0].float().abs().amax(-1, keepdim=True)
    assert ((ko.float().cpu() - k[0].float()).abs() <= tol).all()
    far = table.copy()
    far[0, 1] = -7
    ko.fill_(9)
    B.seq_tree_kv4_read(dev, torch.from_numpy(far).cuda(), ko, vo, dev_status=status)
    assert int(status) == B.SEQ_DEV_BAD_PAGE and (ko[0, 16:] == 9).all() and not (ko[0, :16] == 9).any()


def test_strided_rows():
    lengths, rows = [3, 14], 5
    table, pool, k, v = make(lengths, rows, 2, 2, 16, torch.float16)
    big = torch.full((2, 2, rows + 1, 2, 2, 2, 136), float("nan"), dtype=torch.float16)
    ks, vs = big[:, :, :rows, :, 0, 1, 8:], big[:, :, :rows, :, 1, 1, 8:]
    ks.copy_(k), vs.copy_(v)
    bigd = big.cuda()
    dev = torch.from_numpy(pool).reshape(pool.shape[0], 2, 2, 16 * 136).cuda()
    B.seq_tree_kv4_append(bigd[:, :, :rows, :, 0, 1, 8:], bigd[:, :, :rows, :, 1, 1, 8:], dev, torch.from_numpy(table).cuda(),
                          torch.tensor(lengths, dtype=torch.int32, device="cuda"))
    assert np.array_equal(dev.reshape(pool.shape).cpu().numpy(), expect(pool, table, k, v, lengths, [rows] * 2, None, 16))


def test_appended_rows_that_are_already_codes_keep_their_values():
    """What the format can represent is stored without loss: reading, appending and reading again changes nothing."""
    table, pool, k, v = make([0], 64, 1, 4, 16, torch.float16, seed=3)
    nib = np.random.default_rng(0).integers(0, 16, (64, 4, 128))
    nib[..., 0], nib[..., 1] = 0, 15
    x = torch.tensor((nib - 8) * 0.125 + 0.5).to(torch.float16)[None, None]
    _, _, status, dev = run(pool, table, x, x, [0], 16)
    ko, vo = torch.zeros_like(x[0]).cuda(), torch.zeros_like(x[0]).cuda()
    B.seq_tree_kv4_read(dev, torch.from_numpy(table).cuda(), ko, vo)
    assert status == 0 and torch.equal(ko.cpu(), x[0]) and torch.equal(vo.cpu(), x[0])
