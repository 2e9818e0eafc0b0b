"""Plain 64-bit forms of the paged 4-bit cache's operators, on the CPU, for the tests.  Nothing here shares code with the library."""
from __future__ import annotations

import numpy as np
import torch

D = 128
EPS2 = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}  # half a step of the type, relative
HALF = 2.0 ** -11


def quantise(x):
    """float64 [..., 128] -> (nibbles [..., 128], scale, mid [...]) after the definition; rows that are not finite in half: zeros."""
    x = np.asarray(x, dtype=np.float64)
    with np.errstate(invalid="ignore", over="ignore", divide="ignore"):
        lo, hi = x.min(-1), x.max(-1)
        scale = ((hi - lo) / 15).astype(np.float32).astype(np.float16)
        mid = (lo + 8 * scale.astype(np.float64)).astype(np.float32).astype(np.float16)
        s, m = scale.astype(np.float64)[..., None], mid.astype(np.float64)[..., None]
        code = np.where(s > 0, np.clip(np.rint((x - m) / s), -8, 7), 0.0)
        bad = ~(np.abs(x) <= 65504).all(-1)
    zero = np.float16(0)
    return np.where(bad[..., None], 8, code + 8).astype(np.uint8), np.where(bad, zero, scale), np.where(bad, zero, mid)


def place(page_size, heads, head, token):
    """Byte offsets inside a page (one layer) of a token's parts: K codes, V codes, K params, V params."""
    t = token % page_size
    base = head * page_size * 136 + t // 16 * 2176
    return base + t % 16 * 64, base + 1024 + t % 16 * 64, base + 2048 + t % 16 * 4, base + 2112 + t % 16 * 4


def store(pool, page, layer, head, page_size, token, which, nib, scale, mid):
    """pool: numpy uint8 [pages, layers, heads * page_size * 136]"""
    at = place(page_size, 0, head, token)
    row = pool[page, layer]
    row[at[which]:at[which] + 64] = nib[0::2] | (nib[1::2] << 4)
    row[at[2 + which]:at[2 + which] + 4] = np.array([scale, mid], dtype=np.float16).view(np.uint8)


def fetch(pool, page, layer, head, page_size, token, which):
    at = place(page_size, 0, head, token)
    row = pool[page, layer]
    c = row[at[which]:at[which] + 64]
    nib = np.stack([c & 15, c >> 4], -1).reshape(D).astype(np.float64)
    s, m = row[at[2 + which]:at[2 + which] + 4].view(np.float16).astype(np.float64)
    return s * (nib - 8) + m


def random_pool(pages, layers, heads, page_size, rng, offset=0.7):
    """Quantised normal rows, numpy uint8 [pages, layers, heads * page_size * 136]."""
    g = page_size // 16
    x = rng.standard_normal((pages, layers, heads, g, 2, 16, D)) + offset * rng.standard_normal((heads, 1, 2, 1, D))
    nib, scale, mid = quantise(x)
    codes = (nib[..., 0::2] | (nib[..., 1::2] << 4)).reshape(pages, layers, heads, g, 2048)
    params = np.stack([scale, mid], -1).view(np.uint8).reshape(pages, layers, heads, g, 128)
    return np.concatenate([codes, params], -1).reshape(pages, layers, heads * page_size * 136)


def prefix_rows(pool, layer, table_row, length, heads, page_size):
    """K, V float64 [heads, length, 128]"""
    k, v = np.zeros((heads, length, D)), np.zeros((heads, length, D))
    for p in range(-(-length // page_size)):
        page = pool[table_row[p], layer].reshape(heads, page_size // 16, 2176)
        m = min(page_size, length - p * page_size)
        for which, out in ((0, k), (1, v)):
            c = page[:, :, 1024 * which:1024 * (which + 1)].reshape(heads, page_size, 64)
            nib = np.stack([c & 15, c >> 4], -1).reshape(heads, page_size, D).astype(np.float64)
            sm = np.ascontiguousarray(page[:, :, 2048 + 64 * which:2112 + 64 * which]).view(np.float16).reshape(heads, page_size, 2).astype(np.float64)
            out[:, p * page_size:p * page_size + m] = (sm[..., :1] * (nib - 8) + sm[..., 1:])[:, :m]
    return k, v


def tree(n, rng, wide=6):
    """A random parent array; ancestor matrix [n, n] bool."""
    parent = np.array([-1] + [max(0, i - 1 - int(rng.integers(0, wide))) for i in range(1, n)], dtype=np.int32)
    return parent, ancestors(parent)


def ancestors(parent):
    n = len(parent)
    seen = np.zeros((n, n), dtype=bool)
    for i in range(n):
        j = i
        while j >= 0:
            seen[i, j] = True
            j = parent[j]
    return seen


def mask_words(seen):
    n = seen.shape[-1]
    bits = np.zeros((*seen.shape[:-1], (n + 31) // 32 * 32), dtype=np.uint8)
    bits[..., :n] = seen
    return np.packbits(bits, axis=-1, bitorder="little").view(np.int32)


def attention(q, kt, vt, k, v, seen, scale=None, window=0, sinks=0):
    """One request in 64 bits.  q [n, Hq, 128], kt, vt [n, Hkv, 128], k, v [Hkv, L, 128]; returns out, lse [Hq, n], and what bounds the
    rounding: sum p |v| [n, Hq, 128] and sqrt(sum (q k)^2) * scale, its maximum over the row's keys [n, Hq]."""
    q, kt, vt, k, v = (torch.as_tensor(x).double() for x in (q, kt, vt, k, v))
    n, Hq, _ = q.shape
    Hkv, L, _ = k.shape
    G = Hq // Hkv
    scale = D ** -0.5 if scale is None else scale
    depth = torch.as_tensor(seen.sum(1) - 1)
    where = torch.cat([torch.arange(L), L + depth])
    vis = torch.cat([torch.ones(n, L, dtype=torch.bool), torch.as_tensor(seen)], 1)
    if window:
        vis &= (where[None] > (L + depth)[:, None] - window) | (where[None] < sinks)
    out, lse = torch.zeros(n, Hq, D, dtype=torch.float64), torch.zeros(Hq, n, dtype=torch.float64)
    spread, noise = torch.zeros_like(out), torch.zeros(n, Hq, dtype=torch.float64)
    for h in range(Hq):
        kk, vv = torch.cat([k[h // G], kt[:, h // G]]), torch.cat([v[h // G], vt[:, h // G]])
        s = (q[:, h] @ kk.T * scale).masked_fill(~vis, -torch.inf)
        lse[h] = torch.logsumexp(s, 1)
        p = torch.exp(s - lse[h][:, None])
        gone = ~vis.any(0)
        vv = vv.masked_fill(gone[:, None], 0.0)
        out[:, h], spread[:, h] = p @ vv, p @ vv.abs()
        w = ((q[:, h] ** 2) @ (kk ** 2).T).sqrt() * scale
        noise[:, h] = w.masked_fill(~vis, 0.0).amax(1)
    return out, lse, spread, noise


def check_attention(got, got_lse, ref, dt, exact_keys):
    """Roundings: the output's, half a step; V's and P's to half precision; a key's value to half precision in 128 channels
    (independent: four standard deviations of a uniform error) where codes are not used exactly.  A score that is off by d
    changes a probability by d and the sum by as much.  fp32 sums and ex2.approx: 2e-5.  With exact_keys the scores (lse shows them) have no
    term for the keys.  The output keeps it: where codes enter exactly, what is rounded is a probability times a scale, which is
    off by half a step of |scale * code| <= |v| + |mid|, not of |v|."""
    out, lse, spread, noise = ref
    rounded = 4 / 3 ** 0.5 * HALF * noise
    score = 2e-5 + (0.0 if exact_keys else 1.0) * rounded
    tol = EPS2[dt] * out.abs() + spread * (2 * HALF + 2 * (2e-5 + rounded)[..., None]) + 1e-7
    err = (got.double().cpu() - out).abs()
    assert torch.isfinite(got.float()).all()
    worst = (err / tol).max().item()
    assert worst <= 1, f"output off by {worst:.3g} of what rounding explains (max abs {err.max().item():.3g})"
    if got_lse is not None:
        lerr = (got_lse.double().cpu() - lse).abs()
        assert (lerr <= score.T + 2e-6 * lse.abs() + 2e-5).all(), f"lse off by {lerr.max().item():.3g}"


# ---------------------------------------------------------------- pages
def resize(table, count, refs, tokens, page_size):
    """The definition, slot by slot; returns (table, count, refs, no_pages)."""
    table, count, refs = table.copy(), count.copy(), refs.copy()
    slots, most = table.shape
    want = [count[r] if tokens[r] < 0 or -(-int(tokens[r]) // page_size) > most else -(-int(tokens[r]) // page_size) for r in range(slots)]
    for r in range(slots):
        for i in range(want[r], count[r]):
            refs[table[r, i]] -= 1
            table[r, i] = -1
    free = [p for p in range(len(refs)) if refs[p] <= 0]
    needed, short = 0, False
    old = count.copy()
    for r in range(slots):
        grow = want[r] - old[r]
        if grow <= 0:
            count[r] = want[r]
            continue
        pages = free[needed:needed + grow]
        needed += grow
        if needed > len(free):
            short = True
            continue
        for j, p in enumerate(pages):
            table[r, old[r] + j], refs[p] = p, 1
        count[r] = want[r]
    return table, count, refs, short


def fork(pool, table, count, refs, lengths, source, page_size):
    """Returns (pool, table, count, refs, lengths, bad_slot, no_pages)."""
    pool, table, count, refs, lengths = pool.copy(), table.copy(), count.copy(), refs.copy(), lengths.copy()
    t0, c0, l0 = table.copy(), count.copy(), lengths.copy()
    free = [p for p in range(len(refs)) if refs[p] <= 0]
    bad = short = False
    taken = 0
    for r, s in enumerate(source):
        if s < 0:
            continue
        if s >= len(source) or s == r or c0[r] != 0 or l0[s] < 0 or -(-int(l0[s]) // page_size) > c0[s]:
            bad = True
            continue
        full, rest = divmod(int(l0[s]), page_size)
        if rest:
            taken += 1
            if taken > len(free):
                short = True
                continue
        for i in range(full):
            table[r, i] = t0[s, i]
            refs[t0[s, i]] += 1
        if rest:
            p = free[taken - 1]
            pool[p] = pool[t0[s, full]]
            table[r, full], refs[p] = p, 1
        count[r], lengths[r] = full + bool(rest), l0[s]
    return pool, table, count, refs, lengths, bad, short


def compact(pool, table, count, refs):
    pool, table, refs = pool.copy(), table.copy(), refs.copy()
    live = int((refs > 0).sum())
    holes = [p for p in range(live) if refs[p] <= 0]
    far = [p for p in range(live, len(refs)) if refs[p] > 0]
    to = np.arange(len(refs))
    for p, q in zip(far, holes):
        pool[q], refs[q], refs[p], to[p] = pool[p], refs[p], 0, q
    for r in range(len(count)):
        table[r, :count[r]] = to[table[r, :count[r]]]
    return pool, table, refs, live
