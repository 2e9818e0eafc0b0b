"""The paged cache next to the calls that its own are made for: masks from parents, attention, verification of a batch, append."""
import numpy as np
import pytest
import torch

from paper_2402_12374_b200 import binding as B
from tests import kv4_util as U

pytestmark = pytest.mark.gpu


def stored(x):
    """Rows [m, heads, 128] as the pages hold them, float64 [heads, m, 128]."""
    nib, s, m = U.quantise(x.double().numpy())
    return (s[..., None].astype(float) * (nib.astype(float) - 8) + m[..., None]).transpose(1, 0, 2)


@pytest.mark.parametrize("dt", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("n,Hq,heads,one_tree", [(7, 4, 2, False), (24, 8, 2, True), (40, 4, 1, False)])
def test_steps_of_a_batch(n, Hq, heads, one_tree, dt):
    """Prompts, then steps of three requests and an idle slot: the library's own mask words (a common tree's, or each request's), the tree's
    attention in every layer, the walk, and the accepted paths into the pages.  One request's walk is given up: no token, path length 0."""
    R, layers, page, V, most = 4, 2, 16, 64, 12
    g = torch.Generator(device="cuda").manual_seed(n)
    rng = np.random.default_rng(n)
    i32 = dict(dtype=torch.int32, device="cuda")
    st = torch.zeros(1, **i32)
    table, count, refs = torch.full((R, most), -1, **i32), torch.zeros(R, **i32), torch.zeros(R * most, **i32)
    pool = torch.full((R * most, layers, heads, page * 136), 0xFF, dtype=torch.uint8, device="cuda")
    have = torch.tensor([37, 5, 0, 16], **i32)
    lengths, after = torch.zeros(R, **i32), torch.zeros(R, **i32)
    randn = lambda *shape: torch.randn(shape, device="cuda", generator=g).to(dt)  # noqa: E731
    k, v = randn(layers, R, 37, heads, 128), randn(layers, R, 37, heads, 128)
    B.seq_tree_pages_resize(table, count, refs, have, page, dev_status=st)
    B.seq_tree_kv4_append(k, v, pool, table, lengths, count=have, new_lengths=after, dev_status=st)
    assert int(st) == 0 and torch.equal(after, have)
    lengths.copy_(after)
    lengths[2] = -1
    rows = [[[x[l, r, :int(have[r])].cpu() for x in (k, v)] for l in range(layers)] for r in range(R)]
    for step in range(4):
        parents = [U.tree(n, rng)[0] for _ in range(R)]
        if one_tree:
            parents = parents[:1] * R
        seen = [U.ancestors(p) for p in parents]
        parent = torch.from_numpy(np.stack(parents)).cuda()
        words = [B.seq_tree_mask_from_parents(parent[r], dev_status=st)[0] for r in range(1 if one_tree else R)]
        mask = words[0] if one_tree else torch.stack(words)
        q, k, v = randn(layers, R, n, Hq, 128), randn(layers, R, n, heads, 128), randn(layers, R, n, heads, 128)
        grown = torch.where(lengths < 0, lengths, lengths + n)
        B.seq_tree_pages_resize(table, count, refs, grown, page, dev_status=st)
        before = lengths.tolist()
        window = 20 if step % 2 else 0
        for l in range(layers):
            out = B.seq_tree_kv4_attention(q[l], k[l], v[l], pool[:, l], table, lengths, mask_bits=mask, window=window, sinks=2, dev_status=st)
            for r in (0, 1, 3):
                kk, vv = (stored(x) for x in rows[r][l])
                assert kk.shape[1] == before[r]
                U.check_attention(out[r], None, U.attention(q[l, r].cpu(), k[l, r].cpu(), v[l, r].cpu(), kk, vv, seen[r], window=window, sinks=2), dt, False)
        tokens = torch.randint(0, V, (R, n), generator=g, **i32)
        logits, draft = (torch.randn((R, n, V), device="cuda", generator=g) for _ in range(2))
        path, path_len, _ = B.seq_tree_verify_batch(parent, tokens, logits, draft, 1.0, torch.rand((R, n + 1), device="cuda", generator=g), dev_status=st)
        assert path_len.min() >= 1
        path_len[step % 2] = 0  # (what a walk leaves whose wait ran out)
        B.seq_tree_kv4_append(k, v, pool, table, lengths, count=path_len, path=path, new_lengths=after, dev_status=st)
        lengths.copy_(after)
        assert int(st) == 0
        for r in (0, 1, 3):
            nodes = path[r, :int(path_len[r])].long().cpu()
            for l in range(layers):
                rows[r][l] = [torch.cat([have_, x[l, r].cpu()[nodes]]) for have_, x in zip(rows[r][l], (k, v))]
        assert lengths.tolist() == [before[r] + (0 if r == 2 else int(path_len[r])) for r in range(R)]
    assert lengths[2] == -1
