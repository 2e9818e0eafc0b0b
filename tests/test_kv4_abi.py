"""Host-side checks of the paged 4-bit cache's calls that need no GPU: struct layouts, refusals before anything is launched."""
import ctypes as C
import os
import subprocess

import numpy as np
import pytest
import torch

from paper_2402_12374_b200 import binding as B
from tests import kv4_util as U

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 0x1000  # never dereferenced: validation fails first


@pytest.fixture(scope="module")
def lib():
    from paper_2402_12374_b200 import build

    build.build()
    return B.load()


def test_ctypes_structs_match_the_header(tmp_path):
    structs = (("seq_tree_kv4_attention_params", B.Kv4AttentionParams), ("seq_tree_kv4_append_params", B.Kv4AppendParams),
               ("seq_tree_pages_params", B.PagesParams))
    lines = ['#include <stdio.h>', '#include <stddef.h>', '#include "seq_tree.h"', "int main(void){"]
    want = [B.SEQ_DEV_BAD_PAGE, B.SEQ_DEV_BAD_SLOT, B.SEQ_DEV_NO_PAGES, B.SEQ_KV4_GRANULE_BYTES, B.SEQ_MAX_BATCH, B.SEQ_MAX_SLOTS]
    lines.append('printf("%d %d %d %d %d %d\\n", SEQ_DEV_BAD_PAGE, SEQ_DEV_BAD_SLOT, SEQ_DEV_NO_PAGES, SEQ_KV4_GRANULE_BYTES, SEQ_MAX_BATCH, SEQ_MAX_SLOTS);')
    for name, st in structs:
        lines.append(f'printf("%zu\\n", sizeof({name}));')
        lines += [f'printf("%zu\\n", offsetof({name}, {f[0]}));' for f in st._fields_]
        want += [C.sizeof(st)] + [getattr(st, f[0]).offset for f in st._fields_]
    src = tmp_path / "layout.c"
    src.write_text("\n".join(lines + ["return 0;}"]))
    exe = tmp_path / "layout"
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    assert [int(x) for x in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()] == want


def attention(**kw):
    p = B.Kv4AttentionParams()
    p.batch, p.n_tree, p.max_len, p.num_q_heads, p.num_kv_heads, p.head_dim, p.dtype = 2, 16, 100, 32, 8, 128, B.SEQ_BF16
    p.q = p.k_tree = p.v_tree = p.out = p.pages = p.page_table = p.lengths = p.workspace = FAKE
    p.q_stride_req, p.q_stride_tok, p.q_stride_head = 16 * 4096, 4096, 128
    p.o_stride_req, p.o_stride_tok, p.o_stride_head = 16 * 4096, 4096, 128
    p.t_stride_req, p.t_stride_tok, p.t_stride_head = 16 * 1024, 1024, 128
    p.page_stride_bytes, p.num_pages, p.page_size, p.table_stride, p.max_pages = 8 * 16 * 136, 50, 16, 7, 7
    p.mask_bits, p.mask_words_per_row, p.workspace_bytes = FAKE, 1, 1 << 40
    for k, v in kw.items():
        setattr(p, k, v)
    return p


ROOMY = dict(max_pages=4000, table_stride=4000, max_len=60000)  # more than clusters take


@pytest.mark.parametrize("bad", [dict(q=None), dict(k_tree=None), dict(v_tree=None), dict(pages=None), dict(page_table=None), dict(lengths=None),
                                 dict(out=None), dict(batch=0), dict(batch=1025), dict(n_tree=0), dict(n_tree=1025), dict(max_len=-1), dict(max_len=113),
                                 dict(num_kv_heads=5), dict(num_kv_heads=0), dict(num_q_heads=0), dict(window=-1), dict(sinks=-1), dict(num_pages=0),
                                 dict(max_pages=0), dict(table_stride=6), dict(page_stride_bytes=8 * 16 * 136 - 16), dict(page_stride_bytes=8 * 16 * 136 + 8),
                                 dict(q=FAKE + 2), dict(pages=FAKE + 8), dict(out=FAKE + 4), dict(q_stride_head=129), dict(o_stride_tok=-128),
                                 dict(t_stride_req=4), dict(mask_words_per_row=0), dict(mask_stride_req=-1), dict(softmax_scale=float("nan")),
                                 dict(softmax_scale=float("inf")), dict(workspace=FAKE + 16, **ROOMY)])
def test_attention_refuses(lib, bad):
    assert lib.seq_tree_kv4_attention(C.byref(attention(**bad)), None) == B.SEQ_ERR_INVALID_ARG


@pytest.mark.parametrize("bad", [dict(head_dim=64), dict(dtype=B.SEQ_F32), dict(dtype=9), dict(page_size=8), dict(page_size=48), dict(page_size=256, max_len=0)])
def test_attention_does_not_support(lib, bad):
    assert lib.seq_tree_kv4_attention(C.byref(attention(**bad)), None) == B.SEQ_ERR_UNSUPPORTED


@pytest.mark.parametrize("bad", [dict(o_stride_req=0), dict(o_stride_tok=0), dict(o_stride_head=0)])
def test_attention_refuses_rows_of_out_over_one_another(lib, bad):
    assert lib.seq_tree_kv4_attention(C.byref(attention(**bad)), None) == B.SEQ_ERR_INVALID_ARG


def test_attention_needs_its_workspace(lib):
    for n in (1, 4, 16):  # one tile of rows, two, tensor-core tiles
        need = lib.seq_tree_kv4_attention_workspace_bytes(C.byref(attention(n_tree=n, **ROOMY)))
        for bad in (dict(workspace=None), dict(workspace_bytes=need - 1)):
            assert need > 0 and lib.seq_tree_kv4_attention(C.byref(attention(n_tree=n, **ROOMY, **bad)), None) == B.SEQ_ERR_WORKSPACE
    assert lib.seq_tree_kv4_attention_workspace_bytes(C.byref(attention())) == 0  # clusters
    assert lib.seq_tree_kv4_attention(None, None) == B.SEQ_ERR_INVALID_ARG
    assert lib.seq_tree_kv4_attention_workspace_bytes(None) == 0
    assert lib.seq_tree_kv4_attention_workspace_bytes(C.byref(attention(num_kv_heads=0))) == 0


def rows(**kw):
    p = B.Kv4AppendParams()
    p.num_layers, p.batch, p.n_rows, p.num_kv_heads, p.head_dim, p.dtype = 2, 2, 16, 8, 128, B.SEQ_BF16
    p.k = p.v = p.pages = p.page_table = p.lengths = FAKE
    p.stride_layer, p.stride_req, p.stride_tok, p.stride_head = 1 << 20, 16 * 1024, 1024, 128
    p.page_stride_bytes, p.layer_stride_bytes, p.num_pages, p.page_size = 2 * 8 * 16 * 136, 8 * 16 * 136, 50, 16
    p.table_stride, p.max_pages = 7, 7
    for k, v in kw.items():
        setattr(p, k, v)
    return p


BAD_ROWS = [dict(k=None), dict(v=None), dict(pages=None), dict(page_table=None), dict(num_layers=0), dict(batch=0), dict(batch=1025), dict(n_rows=0),
            dict(n_rows=1 << 21), dict(num_kv_heads=0), dict(num_pages=0), dict(max_pages=0), dict(table_stride=6), dict(page_stride_bytes=100),
            dict(page_stride_bytes=2 * 8 * 16 * 136 + 8), dict(layer_stride_bytes=16), dict(k=FAKE + 2), dict(v=FAKE + 8), dict(pages=FAKE + 4),
            dict(stride_tok=1023), dict(stride_head=-128), dict(max_pages=1 << 27, table_stride=1 << 27)]


@pytest.mark.parametrize("bad", BAD_ROWS)
def test_append_and_read_refuse(lib, bad):
    assert lib.seq_tree_kv4_append(C.byref(rows(**bad)), None) == B.SEQ_ERR_INVALID_ARG
    assert lib.seq_tree_kv4_read(C.byref(rows(**bad)), None) == B.SEQ_ERR_INVALID_ARG


def test_append_and_read_refuse_what_is_not_theirs(lib):
    for bad in (dict(lengths=None), dict(new_lengths=FAKE), dict(path=FAKE, path_stride=15)):
        assert lib.seq_tree_kv4_append(C.byref(rows(**bad)), None) == B.SEQ_ERR_INVALID_ARG
    for bad in (dict(path=FAKE, path_stride=16), dict(new_lengths=FAKE + 16), dict(stride_layer=0), dict(stride_req=0), dict(stride_tok=0), dict(stride_head=0)):
        assert lib.seq_tree_kv4_read(C.byref(rows(**bad)), None) == B.SEQ_ERR_INVALID_ARG
    for bad in (dict(head_dim=96), dict(dtype=B.SEQ_F32), dict(page_size=24)):
        for fn in (lib.seq_tree_kv4_append, lib.seq_tree_kv4_read):
            assert fn(C.byref(rows(**bad)), None) == B.SEQ_ERR_UNSUPPORTED
    assert lib.seq_tree_kv4_append(None, None) == lib.seq_tree_kv4_read(None, None) == B.SEQ_ERR_INVALID_ARG


def pages(**kw):
    p = B.PagesParams()
    p.slots, p.max_pages, p.num_pages, p.page_size = 4, 10, 50, 16
    p.page_table, p.page_count, p.ref_count, p.lengths = FAKE, FAKE + 256, FAKE + 512, FAKE + 768
    p.table_out, p.count_out, p.refs_out, p.lengths_out = p.page_table, p.page_count, p.ref_count, p.lengths
    p.table_stride = p.table_out_stride = 10
    p.tokens, p.source, p.pages, p.workspace = FAKE + 1024, FAKE + 1280, FAKE, FAKE
    p.num_planes, p.page_stride_bytes, p.page_bytes, p.workspace_bytes = 1, 4096, 4096, 1 << 30
    for k, v in kw.items():
        setattr(p, k, v)
    return p


@pytest.mark.parametrize("bad", [dict(page_table=None), dict(page_count=None), dict(ref_count=None), dict(table_out=None), dict(refs_out=None), dict(slots=0),
                                 dict(slots=2049), dict(max_pages=0), dict(num_pages=0), dict(num_pages=1 << 30), dict(table_stride=9),
                                 dict(table_out_stride=9), dict(table_out_stride=11), dict(table_out=FAKE + 8192), dict(refs_out=FAKE + 8192),
                                 dict(max_pages=1 << 29, table_stride=1 << 29, table_out_stride=1 << 29)])
def test_pages_calls_refuse(lib, bad):
    for fn in (lib.seq_tree_pages_resize, lib.seq_tree_pages_fork, lib.seq_tree_pages_compact):
        assert fn(C.byref(pages(**bad)), None) == B.SEQ_ERR_INVALID_ARG


def test_pages_calls_refuse_what_each_needs(lib):
    for bad in (dict(tokens=None), dict(count_out=None), dict(page_size=0), dict(count_out=FAKE + 4096)):
        assert lib.seq_tree_pages_resize(C.byref(pages(**bad)), None) == B.SEQ_ERR_INVALID_ARG
    for bad in (dict(source=None), dict(lengths=None), dict(lengths_out=None), dict(count_out=None), dict(page_size=0), dict(lengths_out=FAKE + 4096)):
        assert lib.seq_tree_pages_fork(C.byref(pages(**bad)), None) == B.SEQ_ERR_INVALID_ARG
    need = lib.seq_tree_pages_workspace_bytes(C.byref(pages()))
    for bad in (dict(workspace=None), dict(workspace_bytes=need - 1)):
        assert lib.seq_tree_pages_resize(C.byref(pages(**bad)), None) == B.SEQ_ERR_WORKSPACE
    for fn in (lib.seq_tree_pages_fork, lib.seq_tree_pages_compact):
        for bad in (dict(pages=None), dict(pages=FAKE + 8), dict(num_planes=0), dict(page_bytes=0), dict(page_bytes=24), dict(page_stride_bytes=4080),
                    dict(page_stride_bytes=4104), dict(num_planes=2, plane_stride_bytes=16), dict(workspace=FAKE + 4),
                    dict(num_planes=1 << 30, plane_stride_bytes=1 << 20, page_stride_bytes=1 << 20, page_bytes=1 << 20)):
            assert fn(C.byref(pages(**bad)), None) == B.SEQ_ERR_INVALID_ARG, bad
        for bad in (dict(workspace=None), dict(workspace_bytes=need - 1)):
            assert fn(C.byref(pages(**bad)), None) == B.SEQ_ERR_WORKSPACE
    for fn in (lib.seq_tree_pages_resize, lib.seq_tree_pages_fork, lib.seq_tree_pages_compact):
        assert fn(None, None) == B.SEQ_ERR_INVALID_ARG
    assert lib.seq_tree_pages_workspace_bytes(None) == 0


def test_the_binding_refuses_tensors_on_the_host_and_shapes_that_do_not_fit():
    pool = torch.zeros((3, 2, 16 * 136), dtype=torch.uint8)
    table, lengths = torch.zeros((1, 2), dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    q, k = torch.zeros((1, 1, 4, 128), dtype=torch.float16), torch.zeros((1, 1, 2, 128), dtype=torch.float16)
    with pytest.raises(ValueError, match="CUDA"):
        B.KV4AttentionCall(q, k, k, pool, table, lengths)
    for args in ((q.float(), k, k, pool, table), (q, k.bfloat16(), k, pool, table), (q, k[..., :1, :], k[..., :1, :], pool, table),
                 (q, k, k, pool.to(torch.int16), table), (q, k, k, pool[..., :100], table), (q, k, k, pool[:, ::2], table),
                 (q, k, k, pool.unsqueeze(1).repeat(1, 2, 1, 1), table), (q, k, k, pool, table.repeat(2, 1))):
        with pytest.raises(ValueError):
            B.KV4AttentionCall(*args, lengths)
    with pytest.raises(ValueError):
        B.seq_tree_kv4_append(k, k, pool, table, torch.zeros(2, dtype=torch.int32))
    with pytest.raises(ValueError):
        B.seq_tree_kv4_append(k, k.transpose(1, 2), pool, table, lengths)
    with pytest.raises(ValueError):
        B.seq_tree_pages_resize(table, torch.zeros(2, dtype=torch.int32), torch.zeros(3, dtype=torch.int32), lengths, 16)


def test_the_plain_forms_agree_with_each_other():
    """What the GPU is held to: rows stored one by one are those of a whole pool, a slot that is forked and freed leaves no trace."""
    rng = np.random.default_rng(0)
    x = rng.standard_normal((20, 2, 128))
    nib, s, m = U.quantise(x)
    pool = np.zeros((3, 1, 2 * 16 * 136), dtype=np.uint8)
    for t in range(20):
        for h in range(2):
            for which in (0, 1):
                U.store(pool, [2, 0][t // 16], 0, h, 16, t, which, nib[t, h], s[t, h], m[t, h])
    k, v = U.prefix_rows(pool, 0, [2, 0], 20, 2, 16)
    want = (s[..., None].astype(float) * (nib.astype(float) - 8) + m[..., None]).transpose(1, 0, 2)
    assert np.array_equal(k, want) and np.array_equal(v, want)
    assert np.array_equal(U.fetch(pool, 0, 0, 1, 16, 18, 1), want[1, 18])
    # a step's rounding is half a code, but for what rounding scale and mid adds
    assert (np.abs(want.transpose(1, 0, 2) - x) <= s[..., None] * 0.5 + 20 * U.HALF * np.abs(x).max(-1, keepdims=True)).all()

    table = np.array([[3, 1], [-1, -1]], dtype=np.int32)
    count, refs, lengths = np.array([2, 0], dtype=np.int32), np.array([0, 1, 0, 1], dtype=np.int32), np.array([20, 0], dtype=np.int32)
    contents = np.arange(4)
    _, t2, c2, r2, _, bad, short = U.fork(contents, table, count, refs, lengths, np.array([-1, 0]), 16)
    assert t2.tolist() == [[3, 1], [3, 0]] and r2.tolist() == [1, 1, 0, 2] and not bad and not short
    t3, c3, r3, _ = U.resize(t2, c2, r2, np.array([-1, 0]), 16)
    assert np.array_equal(t3, table) and np.array_equal(r3, refs) and np.array_equal(c3, count)
    p4, t4, r4, live = U.compact(contents, table, count, refs)
    assert live == 2 and t4.tolist() == [[0, 1], [-1, -1]] and p4[0] == 3 and r4.tolist() == [1, 1, 0, 0]
