"""What the operators of a served layer refuse before anything is launched: by the arguments alone, without a GPU."""
import ctypes as C
import os
import subprocess

import pytest

from paper_2609_09800_b200 import build as hbf_build, hbf

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def lib():
    hbf_build.build()
    return hbf.lib()


def attention(**kw):
    a = hbf.hbf_attention_t()
    a.kv.n_pages, a.kv.page_tokens, a.kv.kv_heads, a.kv.head_dim = 8, 16, 2, 128
    a.kv.k, a.kv.v = 4096, 8192
    a.kv.page_stride, a.kv.slot_stride, a.kv.head_stride = 16 * 256, 256, 128
    a.batch, a.q_heads, a.prefix_len, a.max_own_len, a.own_pages_stride, a.scale = 3, 8, 40, 33, 3, 0.1
    a.prefix_pages, a.own_pages, a.own_len, a.q, a.out = 256, 512, 1024, 16384, 32768
    a.q_row_stride, a.q_head_stride, a.out_row_stride, a.out_head_stride = 1024, 128, 1024, 128
    for k, v in kw.items():
        setattr(a.kv if k in dict(hbf.hbf_kv_t._fields_) else a, k, v)
    return a


@pytest.mark.parametrize("kw", [dict(head_dim=96), dict(head_dim=0), dict(page_tokens=0), dict(n_pages=0), dict(kv_heads=0), dict(kv_heads=3), dict(dtype=2),
                                dict(q_heads=0), dict(scale=float("nan")), dict(scale=float("inf")), dict(prefix_len=(1 << 30) + 1), dict(max_own_len=1 << 31),
                                dict(page_stride=12), dict(slot_stride=-8), dict(head_stride=4), dict(k=0), dict(v=8), dict(prefix_pages=0), dict(own_pages=0), dict(own_len=0),
                                dict(own_len=2), dict(own_pages_stride=2), dict(q=0), dict(q=8), dict(out=0), dict(out=24), dict(q_row_stride=1022), dict(q_head_stride=4),
                                dict(out_row_stride=4), dict(out_head_stride=4), dict(lse=2), dict(batch=70000)])
def test_attention(lib, kw):
    a = attention(**kw)
    assert lib.hbf_prefix_attention(C.byref(a), 256, 1 << 30, None) == hbf.E_INVAL


def test_attention_of_nobody_is_done(lib):
    a = attention(batch=0, q=0, out=0)
    assert lib.hbf_prefix_attention(C.byref(a), None, 0, None) == hbf.OK
    assert lib.hbf_prefix_attention(None, None, 0, None) == hbf.E_INVAL
    assert lib.hbf_attention_workspace_bytes(None) == 0 and lib.hbf_attention_access_count(None) == 0


def test_attention_records(lib):
    a = attention()
    n = lib.hbf_attention_access_count(C.byref(a))
    assert n == 2 * (3 + 3 * 3)
    f = lib.hbf_attention_accesses
    assert f(C.byref(a), 0, 0, 64, n - 1, None) == hbf.E_INVAL and f(C.byref(a), -1, 0, 64, n, None) == hbf.E_INVAL
    assert f(C.byref(a), 0, -1, 64, n, None) == hbf.E_INVAL and f(C.byref(a), 0, 0, None, n, None) == hbf.E_INVAL
    a = attention(slot_stride=512)                            # pages with holes
    assert f(C.byref(a), 0, 0, 64, n, None) == hbf.E_INVAL
    a = attention(prefix_len=0, max_own_len=0, prefix_pages=0, own_pages=0, own_len=0)
    assert lib.hbf_attention_access_count(C.byref(a)) == 0 and f(C.byref(a), 0, 0, None, 0, None) == hbf.OK


def moe(**kw):
    m = hbf.hbf_moe_t()
    m.tokens, m.hidden, m.inter, m.n_experts, m.top_k, m.renormalise = 5, 64, 32, 8, 2, 1
    m.x, m.x_stride, m.scores, m.scores_stride, m.experts, m.expert_stride, m.out, m.out_stride = 4096, 64, 8192, 8, 16384, 3 * 64 * 32, 32768, 64
    for k, v in kw.items():
        setattr(m, k, v)
    return m


@pytest.mark.parametrize("kw", [dict(tokens=129), dict(hidden=0), dict(hidden=60), dict(inter=0), dict(inter=12), dict(hidden=(1 << 20) + 8), dict(n_experts=0), dict(n_experts=513),
                                dict(top_k=0), dict(top_k=9), dict(n_experts=32, scores_stride=32, top_k=17), dict(dtype=2), dict(renormalise=2), dict(expert_stride=3 * 64 * 32 - 8),
                                dict(expert_stride=3 * 64 * 32 + 4), dict(x=0), dict(x=8), dict(x_stride=56), dict(x_stride=68), dict(scores=0), dict(scores=2),
                                dict(scores_stride=7), dict(experts=0), dict(experts=8), dict(out=0), dict(out=1), dict(out_stride=63)])
def test_moe(lib, kw):
    assert lib.hbf_moe_layer(C.byref(moe(**kw)), 256, 1 << 30, None) == hbf.E_INVAL


def test_moe_workspace_and_records(lib):
    m = moe()
    need = lib.hbf_moe_workspace_bytes(C.byref(m))
    assert need == 5 * 2 * 32 * 4
    assert lib.hbf_moe_layer(C.byref(m), 256, need - 1, None) == hbf.E_WORKSPACE
    assert lib.hbf_moe_layer(C.byref(m), 128, need, None) == hbf.E_WORKSPACE and lib.hbf_moe_layer(C.byref(m), None, need, None) == hbf.E_WORKSPACE
    assert lib.hbf_moe_layer(None, 256, need, None) == hbf.E_INVAL and lib.hbf_moe_workspace_bytes(None) == 0
    assert lib.hbf_moe_layer(C.byref(moe(tokens=0)), None, 0, None) == hbf.OK
    assert lib.hbf_moe_access_count(C.byref(m), 5000) == 8 * 3 and lib.hbf_moe_access_count(C.byref(moe(tokens=1)), 4096) == 2 * 3
    assert lib.hbf_moe_access_count(C.byref(m), 0) == 0
    f = lib.hbf_moe_accesses
    assert f(C.byref(m), 5000, 0, 0, 64, 23, None) == hbf.E_INVAL and f(C.byref(m), 0, 0, 0, 64, 24, None) == hbf.E_INVAL
    assert f(C.byref(m), 5000, -1, 0, 64, 24, None) == hbf.E_INVAL and f(C.byref(m), 5000, 0, 0, None, 24, None) == hbf.E_INVAL
    assert f(C.byref(m), 5000, 0, 0, 12, 24, None) == hbf.E_INVAL


def pages(**kw):
    p = hbf.hbf_pages_t()
    p.base, p.page_bytes, p.page_stride, p.slab_stride = 4096, 64, 64, 640
    p.n_slabs, p.n_pages, p.page_tokens, p.rows, p.table_cols, p.table_stride = 3, 10, 4, 5, 6, 6
    p.refs, p.lens, p.tables = 256, 512, 1024
    for k, v in kw.items():
        setattr(p, k, v)
    return p


BAD_PAGES = [dict(base=0), dict(base=8), dict(page_bytes=0), dict(page_bytes=24), dict(page_stride=48), dict(page_stride=72), dict(slab_stride=624), dict(slab_stride=8),
             dict(n_slabs=0), dict(n_pages=0), dict(n_pages=(1 << 20) + 1, slab_stride=1 << 30), dict(rows=(1 << 20) + 1), dict(page_tokens=0)]
BAD_STATE = [dict(refs=0), dict(refs=2), dict(lens=0), dict(tables=0), dict(table_cols=0), dict(table_stride=5), dict(tables=1026)]


@pytest.mark.parametrize("kw", BAD_PAGES + BAD_STATE)
def test_pages(lib, kw):
    p, big = C.byref(pages(**kw)), 1 << 30
    assert lib.hbf_pages_fork(p, 64, 64, 2, None, 256, big, None) == hbf.E_INVAL
    assert lib.hbf_pages_free(p, 64, 2, None, 256, big, None) == hbf.E_INVAL
    assert lib.hbf_pages_compact(p, None, 256, big, None) == hbf.E_INVAL
    if kw in BAD_PAGES:
        assert lib.hbf_pages_copy(p, 64, 64, 2, None, 256, big, None) == hbf.E_INVAL and lib.hbf_pages_workspace_bytes(p) == 0
        assert lib.hbf_pages_accesses(p, 256, 0, 0, 64, 4, None) == hbf.E_INVAL


def test_pages_lists_and_workspace(lib):
    p, big = C.byref(pages()), 1 << 30
    assert lib.hbf_pages_copy(p, None, 64, 2, None, 256, big, None) == hbf.E_INVAL and lib.hbf_pages_copy(p, 64, 66, 2, None, 256, big, None) == hbf.E_INVAL
    assert lib.hbf_pages_copy(p, 64, 64, 11, None, 256, big, None) == hbf.E_INVAL and lib.hbf_pages_fork(p, 64, 64, 6, None, 256, big, None) == hbf.E_INVAL
    assert lib.hbf_pages_free(p, None, 1, None, 256, big, None) == hbf.E_INVAL and lib.hbf_pages_free(p, 64, 1, 2, 256, big, None) == hbf.E_INVAL
    need = lib.hbf_pages_workspace_bytes(p)
    assert need >= 256 + 4 * 4 * 10
    assert lib.hbf_pages_compact(p, None, 256, need - 1, None) == hbf.E_WORKSPACE and lib.hbf_pages_compact(p, None, 64, need, None) == hbf.E_WORKSPACE
    assert lib.hbf_pages_compact(None, None, 256, need, None) == hbf.E_INVAL
    # pages of all slabs side by side are as good a layout
    assert lib.hbf_pages_workspace_bytes(C.byref(pages(slab_stride=64, page_stride=192))) == need
    assert lib.hbf_pages_workspace_bytes(C.byref(pages(slab_stride=64, page_stride=176))) == 0
    f = lib.hbf_pages_accesses
    assert f(p, None, 0, 0, 64, 4, None) == hbf.E_INVAL and f(p, 256, -1, 0, 64, 4, None) == hbf.E_INVAL and f(p, 256, 0, 0, None, 4, None) == hbf.E_INVAL
    assert f(p, 256, 0, 0, None, 0, None) == hbf.OK


def test_struct_layouts_match_the_header(tmp_path):
    names = ("hbf_kv_t", "hbf_attention_t", "hbf_moe_t", "hbf_pages_t")
    lines = ["printf(\"%%zu\\n\", sizeof(%s));" % n for n in names]
    lines += ["printf(\"%%zu\\n\", offsetof(%s, %s));" % (n, f) for n in names for f, _ in getattr(hbf, n)._fields_]
    src = tmp_path / "layout.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "hbf.h"\nint main(void){\n%s\nreturn 0;}\n' % "\n".join(lines))
    exe = tmp_path / "layout"
    subprocess.check_call(["gcc", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)])
    out = [int(x) for x in subprocess.check_output([str(exe)]).decode().split()]
    want = [C.sizeof(getattr(hbf, n)) for n in names] + [getattr(getattr(hbf, n), f).offset for n in names for f, _ in getattr(hbf, n)._fields_]
    assert out == want
