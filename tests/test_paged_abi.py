"""Host side of the paged 8-bit cache: layout, sizes and refusals, without a GPU."""
import ctypes as C
import os
import subprocess

import pytest

from paper_2408_01890_b200 import binding as lb
from paper_2408_01890_b200 import build as lbuild

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 1 << 20            # an aligned address: nothing is dereferenced before a refusal


@pytest.fixture(scope="module")
def lib():
    lbuild.build()
    return lb.load()


STRUCTS = [(lb.CPagedLayer, "lisa_paged_layer"), (lb.CPagedLayout, "lisa_paged_layout"), (lb.CPageTable, "lisa_page_table"),
           (lb.PagedRowsArgs, "lisa_paged_rows_args"), (lb.PagedAnchorArgs, "lisa_paged_anchor_args"),
           (lb.PagedSharedArgs, "lisa_paged_shared_args"), (lb.CPages, "lisa_pages")]


def test_ctypes_structs_are_the_headers(tmp_path):
    lines = ['#include <stddef.h>', '#include <stdio.h>', '#include "lisa.h"', "int main(void) {"]
    for cls, name in STRUCTS:
        lines.append('printf("%s %%zu\\n", sizeof(%s));' % (name, name))
        for f in cls._fields_:
            lines.append('printf("%s.%s %%zu %%zu\\n", offsetof(%s, %s), sizeof(((%s*)0)->%s));' % (name, f[0], name, f[0], name, f[0]))
    lines.append('printf("%d %d %d %d %d\\n", LISA_S8, LISA_E4M3, LISA_OP_ANCHOR_PAGED, LISA_OP_SHARED_DECODE_PAGED, LISA_ERR_NO_PAGES);')
    lines.append('printf("%d %d\\n", LISA_PAGE_BLOCK, LISA_MAX_PAGE_ROWS);')
    (tmp_path / "layout.c").write_text("\n".join(lines + ["return 0; }"]))
    subprocess.check_call(["gcc", "-std=c11", "-I", os.path.join(ROOT, "include"), str(tmp_path / "layout.c"), "-o", str(tmp_path / "layout")])
    header = subprocess.check_output([str(tmp_path / "layout")], text=True).split("\n")[:-1]
    binding = []
    for cls, name in STRUCTS:
        binding.append("%s %d" % (name, C.sizeof(cls)))
        binding += ["%s.%s %d %d" % (name, f[0], getattr(cls, f[0]).offset, getattr(cls, f[0]).size) for f in cls._fields_]
    binding.append("%d %d %d %d %d" % (lb.S8, lb.E4M3, lb.OP_ANCHOR_PAGED, lb.OP_SHARED_DECODE_PAGED, lb.ERR_NO_PAGES))
    binding.append("%d %d" % (lb.PAGE_BLOCK, lb.MAX_PAGE_ROWS))
    assert binding == header


def layer(kind=lb.CACHE_STANDARD, dtype=lb.S8, Hkv=8, d=128, r=21, P=64, n_pages=10, pages=FAKE):
    return lb.CPagedLayer(kind, dtype, Hkv, d, r, P, n_pages, 0, pages)


@pytest.mark.parametrize("kind,Hkv,d,r,P", [(0, 8, 128, 0, 64), (0, 1, 32, 0, 16), (1, 40, 128, 21, 16), (1, 3, 64, 1, 128), (1, 1, 32, 32, 16)])
def test_page_layout(lib, kind, Hkv, d, r, P):
    lay = lb.CPagedLayout()
    assert lib.lisa_paged_layout_of(C.byref(layer(kind, lb.E4M3, Hkv, d, r, P)), C.byref(lay)) == lb.OK
    up = lambda n: (n + 127) // 128 * 128
    assert lay.v_offset == up(Hkv * P * (r if kind else d))
    assert lay.scale_offset == lay.v_offset + Hkv * P * d
    assert lay.page_bytes == up(lay.scale_offset + Hkv * P // 16 * 8)


def test_eight_bit_pages_are_half_of_the_bf16_cache(lib):
    """A page's bytes against the bf16 cache of as many positions: half, plus four bytes of scale for every 16 positions, head and half."""
    for kind in (lb.CACHE_STANDARD, lb.CACHE_SHARED):
        lay = lb.CPagedLayout()
        assert lib.lisa_paged_layout_of(C.byref(layer(kind, P=128)), C.byref(lay)) == lb.OK
        k, v = lb.lisa_kvcache_bytes(kind, 1, 8, 128, 128, 21)
        assert 0 <= lay.page_bytes - (k + v) // 2 - 8 * 8 * 8 < 256


BAD_LAYERS = [(dict(kind=2), lb.ERR_INVALID_ARG), (dict(dtype=lb.BF16), lb.ERR_INVALID_ARG), (dict(dtype=4), lb.ERR_INVALID_ARG),
              (dict(Hkv=0), lb.ERR_INVALID_ARG), (dict(Hkv=65), lb.ERR_UNSUPPORTED), (dict(d=48), lb.ERR_UNSUPPORTED), (dict(P=8), lb.ERR_INVALID_ARG),
              (dict(P=48), lb.ERR_INVALID_ARG), (dict(P=256), lb.ERR_INVALID_ARG), (dict(n_pages=0), lb.ERR_INVALID_ARG),
              (dict(kind=1, r=0), lb.ERR_INVALID_ARG), (dict(kind=1, r=33), lb.ERR_UNSUPPORTED)]


@pytest.mark.parametrize("change,status", BAD_LAYERS)
def test_layers_are_checked(lib, change, status):
    bad, lay = layer(**change), lb.CPagedLayout()
    assert lib.lisa_paged_layout_of(C.byref(bad), C.byref(lay)) == status
    a = rows_args(bad)
    assert lib.lisa_paged_append(C.byref(a), None) == status and lib.lisa_paged_read(C.byref(a), None) == status


def tensor(Hkv=8, x=128, n=4, dtype=lb.BF16, ptr=FAKE):
    return lb.Tensor(ptr, dtype, 0, n * Hkv * x, Hkv * x, x)


def table(B=2, max_pages=4, stride=4, pages=FAKE):
    return lb.CPageTable(pages, stride, B, max_pages)


def rows_args(l, **change):
    a = lb.PagedRowsArgs()
    a.struct_size, a.B, a.n, a.layer, a.table = C.sizeof(lb.PagedRowsArgs), 2, 4, C.pointer(l), table()
    a.k_or_kp, a.v = tensor(x=l.r if l.kind == 1 else 128), tensor()
    for k, v in change.items():
        setattr(a, k, v)
    return a


@pytest.mark.parametrize("change", [dict(struct_size=8), dict(B=0), dict(n=0), dict(table=table(B=1)), dict(table=table(pages=None)),
                                    dict(table=table(stride=3)), dict(table=table(max_pages=0)), dict(k_or_kp=tensor(ptr=None)), dict(v=tensor(ptr=FAKE + 8)),
                                    dict(v=tensor(x=126)), dict(k_or_kp=tensor(dtype=lb.F32)), dict(v=tensor(dtype=lb.S8)), dict(first=FAKE + 2),
                                    dict(counts=FAKE + 1), dict(layer=C.pointer(layer(pages=None))), dict(layer=C.pointer(layer(pages=FAKE + 64)))])
def test_rows_are_checked(lib, change):
    a = rows_args(layer(), **change)
    assert lib.lisa_paged_append(C.byref(a), None) == lb.ERR_INVALID_ARG
    assert lib.lisa_paged_read(C.byref(a), None) == lb.ERR_INVALID_ARG


def anchor_args(l, **change):
    a = lb.PagedAnchorArgs()
    a.struct_size, a.B, a.Hq, a.L, a.cache, a.table = C.sizeof(lb.PagedAnchorArgs), 2, 32, 200, C.pointer(l), table()
    a.q, a.o = tensor(32, 128, 1), tensor(32, 128, 1)
    a.workspace, a.workspace_bytes = FAKE, 1 << 40
    for k, v in change.items():
        setattr(a, k, v)
    return a


@pytest.mark.parametrize("change,status", [
    (dict(struct_size=0), lb.ERR_INVALID_ARG), (dict(B=0), lb.ERR_INVALID_ARG), (dict(Hq=20), lb.ERR_INVALID_ARG), (dict(Hq=128), lb.ERR_UNSUPPORTED),
    (dict(L=0), lb.ERR_INVALID_ARG), (dict(L=257), lb.ERR_INVALID_ARG), (dict(cache=C.pointer(layer(kind=1))), lb.ERR_INVALID_ARG),
    (dict(q=tensor(ptr=None)), lb.ERR_INVALID_ARG), (dict(o=tensor(dtype=lb.E4M3)), lb.ERR_INVALID_ARG), (dict(seq_lens=FAKE + 1), lb.ERR_INVALID_ARG),
    (dict(out_scores=FAKE, scores_dtype=lb.S8), lb.ERR_INVALID_ARG), (dict(out_scores=FAKE + 2), lb.ERR_INVALID_ARG),
    (dict(workspace=None), lb.ERR_WORKSPACE), (dict(workspace_bytes=16), lb.ERR_WORKSPACE), (dict(workspace=FAKE + 4), lb.ERR_WORKSPACE),
    (dict(table=table(B=1)), lb.ERR_INVALID_ARG), (dict(B=70000, table=table(B=70000)), lb.ERR_UNSUPPORTED)])
def test_anchor_steps_are_checked(lib, change, status):
    assert lib.lisa_attn_anchor_paged(C.byref(anchor_args(layer(), **change)), None) == status


def test_sizes_beyond_the_largest_are_refused(lib):
    """Sequences of over 2^29 positions, and batches whose blocks of 16 positions are more than a grid has CTAs, before anything is launched."""
    pages = (1 << 29) // 64
    for change in (dict(table=table(max_pages=pages + 1, stride=pages + 1)), dict(B=60000, L=1 << 29, table=table(B=60000, max_pages=pages, stride=pages))):
        assert lib.lisa_attn_anchor_paged(C.byref(anchor_args(layer(), **change)), None) == lb.ERR_UNSUPPORTED
        assert lib.lisa_attn_shared_decode_paged(C.byref(shared_args(layer(kind=1), **change)), None) == lb.ERR_UNSUPPORTED


def shared_args(l, **change):
    a = lb.PagedSharedArgs()
    a.struct_size, a.B, a.Hq, a.L, a.cache, a.table = C.sizeof(lb.PagedSharedArgs), 2, 32, 200, C.pointer(l), table()
    a.prev_scores, a.prev_stride_b, a.prev_stride_h = FAKE, 32 * 200, 200
    a.link = lb.CLink(tensor(32, 21, 1), lb.Tensor(), FAKE, None, FAKE, None, lb.BF16, 21, 64, lb.ACT_RELU, lb.INTEGRATE_ADD, 2)
    a.o = tensor(32, 128, 1)
    a.workspace, a.workspace_bytes = FAKE, 1 << 40
    for k, v in change.items():
        setattr(a, k, v)
    return a


def link(**change):
    l = shared_args(layer(kind=1)).link
    for k, v in change.items():
        setattr(l, k, v)
    return l


@pytest.mark.parametrize("change,status", [
    (dict(struct_size=0), lb.ERR_INVALID_ARG), (dict(cache=C.pointer(layer())), lb.ERR_INVALID_ARG), (dict(L=257), lb.ERR_INVALID_ARG),
    (dict(prev_scores=None), lb.ERR_INVALID_ARG), (dict(prev_scores=FAKE + 2), lb.ERR_INVALID_ARG), (dict(scores_dtype=2), lb.ERR_INVALID_ARG),
    (dict(out_scores=FAKE), lb.ERR_INVALID_ARG), (dict(link=link(r=20)), lb.ERR_INVALID_ARG), (dict(link=link(m=257)), lb.ERR_UNSUPPORTED),
    (dict(link=link(w1=None)), lb.ERR_INVALID_ARG), (dict(link=link(w2=None)), lb.ERR_INVALID_ARG), (dict(link=link(integrate=3)), lb.ERR_INVALID_ARG),
    (dict(link=link(ffn_layers=1)), lb.ERR_INVALID_ARG), (dict(o=tensor(ptr=FAKE + 4)), lb.ERR_INVALID_ARG), (dict(workspace_bytes=100), lb.ERR_WORKSPACE)])
def test_shared_steps_are_checked(lib, change, status):
    assert lib.lisa_attn_shared_decode_paged(C.byref(shared_args(layer(kind=1), **change)), None) == status


def pages(**change):
    p = lb.CPages(C.sizeof(lb.CPages), 4, 8, 10, 64, 8, FAKE, FAKE, FAKE, FAKE, 1 << 30)
    for k, v in change.items():
        setattr(p, k, v)
    return p


def test_bookkeeping_is_checked(lib):
    layers = (lb.CPagedLayer * 2)(layer(), layer(kind=1))
    fork = lambda p, parent=FAKE: lib.lisa_pages_fork(C.byref(p), parent, None)
    both = lambda p, l=layers, n=2: {lib.lisa_pages_reserve(C.byref(p), l, n, None, None), lib.lisa_pages_compact(C.byref(p), l, n, None)}
    for change in (dict(struct_size=0), dict(B=0), dict(max_pages=0), dict(n_pages=0), dict(page_tokens=24), dict(table=None), dict(lens=None),
                   dict(refs=FAKE + 2), dict(table_stride=7)):
        assert fork(pages(**change)) == lb.ERR_INVALID_ARG and both(pages(**change)) == {lb.ERR_INVALID_ARG}
    assert fork(pages(B=1025)) == lb.ERR_UNSUPPORTED and both(pages(B=1025)) == {lb.ERR_UNSUPPORTED}
    assert fork(pages(), None) == lb.ERR_INVALID_ARG
    assert both(pages(work=None)) == {lb.ERR_WORKSPACE} and both(pages(work_bytes=64)) == {lb.ERR_WORKSPACE}
    assert both(pages(), n=0) == {lb.ERR_INVALID_ARG} and both(pages(), n=129) == {lb.ERR_INVALID_ARG}
    assert both(pages(n_pages=11)) == {lb.ERR_INVALID_ARG} and both(pages(page_tokens=32)) == {lb.ERR_INVALID_ARG}
    assert lib.lisa_pages_reserve(C.byref(pages()), layers, 2, FAKE + 1, None) == lb.ERR_INVALID_ARG
    mixed = (lb.CPagedLayer * 2)(layer(), layer(P=16))
    assert lib.lisa_pages_copy(mixed, 2, FAKE, FAKE, 1, None) == lb.ERR_INVALID_ARG
    assert lib.lisa_pages_copy(layers, 2, FAKE, FAKE, 0, None) == lb.ERR_INVALID_ARG
    assert lib.lisa_pages_copy(layers, 2, None, FAKE, 1, None) == lb.ERR_INVALID_ARG
    n = C.c_size_t()
    assert lib.lisa_pages_work_bytes(C.byref(pages(B=0)), C.byref(n)) == lb.ERR_INVALID_ARG
    assert lib.lisa_pages_work_bytes(C.byref(pages()), C.byref(n)) == lb.OK and n.value >= 3 * 10 * 4


def test_a_workspace_for_the_largest_step_serves_every_smaller_one(lib):
    def need(op, B, L, Hq, Hkv, d):
        l = layer(kind=int(op == lb.OP_SHARED_DECODE_PAGED), Hkv=Hkv, d=d)
        a = (shared_args if op == lb.OP_SHARED_DECODE_PAGED else anchor_args)(l, B=B, L=L, Hq=Hq)
        n = C.c_size_t()
        assert lib.lisa_workspace_bytes(op, C.byref(a), C.byref(n)) == lb.OK
        return n.value
    for op in (lb.OP_ANCHOR_PAGED, lb.OP_SHARED_DECODE_PAGED):
        for Hq, Hkv, d in ((32, 32, 128), (32, 8, 128), (40, 40, 128), (64, 1, 32), (7, 7, 64)):
            for small, large in (((1, 1), (1, 2)), ((1, 1000), (2, 1000)), ((1, 70000), (64, 70000)), ((3, 129), (500, 4096))):
                assert 0 < need(op, *small, Hq, Hkv, d) <= need(op, *large, Hq, Hkv, d)
        a = (shared_args if op == lb.OP_SHARED_DECODE_PAGED else anchor_args)(layer(kind=int(op == lb.OP_SHARED_DECODE_PAGED)))
        a.L = 0
        assert lib.lisa_workspace_bytes(op, C.byref(a), C.byref(C.c_size_t())) == lb.ERR_INVALID_ARG
