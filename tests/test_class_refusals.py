"""What the many-class entry points refuse, seen from the C ABI on the host: every refusal comes before any work on a device."""
import ctypes
import math

import pytest

from paper_1708_04801_amd import api

GB = 1 << 30            # addresses that no call gets as far as using


def blocks(rows=4, cols=200, ld=256, ld_exps=4, codes=GB, exps=2 * GB):
    return api._CBlocks(rows, cols, codes, ld, exps, ld_exps)


def matmul(a, b, out=3 * GB, ld=100, dtype=api.F32, ws=None, ws_bytes=0):
    return api.load().wpsgd_block_matmul(ctypes.byref(a), ctypes.byref(b), out, ld, dtype, ws, ws_bytes, None)


@pytest.mark.parametrize("change", [dict(rows=-1), dict(cols=-1), dict(cols=(1 << 31) + 1), dict(ld=255), dict(ld=240), dict(codes=None), dict(exps=None),
                                    dict(codes=GB + 8), dict(exps=GB + 2), dict(ld_exps=1), dict(ld_exps=6), dict(cols=600)])
def test_block_matrices(change):
    assert matmul(blocks(**change), blocks()) == api.INVALID_ARG
    assert matmul(blocks(), blocks(**change)) == api.INVALID_ARG
    m = api._CMatrix(4, 200, GB, 200, api.F32, None, None, None)
    assert api.load().wpsgd_quantize(ctypes.byref(m), None, 4, 0, ctypes.byref(blocks(**change)), None) == api.INVALID_ARG


@pytest.mark.parametrize("change", [dict(out=None), dict(ld=3), dict(dtype=2), dict(out=GB + 2)])
def test_products(change):
    assert matmul(blocks(), blocks(), **change) == api.INVALID_ARG


def test_product_workspace():
    L = api.load()
    need = L.wpsgd_block_matmul_workspace(300, 700, 65536)       # few tiles, a long sum: split
    assert need >= 2 * 300 * 700 * 4 and need % 256 == 0
    a, b = blocks(300, 65536, 65536, 512), blocks(700, 65536, 65536, 512)
    assert matmul(a, b, ld=700) == api.INVALID_ARG
    assert matmul(a, b, ld=700, ws=GB + 64, ws_bytes=need) == api.INVALID_ARG
    assert matmul(a, b, ld=700, ws=GB, ws_bytes=need - 1) == api.WORKSPACE_TOO_SMALL
    assert L.wpsgd_block_matmul_workspace(0, 700, 65536) == L.wpsgd_block_matmul_workspace(8192, 65536, 4096) == L.wpsgd_block_matmul_workspace(1, 9, 0) == 0


def test_quantize():
    L = api.load()

    def call(n=4, transpose=0, out=None, **matrix):
        m = api._CMatrix(*{**dict(m=4, d=200, dense=GB, ld=200, dtype=api.F32, row_ptr=None, col_idx=None, vals=None), **matrix}.values())
        return L.wpsgd_quantize(ctypes.byref(m), None, n, transpose, ctypes.byref(out or blocks()), None)

    assert call(n=5) == call(n=-1) == call(n=3) == api.INVALID_ARG          # more rows than there are; fewer than the result has
    assert call(transpose=1) == api.INVALID_ARG                              # 200 x 4 is asked for
    assert call(dense=GB + 2) == call(ld=199) == call(dtype=5) == call(m=0) == api.INVALID_ARG
    assert call(dense=None, row_ptr=GB, col_idx=GB, vals=GB) == api.UNSUPPORTED
    assert call(n=0, out=blocks(rows=0)) == api.OK                           # nothing to do


def loss(Z=GB, n=4, c=10, ld=10, dtype=api.F32, labels=GB, scale=1.0, out=GB, grad=2 * GB, ld_grad=10):
    return api.load().wpsgd_softmax_loss(Z, n, c, ld, dtype, labels, None, scale, out, grad, ld_grad, None)


@pytest.mark.parametrize("change", [dict(Z=None), dict(n=-1), dict(c=0), dict(ld=9), dict(dtype=3), dict(labels=None), dict(scale=math.nan), dict(scale=math.inf),
                                    dict(out=None), dict(ld_grad=9), dict(Z=GB + 1), dict(grad=GB + 3), dict(Z=GB, grad=GB, ld_grad=12)])
def test_loss(change):
    assert loss(**change) == api.INVALID_ARG


def draw(Z=GB, n=4, c=10, ld=10, dtype=api.F32, u=GB, drawn=GB, **rule):
    r = api._CDrawRule(1.0, 0, 1.0, 0.0)
    for k, v in rule.items():
        setattr(r, k, v)
    return api.load().wpsgd_draw_classes(Z, n, c, ld, dtype, u, ctypes.byref(r), drawn, None, None)


@pytest.mark.parametrize("change", [dict(Z=None), dict(n=-1), dict(c=0), dict(ld=9), dict(dtype=2), dict(u=None), dict(drawn=None), dict(temperature=-0.5),
                                    dict(temperature=math.nan), dict(top_p=math.nan), dict(min_p=1.25), dict(min_p=math.nan), dict(Z=GB + 2)])
def test_draw(change):
    assert draw(**change) == api.INVALID_ARG


def test_draw_limits():
    assert draw(c=(1 << 18) + 1, ld=1 << 19) == api.UNSUPPORTED
    assert draw(n=0) == loss(n=0) == api.OK
    assert api.load().wpsgd_draw_classes(GB, 4, 10, 10, 0, GB, None, GB, None, None) == api.INVALID_ARG


def test_tensor_lists():
    L = api.load()
    t = (api._CTensor * 2)(api._CTensor(GB, GB, 100, api.F32), api._CTensor(GB, None, 5, api.BF16))
    need = L.wpsgd_tensor_list_bytes(t, 2)
    assert need == 256 and L.wpsgd_tensor_list_bytes(None, 0) == 256 and L.wpsgd_tensor_list_bytes(None, 1) == 0 and L.wpsgd_tensor_list_bytes(t, -1) == 0
    out = api._CTensorList()
    make = lambda items, table=GB, n=need, o=out: L.wpsgd_tensor_list_make(items, 2, table, n, ctypes.byref(o) if o is not None else None, None)  # noqa: E731
    assert make(t, table=None) == make(t, table=GB + 8) == make(t, o=None) == api.INVALID_ARG
    assert make(t, n=255) == api.WORKSPACE_TOO_SMALL
    for bad in (api._CTensor(None, GB, 5, api.F32), api._CTensor(GB + 2, GB, 5, api.F32), api._CTensor(GB, GB + 1, 5, api.F32), api._CTensor(GB, GB, -1, api.F32),
                api._CTensor(GB, GB, 5, 9)):
        assert make((api._CTensor * 2)(t[0], bad)) == api.INVALID_ARG
    listed = api._CTensorList(GB, 1, 100, 1)
    p = ctypes.byref(listed)
    ws = L.wpsgd_grad_norm_workspace(p)
    for args in ((None, GB, GB, ws), (p, None, GB, ws), (p, GB, None, ws), (p, GB, GB + 8, ws)):
        assert L.wpsgd_grad_norm(*args, None) == api.INVALID_ARG
    assert L.wpsgd_grad_norm(p, GB, GB, ws - 1, None) == api.WORKSPACE_TOO_SMALL
    step = lambda eta=0.1, lam=0.1, most=1.0, q=p: L.wpsgd_clipped_step(q, eta, lam, most, GB, GB, ws, None)  # noqa: E731
    assert step(eta=0.0) == step(eta=math.inf) == step(eta=math.nan) == step(lam=-1.0) == step(eta=10.0) == step(most=0.0) == step(most=math.nan) == api.INVALID_ARG
    assert step(q=ctypes.byref(api._CTensorList(GB, 1, 100, 0))) == api.INVALID_ARG         # no weights
    assert L.wpsgd_clip_grads(p, 0.0, GB, GB, ws, None) == L.wpsgd_clip_grads(p, math.nan, GB, GB, ws, None) == api.INVALID_ARG
