"""What the entry points for training on answers, dropout and four bits refuse, seen from the C ABI on the host: every refusal comes before any work on a device."""
import ctypes
import math

import pytest

from paper_1708_04801_amd import api

GB = 1 << 30            # addresses that no call gets as far as using


def policy(Z=GB, n=4, c=10, ld=10, dtype=api.F32, drawn=GB, old=GB, ref=GB, advantage=GB, weights=None, low=0.2, high=0.2, kl=0.1, scale=1.0, loss=GB, log_prob=GB,
           grad=2 * GB, ld_grad=10):
    return api.load().wpsgd_policy_loss(Z, n, c, ld, dtype, drawn, old, ref, advantage, weights, low, high, kl, scale, loss, log_prob, grad, ld_grad, None)


@pytest.mark.parametrize("change", [dict(Z=None), dict(n=-1), dict(n=1 << 31), dict(c=0), dict(c=1 << 31, ld=1 << 31), dict(ld=9), dict(dtype=3), dict(drawn=None), dict(ref=None), dict(advantage=None),
                                    dict(loss=None), dict(ld_grad=9), dict(Z=GB + 1), dict(grad=GB + 3), dict(Z=GB, grad=GB, ld_grad=12), dict(low=-0.1), dict(low=1.1),
                                    dict(low=math.nan), dict(high=-0.1), dict(high=math.nan), dict(kl=-0.1), dict(kl=math.inf), dict(kl=math.nan), dict(scale=math.inf),
                                    dict(scale=math.nan), dict(n=0, kl=-1.0)])
def test_policy(change):
    assert policy(**change) == api.INVALID_ARG


def test_policy_without_rows():
    assert policy(n=0, Z=None, drawn=None, loss=None) == api.OK


def preference(Z=GB, n=8, c=3000, ld=3000, dtype=api.F32, labels=GB, offsets=GB, pairs=2, ref=None, weights=None, pair_weights=None, kind=api.HINGE, beta=0.1, eps=0.0, scale=1.0,
               loss=GB, margin=GB, grad=2 * GB, ld_grad=3000, ws=GB, ws_bytes=None):
    L = api.load()
    need = L.wpsgd_preference_loss_workspace(n, c, pairs, dtype) if ws_bytes is None else ws_bytes
    return L.wpsgd_preference_loss(Z, n, c, ld, dtype, labels, offsets, pairs, ref, weights, pair_weights, kind, beta, eps, scale, loss, margin, grad, ld_grad, ws, need, None)


@pytest.mark.parametrize("change", [dict(Z=None), dict(n=-1), dict(c=0), dict(ld=2999), dict(dtype=2), dict(labels=None), dict(offsets=None), dict(pairs=-1), dict(kind=2),
                                    dict(beta=math.inf), dict(beta=math.nan), dict(eps=-0.1), dict(eps=1.5), dict(eps=math.nan), dict(scale=math.nan), dict(loss=None),
                                    dict(margin=None), dict(ld_grad=2999), dict(Z=GB + 2), dict(grad=GB + 2), dict(Z=GB, grad=GB, ld_grad=3016), dict(ws=None), dict(ws=GB + 128)])
def test_preference(change):
    assert preference(**change) == api.INVALID_ARG


def test_preference_workspace():
    L = api.load()
    need = L.wpsgd_preference_loss_workspace(1000, 3000, 20, api.F32)
    assert need >= 20000 and need % 256 == 0
    assert preference(n=1000, pairs=20, ws_bytes=need - 1) == api.WORKSPACE_TOO_SMALL
    # none for pairs that a workgroup forms by itself: up to 1024 classes in fp32, 2048 in bfloat16, 256 rows, 32 rows a pair on average
    one = lambda n, c, pairs, dtype: L.wpsgd_preference_loss_workspace(n, c, pairs, dtype) == 0  # noqa: E731
    assert one(0, 3000, 1, api.F32) and one(-1, 3000, 1, api.F32) and one(256, 1024, 8, api.F32) and one(256, 2048, 8, api.BF16) and one(32, 1, 1, api.F32)
    assert not (one(256, 1025, 8, api.F32) or one(256, 2049, 8, api.BF16) or one(257, 1024, 17, api.F32) or one(256, 1024, 7, api.F32) or one(1, 8, 0, api.F32))
    assert preference(n=0, pairs=0, Z=None, labels=None, loss=None, margin=None, ws=None) == api.OK


def matrix(**change):
    return api._CMatrix(*{**dict(m=4, d=200, dense=GB, ld=200, dtype=api.F32, row_ptr=None, col_idx=None, vals=None), **change}.values())


SPARSE = dict(dense=None, row_ptr=GB, col_idx=GB, vals=GB)
BAD_MATRICES = [dict(dense=GB + 2), dict(ld=199), dict(dtype=5), dict(m=0), dict(d=0)]


def dropout(rows=None, n=4, p=0.5, seed=1, chain=0, step=0, out=2 * GB, ld=200, **m):
    return api.load().wpsgd_dropout(ctypes.byref(matrix(**m)), rows, n, p, seed, chain, step, None, out, ld, None)


@pytest.mark.parametrize("change", [dict(n=5), dict(n=-1), dict(n=1 << 32, rows=GB), dict(p=-0.1), dict(p=1.5), dict(p=math.nan), dict(chain=-1), dict(step=-1), dict(out=None),
                                    dict(out=GB + 2), dict(ld=199), dict(out=GB, rows=GB), dict(out=GB, ld=208)] + BAD_MATRICES)
def test_dropout(change):
    assert dropout(**change) == api.INVALID_ARG


def test_dropout_of_sparse_rows_and_of_none():
    assert dropout(**SPARSE) == api.UNSUPPORTED
    assert dropout(n=0, out=None) == api.OK


def nibbles(rows=4, cols=200, group=64, codes=GB, ld=128, scales=2 * GB, ld_scales=8):
    return api._CNibbles(rows, cols, group, codes, ld, scales, ld_scales)


BAD_NIBBLES = [dict(rows=-1), dict(cols=-1), dict(cols=(1 << 31) + 1), dict(group=16), dict(group=0), dict(group=256), dict(codes=None), dict(scales=None), dict(codes=GB + 8),
               dict(scales=GB + 8), dict(ld=112), dict(ld=130), dict(ld_scales=4), dict(ld_scales=12), dict(cols=300)]


def quantize4(out=None, rows=None, n=4, **m):
    return api.load().wpsgd_quantize_nibbles(ctypes.byref(matrix(**m)), rows, n, ctypes.byref(nibbles(**(out or {}))), None)


def matmul4(W=None, rows=None, n=4, out=3 * GB, ld_out=4, out_dtype=api.F32, **m):
    return api.load().wpsgd_nibble_matmul(ctypes.byref(matrix(**m)), rows, n, ctypes.byref(nibbles(**(W or {}))), out, ld_out, out_dtype, None)


@pytest.mark.parametrize("change", BAD_NIBBLES)
def test_four_bit_matrices(change):
    assert quantize4(out=change) == matmul4(W=change) == api.INVALID_ARG


@pytest.mark.parametrize("change", BAD_MATRICES + [dict(n=5), dict(n=-1), dict(d=199)])
def test_rows_for_four_bits(change):
    assert quantize4(**change) == matmul4(**change) == api.INVALID_ARG


def test_quantize4_and_products():
    assert quantize4(out=dict(rows=5)) == quantize4(out=dict(rows=3)) == api.INVALID_ARG
    assert quantize4(**SPARSE) == matmul4(**SPARSE) == api.UNSUPPORTED
    for change in (dict(out=None), dict(ld_out=3), dict(out_dtype=2), dict(out=GB + 2), dict(n=1 << 31, rows=GB)):
        assert matmul4(**change) == api.INVALID_ARG
    assert quantize4(n=0, out=dict(rows=0)) == matmul4(n=0) == matmul4(W=dict(rows=0)) == api.OK
    L = api.load()
    assert L.wpsgd_quantize_nibbles(ctypes.byref(matrix()), None, 4, None, None) == L.wpsgd_nibble_matmul(ctypes.byref(matrix()), None, 4, None, GB, 4, 0, None) == api.INVALID_ARG
    assert L.wpsgd_quantize_nibbles(None, None, 4, ctypes.byref(nibbles()), None) == L.wpsgd_dropout(None, None, 1, 0.5, 0, 0, 0, None, GB, 8, None) == api.INVALID_ARG
