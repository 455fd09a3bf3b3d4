"""Paged key / value cache: struct layouts and the argument checks that need no device; the 64-bit definitions against each other."""
import ctypes as C
import math

import pytest
import torch

import kv_reference as R
from paper_2601_17702_b200 import binding as B


def test_struct_layouts_match_header():
    assert C.sizeof(B.KvCacheDesc) == 72
    assert C.sizeof(B.KvBatchDesc) == 48
    assert C.sizeof(B.RopeDesc) == 32
    assert C.sizeof(B.AttnParams) == 16


def desc(**kw):
    d = dict(d_k=256, d_v=512, k_page_stride=2 * 64 * 128, v_page_stride=2 * 64 * 128, d_code=None, d_scale=None, n_pages=4, n_kv_heads=2,
             page_size=64, head_dim=128, dtype=B.S3_BF16, reserved=0)
    d.update(kw)
    return B.KvCacheDesc(*[d[f] for f, _ in B.KvCacheDesc._fields_])


@pytest.mark.parametrize("change,code", [
    (dict(d_k=None), B.S3_ERR_INVALID_ARG), (dict(d_v=520), B.S3_ERR_INVALID_ARG), (dict(d_code=256), B.S3_ERR_INVALID_ARG),
    (dict(dtype=B.S3_F32), B.S3_ERR_UNSUPPORTED), (dict(dtype=7), B.S3_ERR_UNSUPPORTED), (dict(head_dim=96), B.S3_ERR_UNSUPPORTED),
    (dict(page_size=48), B.S3_ERR_UNSUPPORTED), (dict(n_pages=0), B.S3_ERR_INVALID_ARG), (dict(n_kv_heads=0), B.S3_ERR_INVALID_ARG),
    (dict(k_page_stride=64), B.S3_ERR_INVALID_ARG), (dict(v_page_stride=2 * 64 * 128 + 4), B.S3_ERR_INVALID_ARG),
    (dict(k_page_stride=1 << 40), B.S3_ERR_UNSUPPORTED)])
def test_cache_refusals(change, code):
    h = C.c_void_p()
    assert B.lib().s3_kv_cache_create(C.byref(h), C.byref(desc(**change))) == code
    assert not h.value and B.lib().s3_last_error()


def test_null_arguments():
    lib = B.lib()
    assert lib.s3_kv_cache_create(None, None) == B.S3_ERR_INVALID_ARG
    h = C.c_void_p()
    assert lib.s3_kv_cache_create(C.byref(h), None) == B.S3_ERR_INVALID_ARG
    assert lib.s3_kv_cache_destroy(None) == B.S3_OK
    assert lib.s3_kv_workspace_bytes(None, None, 4) == 0
    assert lib.s3_kv_append(None, None, None, None, None, 0, 0, None, 0, None, 0, None, 0, None, 0, None) == B.S3_ERR_INVALID_ARG
    assert lib.s3_block_select(None, None, None, 0, 0, 0, 0, 0, None, None, 0, None) == B.S3_ERR_INVALID_ARG
    assert lib.s3_paged_attention(None, None, None, 0, 0, None, None, 0, None, None, 0, None) == B.S3_ERR_INVALID_ARG
    assert lib.s3_block_attention(None, None, None, 0, 0, None, 0, 0, 0, None, None, 0, None, None, 0, None) == B.S3_ERR_INVALID_ARG


def test_reference_attention_over_all_blocks_is_attention():
    s = R.Setup([(3, 40), (1, 1)], 4, 2, 64, 16, outside=0.0)
    lists = torch.arange(4, dtype=torch.int32).view(1, 1, 4).expand(s.T, 1, 4)
    a, la = R.attention(s)
    b, lb = R.attention(s, blocks=lists)
    assert torch.equal(a, b) and torch.equal(la, lb)
    # the softmax definition by hand for one row
    k, v = s.held(0, 1, "k")[:38], s.held(0, 1, "v")[:38]
    x = [sum(float(k[j, d]) * float(s.q[0, 2, d]) for d in range(64)) / 8 for j in range(38)]
    w = [math.exp(y - max(x)) for y in x]
    want = sum(w[j] * v[j] for j in range(38)) / sum(w)
    assert torch.allclose(a[0, 2], want, atol=1e-12)


def test_reference_selection_takes_forced_blocks_and_ties():
    s = R.Setup([(1, 100)], 2, 1, 64, 16, outside=0.0)
    code = torch.zeros((s.n_pages, 1, 64), dtype=torch.int8)
    lists = R.select(s, code, torch.ones((s.n_pages, 1)), 4, 1, 1)
    assert lists[0, 0].tolist() == [0, 1, 2, 6]
