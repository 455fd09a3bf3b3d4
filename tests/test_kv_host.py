"""Paged key / value cache: what holds on the host, without a device."""
import glob
import itertools
import os
import re

import pytest

import paper_2601_17702_b200 as S
from paper_2601_17702_b200 import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_overlapped_kernels_read_through_the_constant_path_only_what_no_launch_writes():
    """A kernel that starts before the one in front of it ends must not read that one's results as read-only memory."""
    found = 0
    for path in glob.glob(os.path.join(ROOT, "paper_2601_17702_b200", "csrc", "*")):
        text = re.sub(r"//.*", "", open(path).read())
        if "cudaGridDependencySynchronize" not in text and "launch_overlapped" not in text:
            continue
        found += 1
        assert "ld.global.nc" not in text and "__restrict__" not in text, path
        for arg in re.findall(r"__ldg\((.*?)[;,]", text):
            assert "cosv" in arg or "sinv" in arg, f"{os.path.basename(path)}: __ldg({arg}"
    assert found >= 5


def test_plans_cover_the_batch():
    """Items hold every new token, thread blocks no more than run at a time, and masks only where a word per 32 blocks is kept."""
    seen = set()
    for sms, (H, K), P, s in itertools.product((1, 148), ((8, 8), (32, 8), (28, 4), (20, 1), (128, 1)), (16, 128), (0, 6, 60)):
        for n, q, kv in itertools.product((1, 3, 40), (1, 5, 70, 1300), (0, 50, 1000, 9000, 200000)):
            p = S.s3_attn_plan_describe(n, n * q, q, kv, H, K, 128, P, sms, s=s)
            assert p.blocks >= 1 and p.blocks <= (1 if p.tile else 2) * sms
            assert p.items * p.tokens_per_item >= n * q and p.items >= (n * q if s and not p.masked else n)
            rows = p.tokens_per_item * (H // K)
            assert p.tokens_per_item >= 1 and rows <= (256 if p.tile else 16)
            assert p.tile or not p.masked
            assert not p.masked or (s > 0 and -(-kv // P) <= 128 * 32)
            assert not p.whole_rounds or (kv * K * 512 > 7e7 and p.shares and p.tile and n == 1 and p.whole_rounds * p.blocks <= p.items * K)
            seen.add((p.tile, p.masked, p.shares, rows > 128))
    assert {(0, 0, 0, False), (0, 0, 1, False), (1, 0, 0, False), (1, 0, 1, True), (1, 1, 0, False), (1, 1, 1, True)} <= seen


@pytest.mark.parametrize("change,code", [
    (dict(n_heads=9), B.S3_ERR_INVALID_ARG), (dict(n_heads=0), B.S3_ERR_INVALID_ARG), (dict(n_heads=1032), B.S3_ERR_UNSUPPORTED),
    (dict(n_kv_heads=0), B.S3_ERR_INVALID_ARG), (dict(page_size=48), B.S3_ERR_UNSUPPORTED), (dict(head_dim=96), B.S3_ERR_UNSUPPORTED), (dict(s=513), B.S3_ERR_UNSUPPORTED),
    (dict(s=-1), B.S3_ERR_INVALID_ARG), (dict(n_sms=0), B.S3_ERR_INVALID_ARG), (dict(max_q=3), B.S3_ERR_INVALID_ARG),
    (dict(max_q=0), B.S3_ERR_INVALID_ARG), (dict(max_kv=-1), B.S3_ERR_INVALID_ARG), (dict(n_seqs=0), B.S3_ERR_INVALID_ARG)])
def test_plan_refusals(change, code):
    args = dict(n_seqs=2, T=2, max_q=1, max_kv=100, n_heads=8, n_kv_heads=8, head_dim=64, page_size=64, n_sms=148)
    S.s3_attn_plan_describe(**args)
    with pytest.raises(S.S3Error) as e:
        S.s3_attn_plan_describe(**{**args, **change})
    assert e.value.code == code
    assert B.lib().s3_attn_plan_describe(None, 8, 8, 64, 64, 0, 1, 148, None) == B.S3_ERR_INVALID_ARG


def test_whole_rounds_go_before_shares_only_past_the_cache():
    """One late chunk: in step where its keys and values exceed what the L2 cache holds of them, in shares alone where they do not."""
    rounds = lambda q, kv, H, K, D: S.s3_attn_plan_describe(1, q, q, kv, H, K, D, 64, 148).whole_rounds
    assert [rounds(2048, kv, 32, 8, 128) for kv in (9000, 16384, 20000, 32768)] == [0, 0, 1, 1]
    assert rounds(2700, 11000, 28, 4, 128) == 0 and rounds(2700, 65536, 28, 4, 128) == 2
    assert rounds(2048, 32768, 32, 8, 64) == 0 and rounds(2048, 65536, 32, 8, 64) == 1
    assert rounds(8192, 20000, 32, 8, 128) == 0
