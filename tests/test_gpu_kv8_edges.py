"""The 8-bit cache and shaped scores where their kernels could go wrong: references that move within a row, caps far from the scores, numbers
at the ends of their types, scales that a caller wrote, and what must not matter.

Tolerances as in test_gpu_kv8.py, derived before the first run: eps = 2^-8 (bf16) or 2^-11 (f16), half a unit in the last place. The result is off by at
most eps (|out| + the weighted mean of |v|), taken per element, plus what the scores are off by: their fp32 errors shift a weight by as much of
itself. A score of size x is a sum of 128 products in fp32 and three roundings of it: 2^-21 times the sum of |q_d k_d| scale at most, below 1e-4
for the scores of up to 40 used here (their products' magnitudes add up to no more than 400). Where values are not of ordinary size the 1e-4 is
taken relative to the weighted mean of |v|."""
import math

import pytest
import torch

import kv8_reference as R8
import kv_reference as R
import paper_2601_17702_b200 as S
from test_gpu_kv8 import BF, EPS, HF, Device

pytestmark = pytest.mark.gpu


def mean_of(s, ref):
    """The definition's weighted mean of |v|."""
    held, s.held = s.held, lambda i, h, which: held(i, h, which).abs() if which == "v" else held(i, h, which)
    mean, _ = ref(s)
    s.held = held
    return mean


def close(s, got, ref, slack=1e-4, lse_slack=0.0):
    """Everything relative to the weighted mean of |v|; slack: what the scores may be off by, as they enter a weight."""
    out, lse = (t.double().cpu() for t in got)
    want, want_lse = ref(s)
    mean = mean_of(s, ref)
    assert torch.isfinite(out).all(), f"{int((~torch.isfinite(out)).sum())} not finite"
    off = (out - want).abs()
    bad = off > EPS[s.dtype] * (want.abs() + mean) + slack * mean
    assert not bad.any(), f"{int(bad.sum())} of {bad.numel()} off, worst {float((off / (mean + 1e-300)).max()):.3g} of the mean, at {bad.nonzero()[:3].tolist()}"
    empty = want_lse == -math.inf
    assert torch.equal(lse == -math.inf, empty) and (out[empty] == 0).all()
    off = (lse - want_lse)[~empty].abs() - 2e-5 * want_lse[~empty].abs().clamp(min=1)
    assert (off <= slack + lse_slack).all(), f"lse off by {float((lse - want_lse)[~empty].abs().max()):.3g}"


# ---------------------------------------------------------------------------------------------- references that move within a row
@pytest.mark.parametrize("make", [R.Setup, R8.Setup8])
@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("rows", [17, 100, 300])
@pytest.mark.parametrize("form", [dict(cap=100.0), dict(slopes=True)])
def test_scores_that_rise_within_64_keys(make, dtype, rows, form):
    """In every run of 64 keys the second half scores some 30 higher (base 2: 43) than the first, by tile and row a little differently: a
    reference that the first half's weights were made with moves, and they follow it."""
    s = make([(rows, 900), (rows // 2, 450)], 4, 2, 128, 64, dtype, seed=rows)
    key = s.q[0, 0].float() * 0 + torch.randn(128, generator=s.g)
    key *= (128 / key.square().sum()).sqrt()
    s.q = (key + 0.2 * torch.randn(s.q.shape, generator=s.g)).to(dtype)
    lift = torch.where(torch.arange(64) % 64 < 32, -1.0, 1.0)[None, None, :, None] * key * 1.35
    for i, (_, kv) in enumerate(s.lens):
        for j in range(-(-kv // 64)):
            p, n = int(s.pages[i, j]), min(64, kv - 64 * j)
            k = 0.3 * torch.randn((2, n, 128), generator=s.g) + lift[0, :, :n] * (0.8 + 0.02 * j)
            if make is R8.Setup8:
                code, scale = R8.held8(k)
                s.k8[p, :, :n], s.k_scale[p, :, :n] = code, scale
            else:
                s.k_cache[p, :, :n] = k.to(dtype)
    host = dict(form)
    if form.get("slopes"):
        host["slopes"] = torch.tensor([0.001, 0.01, -0.01, 0.0])
    dev = {k: v.cuda() if torch.is_tensor(v) else v for k, v in host.items()}
    d = Device(s)
    got = S.s3_paged_attention_scored(d.cache, d.batch, d.q, d.ws, want_lse=True, **dev)
    d.fine()
    # a score is off by 2^-21 of 128 * 1.35 * 1.2 scale < 20, a cap of 100 by another 100 * 2^-21, a slope's term (up to 9) by 9 * 2^-22
    close(s, got, lambda s: R8.scored(s, **host))


# ---------------------------------------------------------------------------------------------- caps far from the scores
@pytest.mark.parametrize("make", [R.Setup, R8.Setup8])
@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("cap", [3.0, 1e4, 1e6, 1e9, 1e20])
@pytest.mark.parametrize("rows", [1, 3, 80])
def test_caps_that_change_next_to_nothing(make, dtype, cap, rows):
    """Under a cap far above the scores tanh(z) is next to z: what is lost may count against the score, not against the cap. Some scores of the
    last sequence are beyond the cap of 3, so that a warp meets both forms."""
    s = make([(rows, 600), (rows, 130)], 8, 2, 128, 32, dtype, seed=rows)
    s.q[: s.cu[1]] *= 0.2 if cap == 3.0 else 2.0
    d = Device(s)
    got = S.s3_paged_attention_scored(d.cache, d.batch, d.q, d.ws, cap=cap, want_lse=True)
    d.fine()
    close(s, got, lambda s: R8.scored(s, cap=cap))            # a relative error of tanh of 2^-21 is 2^-21 of scores of up to 30: 1.4e-5


@pytest.mark.parametrize("make", [R.Setup, R8.Setup8])
def test_few_rows_and_many_agree_under_a_large_cap(make):
    """The last row of a chunk and the same row as a step of its own."""
    s = make([(80, 700)], 8, 2, 128, 64, seed=4)
    one = make([(1, 700)], 8, 2, 128, 64, seed=4)
    d, e = Device(s), Device(one)
    for cap in (1e4, 1e7):
        out, lse = S.s3_paged_attention_scored(d.cache, d.batch, d.q, d.ws, cap=cap, want_lse=True)
        e = Device(one)
        e.cache = d.cache
        batch = S.KvBatch(torch.tensor([0, 1], dtype=torch.int32, device="cuda"), d.batch.kv_len, d.batch.pages, 1, 1, 700)
        got, l1 = S.s3_paged_attention_scored(d.cache, batch, d.q[-1:].contiguous(), e.ws, cap=cap, want_lse=True)
        # each is within eps (|out| + mean |v|) of the definition, |out| and the mean below 1.5 here
        assert ((got[0] - out[-1]).abs().float() <= 2 * EPS[s.dtype] * 3.0).all()
        assert ((l1[0] - lse[-1]).abs() <= 4e-5 * lse[-1].abs().clamp(min=1)).all()


# ---------------------------------------------------------------------------------------------- what must not matter
@pytest.mark.parametrize("make", [R.Setup, R8.Setup8])
@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("H,K", [(14, 2), (9, 3), (8, 2)])
@pytest.mark.parametrize("form", [dict(cap=1e3), dict(cap=30.0, window=70), dict(cap=1e3, slopes=True)])
def test_what_does_not_count_changes_no_bit(make, dtype, H, K, form):
    """Page tails of anything against page tails of zeros, and shared memory that another call has left: 7 heads to a group leave two of a tile's
    128 rows unwritten, a group of 3 as well."""
    results = []
    lens = [(40, 333), (90, 90), (1, 7)]
    for outside in (0.0, float("nan"), float("inf")):
        s = make(lens, H, K, 128, 64, dtype, seed=3, outside=outside)
        if outside != 0.0:                                   # many rows of large numbers first, in tiles of their own
            loud = R.Setup([(300, 400)], 8, 2, 128, 64, dtype, seed=1)
            loud.q = loud.q * 100
            e = Device(loud)
            S.s3_paged_attention(e.cache, e.batch, e.q, e.ws)
        d = Device(s)
        dev = dict(form)
        if form.get("slopes"):
            dev["slopes"] = torch.linspace(-0.01, 0.1, H, device="cuda")
        results.append(S.s3_paged_attention_scored(d.cache, d.batch, d.q, d.ws, want_lse=True, **dev))
        d.fine()
    for out, lse in results[1:]:
        assert torch.equal(out, results[0][0]) and torch.equal(lse, results[0][1])
