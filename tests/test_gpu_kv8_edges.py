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


def close(s, got, ref, slack=1e-4, lse_slack=0.0, lost=0.0):
    """Everything relative to the weighted mean of |v|; slack: what the scores may be off by, as they enter a weight; lost: relative to the row's
    largest such mean."""
    out, lse = (t.double().cpu() for t in got)
    want, want_lse = ref(s)
    mean = mean_of(s, ref)
    assert torch.isfinite(out).all(), f"{int((~torch.isfinite(out)).sum())} not finite"
    off = (out - want).abs()
    bad = off > EPS[s.dtype] * (want.abs() + mean) + slack * mean + lost * mean.amax(-1, keepdim=True)
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


# ---------------------------------------------------------------------------------------------- numbers at the ends of their types
def along(s, rows, amount):
    """Queries and keys along one direction, so that the products are large: score sign(keys of the block) * amount (before a cap)."""
    key = torch.randn(s.D, generator=s.g)
    key *= (s.D / key.square().sum()).sqrt()
    s.q = (key + 0.05 * torch.randn(s.q.shape, generator=s.g)).to(s.dtype)
    for i, (_, kv) in enumerate(s.lens):
        for j in range(-(-kv // s.P)):
            p, n = int(s.pages[i, j]), min(s.P, kv - s.P * j)
            k = (key * amount(j) / s.D ** 0.5 + 0.1 * torch.randn((s.K, n, s.D), generator=s.g)).to(s.dtype)
            if hasattr(s, "k8"):
                s.k8[p, :, :n], s.k_scale[p, :, :n] = R8.held8(k)
            else:
                s.k_cache[p, :, :n] = k


def values_times(s, factor):
    for p in range(s.n_pages):
        f = factor(p)
        if hasattr(s, "v8"):
            s.v_scale[p] *= f
        else:
            s.v_cache[p] *= f


@pytest.mark.parametrize("make", [R.Setup, R8.Setup8])
@pytest.mark.parametrize("rows,lens", [(1, [(1, 300)]), (70, [(70, 300), (70, 150)]), (300, [(300, 2000)])])
@pytest.mark.parametrize("size", [2.0 ** 56, 2.0 ** -56, 1.0])
@pytest.mark.parametrize("sign", [1, -1, 0])
@pytest.mark.parametrize("cap", [30.0, 50.0])
def test_values_of_any_size_at_either_end_of_the_cap(make, rows, lens, size, sign, cap):
    """All scores next to the cap, all next to its negative, or some blocks here and some there; values of 2^56 (codes times scales of up to
    2^58), of 1, and as small; some pages in between, so that not every thread block meets them."""
    s = make(lens, 8, 2, 128, 64, seed=rows)
    along(s, rows, lambda j: 200.0 * (sign if sign else (1 if j % 3 else -1)))
    values_times(s, lambda p: size)
    d = Device(s)
    got = S.s3_paged_attention_scored(d.cache, d.batch, d.q, d.ws, scale=128 ** -0.5, cap=cap, want_lse=True)
    d.fine()
    # scores of 200 to 300 from products of 128 terms whose magnitudes add up to as much: off by 300 * 2^-21, and less behind the cap
    close(s, got, lambda s: R8.scored(s, scale=128 ** -0.5, cap=cap), slack=3e-4)


@pytest.mark.parametrize("make", [R.Setup, R8.Setup8])
def test_marked_blocks_leave_the_others_alone(make):
    """Large values in one sequence of several: its rows are right, and the others have the bits that they have without it. A replayed graph whose
    values become ordinary, and large again, follows."""
    lens = [(70, 400), (70, 500), (40, 300)]
    s = make(lens, 8, 2, 128, 64, seed=5)
    along(s, 70, lambda j: 100.0 if j % 2 else 20.0)
    d = Device(s)
    run = lambda: S.s3_paged_attention_scored(d.cache, d.batch, d.q, d.ws, cap=50.0, want_lse=True)
    plain = [t.clone() for t in run()]
    big = [int(p) for p in s.pages[1, :8]]
    target, host = (d.vs, s.v_scale) if make is R8.Setup8 else (d.v, s.v_cache)
    keep = target.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            got = run()
    side.synchronize()
    for large in (True, False, True):
        target.copy_(keep)
        if large:
            target[big] *= 2.0 ** 57
        with torch.cuda.stream(side):
            side.wait_stream(torch.cuda.default_stream())
            g.replay()
        side.synchronize()
        for a, b in zip(got, plain):
            assert torch.equal(a[:70], b[:70]) and torch.equal(a[140:], b[140:])
            if not large:
                assert torch.equal(a, b)
        assert torch.isfinite(got[0]).all()
    host[big] *= 2.0 ** 57
    close(s, got, lambda s: R8.scored(s, cap=50.0), slack=3e-4)
    d.fine()


@pytest.mark.parametrize("rows", [1, 100, 300])
@pytest.mark.parametrize("form", [dict(), dict(slopes=True), dict(cap=300.0), dict(cap=50.0)])
@pytest.mark.parametrize("rise", [17.0, 20.0])
def test_large_values_under_scores_that_rise(rows, form, rise):
    """bf16 values of 2^101 (their magnitudes add up to 2^111) over scores that are 17 or 20 higher (base 2: 25, 29) from the third block on than before: the
    weights stay small enough that sums in fp32 hold them."""
    s = R.Setup([(rows, 900), (rows, 500)], 8, 2, 128, 64, seed=rows)
    along(s, rows, lambda j: 10.0 + rise if j >= 2 else 10.0)
    values_times(s, lambda p: 2.0 ** 101)
    host = dict(form)
    if form.get("slopes"):
        host["slopes"] = torch.linspace(0.0, 0.001, 8)
    dev = {k: v.cuda() if torch.is_tensor(v) else v for k, v in host.items()}
    d = Device(s)
    got = S.s3_paged_attention_scored(d.cache, d.batch, d.q, d.ws, scale=128 ** -0.5, want_lse=True, **dev)
    d.fine()
    close(s, got, lambda s: R8.scored(s, scale=128 ** -0.5, **host))


# ---------------------------------------------------------------------------------------------- scales that a caller wrote
@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("lens", [[(1, 300), (1, 17)], [(70, 300), (40, 200)], [(300, 500)]])
@pytest.mark.parametrize("form", [None, dict(cap=20.0), dict(slopes=True)])
@pytest.mark.parametrize("D,P", [(128, 16), (64, 64)])
def test_rows_switched_off_and_turned_over(dtype, lens, form, D, P):
    """A value scale of 0 over codes that are not, negative scales of keys and values, scales below any that an append writes: a row counts for
    code * scale whatever wrote it."""
    s = R8.Setup8(lens, 8, 2, D, P, dtype, seed=len(lens))
    x = torch.randint(0, 8, s.v_scale.shape, generator=s.g)
    s.v_scale[x == 0] = 0.0
    s.v_scale[x == 1] *= -1.0
    s.v_scale[x == 2] = 1e-40
    s.v_scale[x == 3] = -(2.0 ** -75)
    s.k_scale[torch.randint(0, 4, x.shape, generator=s.g) == 0] *= -1.0
    d = Device(s)
    if form is None:
        got, ref = S.s3_paged_attention(d.cache, d.batch, d.q, d.ws, want_lse=True), lambda s: R.attention(s)
    else:
        host = dict(form)
        if form.get("slopes"):
            host["slopes"] = torch.linspace(0.0, 0.1, 8)
        dev = {k: v.cuda() if torch.is_tensor(v) else v for k, v in host.items()}
        got, ref = S.s3_paged_attention_scored(d.cache, d.batch, d.q, d.ws, want_lse=True, **dev), lambda s: R8.scored(s, **host)
    d.fine()
    close(s, got, ref)


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("per_token,q", [(True, 1), (True, 90), (False, 90)])
def test_switched_off_rows_in_lists(dtype, per_token, q):
    s = R8.Setup8([(q, 700)], 8, 2, 128, 64, dtype, seed=q)
    s.v_scale[torch.randint(0, 3, s.v_scale.shape, generator=s.g) == 0] = 0.0
    s.v_scale[torch.randint(0, 3, s.v_scale.shape, generator=s.g) == 0] *= -1.0
    lists = torch.stack([torch.stack([torch.randperm(11, generator=s.g)[:6] for _ in range(2)]) for _ in range(q if per_token else 1)]).to(torch.int32)
    d = Device(s)
    got = S.s3_block_attention(d.cache, d.batch, d.q, lists.cuda(), d.ws, per_token=per_token, want_lse=True)
    d.fine()
    close(s, got, lambda s: R.attention(s, blocks=lists, per_token=per_token))


# ---------------------------------------------------------------------------------------------- values far apart
@pytest.mark.parametrize("dtype,small", [(BF, -50), (BF, -30), (HF, -18)])
@pytest.mark.parametrize("lens", [[(1, 300), (1, 40)], [(70, 300)], [(300, 400)]])
@pytest.mark.parametrize("form", [None, dict(cap=20.0)])
def test_zero_values_beside_small_ones(dtype, small, lens, form):
    """A value of zeros weighs in the sum and nowhere else: small values beside it keep their bits, whatever their size."""
    s = R8.Setup8(lens, 8, 2, 128, 16, dtype, seed=3)
    s.v_scale *= 2.0 ** small
    zero = torch.randint(0, 3, s.v_scale.shape, generator=s.g) == 0
    s.v_scale[zero] = 0.0
    s.v8[zero] = 0
    d = Device(s)
    if form is None:
        got, ref = S.s3_paged_attention(d.cache, d.batch, d.q, d.ws, want_lse=True), lambda s: R.attention(s)
    else:
        got, ref = S.s3_paged_attention_scored(d.cache, d.batch, d.q, d.ws, want_lse=True, **form), lambda s: R8.scored(s, **form)
    d.fine()
    close_small(s, got, ref)


def close_small(s, got, ref):
    """As `close`, with results so small that the type's smallest number counts beside them."""
    out, lse = (t.double().cpu() for t in got)
    want, want_lse = ref(s)
    mean = mean_of(s, ref)
    assert ((out - want).abs() <= EPS[s.dtype] * (want.abs() + mean) + 1e-4 * mean + (2.0 ** -25 if s.dtype == HF else 0.0)).all()
    assert ((lse - want_lse).abs() <= 2e-5 * want_lse.abs().clamp(min=1) + 1e-4).all()


@pytest.mark.parametrize("lens", [[(1, 4000), (1, 900)], [(3, 4000)], [(60, 2000)]])
@pytest.mark.parametrize("order", ["small first", "large first", "mixed"])
@pytest.mark.parametrize("low,sizes", [(3.0, (56, -58)), (-1.0, (60, -59.5))])
def test_values_at_both_ends(lens, order, low, sizes):
    """bf16: most values next to 2^-59, a few next to 2^58, and the many small ones carry most of the weight although each scores lower (base 2:
    10, 16) than the large: what they add to the sum of weights divides the large ones.

    In a dimension where the large values' codes are 0 nothing is left but the small ones, 2^-110 of the row. Few rows: a weight times its value's
    scale is an f16 number, at least 2^7 for the row's largest such product, so a key loses at most half of f16's smallest number, 2^-25,
    hence 2^-32 of that product, times a code of at most 127; 127 times the largest product is no more than the largest mean of |v| over the dimensions
    (its value has a code of 127 in one of them). So 4000 keys lose 4000 * 2^-32 of that mean."""
    s = R8.Setup8(lens, 8, 2, 128, 64, seed=4)
    key = torch.randn(128, generator=s.g)
    key *= (128 / key.square().sum()).sqrt()
    s.q = (key + 0.02 * torch.randn(s.q.shape, generator=s.g)).to(BF)
    for i, (n, kv) in enumerate(s.lens):
        for x in range(kv):
            large = {"small first": x == kv - n - 1, "large first": x == 5, "mixed": x % 997 == 500}[order]
            p = int(s.pages[i, x // 64])
            k = key * ((10.0 if large else low) / 128 ** 0.5) + 0.05 * torch.randn((2, 128), generator=s.g)
            s.k8[p, :, x % 64], s.k_scale[p, :, x % 64] = R8.held8(k)
            v = torch.randn((2, 128), generator=s.g).double()
            if low < 0:
                v /= v.abs().amax(-1, keepdim=True)
            s.v8[p, :, x % 64], s.v_scale[p, :, x % 64] = R8.held8(v * 2.0 ** sizes[0 if large else 1])
    d = Device(s)
    got = S.s3_paged_attention(d.cache, d.batch, d.q, d.ws, scale=128 ** -0.5, want_lse=True)
    d.fine()
    close(s, got, lambda s: R.attention(s, scale=128 ** -0.5), lost=4000 * 2.0 ** -32)


@pytest.mark.parametrize("q", [1, 3, 60])
@pytest.mark.parametrize("scale", [2.0 ** -110, 2.0 ** -85, 2.0 ** 100, 1.0 / 16])
@pytest.mark.parametrize("form", [None, dict(slopes=True), dict(cap=50.0)])
def test_queries_at_both_ends(q, scale, form):
    """bf16 rows of 2^111, 2^83 and 2^-105 under scales that bring their scores back (and others', which are then next to 0): powers of two, so that
    the scores are those of ordinary rows."""
    if form and form.get("cap") and not 1e-30 <= scale / 50.0 <= 1e30:
        scale = 2.0 ** -90                                    # the cap's limits
    s = R8.Setup8([(q, 300)], 8, 2, 128, 16, seed=12)
    s.q = s.q.float().clamp(-2, 2)
    for h, e in ((0, 110), (1, 82), (2, -105), (3, 0), (4, 86)):
        s.q[:, h] *= 2.0 ** e
    s.q = s.q.to(s.dtype)
    host = dict(form or {})
    if host.get("slopes"):
        host["slopes"] = torch.full((8,), 0.01)
    dev = {k: v.cuda() if torch.is_tensor(v) else v for k, v in host.items()}
    d = Device(s)
    out, lse = (t.double().cpu() for t in S.s3_paged_attention_scored(d.cache, d.batch, d.q, d.ws, scale=scale, want_lse=True, **dev))
    d.fine()
    want, want_lse = R8.scored(s, scale=scale, **host)
    ok = want_lse.abs() < 100                                 # rows whose scores are of ordinary size
    assert ok.any()
    mean = mean_of(s, lambda s: R8.scored(s, scale=scale, **host))
    # scores of up to 100, whose products' magnitudes add up to less than 400: 400 * 2^-21
    assert ((out - want).abs() <= EPS[s.dtype] * (want.abs() + mean) + 2e-4 * mean)[ok].all()
    assert ((lse - want_lse).abs() <= 2e-5 * want_lse.abs().clamp(min=1) + 2e-4)[ok].all()


@pytest.mark.parametrize("make", [R.Setup, R8.Setup8])
@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("rows", [1, 90, 300])
@pytest.mark.parametrize("cap", [0.0, 40.0])
def test_steep_slopes(make, dtype, rows, cap):
    """Slopes of thousands leave a row its own position and its neighbour's: their scores count the distances 0 and 1, wherever in a tile they lie.
    The product of a slope and a distance of 1 is off by 2^-24 of itself, next to nothing of a weight that it has made 0. The new rows of the
    second and third sequence begin at the last position of a tile of keys."""
    s = make([(rows, 700), (rows, rows + 255), (rows, rows + 127)], 8, 2, 128, 64, dtype, seed=rows)
    slopes = torch.tensor([0.0, 0.5, 3.0, 30.0, 1000.0, 5000.0, -0.01, 9999.0])
    d = Device(s)
    got = S.s3_paged_attention_scored(d.cache, d.batch, d.q, d.ws, cap=cap, slopes=slopes.cuda(), want_lse=True)
    d.fine()
    # where more than one key counts slopes are at most 30 and distances below 10: 300 * 2^-23 more. A dimension in which the one key that counts
    # has a code of 0 holds next to nothing: 700 keys lose up to 700 * 2^-32 there, as in test_values_at_both_ends
    close(s, got, lambda s: R8.scored(s, cap=cap, slopes=slopes), lost=700 * 2.0 ** -32)


# ---------------------------------------------------------------------------------------------- norms
@pytest.mark.parametrize("make", [R.Setup, R8.Setup8])
@pytest.mark.parametrize("D,rot", [(128, 0), (64, 64)])
def test_norms_of_rows_of_any_size(make, D, rot):
    """A norm makes rows of any size alike: bf16 rows from 2^-60 (where eps counts) to 2^126, beside ordinary ones in the same warp. fp32 as in
    test_gpu_kv8.py: 2^-20 of the row's largest, then one rounding."""
    s = make([(40, 100), (1, 33)], 4, 2, D, 16, seed=2)
    sizes = torch.tensor([0, 30, 62, 64, 100, 124, -20, -60, 0, 63])
    s.q = (s.q.float().clamp(-3, 3) * 2.0 ** sizes[torch.arange(s.T) % 10][:, None, None]).to(BF)
    s.k = (s.k.float().clamp(-3, 3) * 2.0 ** sizes[torch.arange(s.T) % 10][:, None, None]).to(BF)
    w = [torch.exp(0.3 * torch.randn(D, generator=s.g)) for _ in range(2)]
    angle = torch.arange(100, dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(0, max(rot, 16), 2, dtype=torch.float64) / max(rot, 16))
    cos, sin = angle.cos().float(), angle.sin().float()
    d = Device(s)
    rope = S.Rope(cos.cuda(), sin.cuda()) if rot else None
    q = S.s3_kv_append_norm(d.cache, d.batch, s.k.cuda(), s.v.cuda(), d.ws, q=s.q.cuda(), rope=rope, norm=S.HeadNorm(w[0].cuda(), w[1].cuda(), 1e-6))
    k, _ = S.s3_kv_read(d.cache, d.batch, d.ws)
    d.fine()
    for got, x, weight, held in ((q, s.q, w[0], False), (k, s.k, w[1], make is R8.Setup8)):
        y = R8.new_rows(s, x, weight, 1e-6, cos, sin, rot, False)
        most = y.abs().amax(-1, keepdim=True)
        if held:
            code, scale = R8.held8(y)
            y = (code.float() * scale[..., None]).double()   # codes are equal, scales within 2^-23
        assert ((got.double().cpu() - y).abs() <= EPS[BF] * y.abs() + 2.0 ** -19 * most).all()


@pytest.mark.parametrize("make", [R.Setup, R8.Setup8])
def test_a_workspace_of_the_header_alone(make):
    """Calls that take whole units need no more; what is not there to mark blocks in is not written."""
    s = make([(20, 200), (30, 90)], 8, 2, 128, 64, seed=6)
    d = Device(s)
    pool = torch.zeros(4096, dtype=torch.uint8, device="cuda")
    pool[64:] = 171
    got = S.s3_paged_attention_scored(d.cache, d.batch, d.q, pool[:64], cap=30.0, want_lse=True)
    close(s, got, lambda s: R8.scored(s, cap=30.0))
    assert (pool[64:] == 171).all() and S.s3_workspace_status(pool[:64]) == 0
