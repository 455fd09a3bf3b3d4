"""Paged key / value cache operators against their 64-bit definitions.

Tolerances, derived before the first run. eps = 2^-8 (bf16) or 2^-11 (f16), half a unit in the last place relative to the
value. The result is a mean of values under weights that are rounded to the type: each weight is off by at most eps of
itself, so the result by at most eps * mean |v| (v of order 1: at most 1.2 per row, summed with the weights), plus its own
rounding, eps |out|; fp32 score errors add about 1e-5. So |out - exact| <= eps * (|out| + mean |v|) + 1e-4, with the weights'
mean of |v| computed along. The log-sum-exp comes from fp32 scores of magnitude < 40: 2e-5 relative to max(1, |lse|), twice the
error of a score of 40 in fp32 products over 128 terms. Rotations: two products and a sum in fp32, then one rounding: within
eps |x| + 2^-22 * 8 of the 64-bit value. Codes, scales and lists are whole numbers or correctly rounded: equal."""
import math

import pytest
import torch

import kv_reference as R
import paper_2601_17702_b200 as S

pytestmark = pytest.mark.gpu
EPS = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


def dev(t):
    return t.cuda()


class Device:
    """The setup's tensors and handles on the GPU."""

    def __init__(self, s, code=None, scale=None, T=None):
        self.k, self.v = dev(s.k_cache), dev(s.v_cache)
        self.code, self.scale = (None, None) if code is None else (dev(code), dev(scale))
        self.cache = S.KvCache(self.k, self.v, self.code, self.scale)
        self.batch = S.KvBatch(torch.tensor(s.cu, dtype=torch.int32, device="cuda"),
                               torch.tensor([kv for _, kv in s.lens], dtype=torch.int32, device="cuda"), dev(s.pages), s.T, s.max_q, s.max_kv)
        self.ws = S.new_workspace(S.s3_kv_workspace_bytes(self.cache, self.batch, s.H))
        self.q = dev(s.q)

    def fine(self):
        assert S.s3_workspace_status(self.ws) == 0


def check(s, out, lse, want, want_lse, mean_abs=None):
    out, lse = out.double().cpu(), lse.double().cpu()
    eps = EPS[s.dtype]
    assert torch.isfinite(out).all()
    room = eps * (want.abs() + (1.2 if mean_abs is None else mean_abs)) + 1e-4
    bad = (out - want).abs() > room
    assert not bad.any(), f"{int(bad.sum())} of {bad.numel()} off, worst {(out - want).abs().max():.3g} at {bad.nonzero()[:3].tolist()}"
    empty = want_lse == -math.inf
    assert torch.equal(lse == -math.inf, empty)
    assert (out[empty] == 0).all()
    d = (lse - want_lse)[~empty].abs()
    assert (d <= 2e-5 * want_lse[~empty].abs().clamp(min=1)).all(), f"lse off by {d.max():.3g}"


HEADS = [(4, 4, 128), (8, 2, 128), (14, 2, 128), (16, 1, 128), (6, 2, 64), (20, 1, 64), (9, 3, 128)]
DECODE = [(1, 1), (1, 2), (1, 63), (1, 64), (1, 65), (0, 70), (1, 257), (1, 1030)]


@pytest.mark.parametrize("H,K,D", HEADS)
@pytest.mark.parametrize("P,dtype", [(16, torch.bfloat16), (64, torch.float16), (128, torch.bfloat16)])
def test_attention_of_single_tokens(H, K, D, P, dtype):
    s = R.Setup(DECODE, H, K, D, P, dtype, seed=H * P)
    d = Device(s)
    out, lse = S.s3_paged_attention(d.cache, d.batch, d.q, d.ws, want_lse=True)
    d.fine()
    check(s, out, lse, *R.attention(s))


CHUNKS = [
    [(5, 5)], [(33, 33)], [(64, 200), (1, 77), (0, 10), (31, 31)], [(150, 150)], [(257, 400), (2, 300)],
    [(3, 1000), (40, 700), (1, 129), (128, 128), (129, 513)],
]


@pytest.mark.parametrize("lens", CHUNKS)
@pytest.mark.parametrize("H,K,D,P,dtype", [(8, 2, 128, 64, torch.bfloat16), (14, 2, 128, 16, torch.float16), (4, 4, 64, 32, torch.bfloat16),
                                           (20, 1, 128, 128, torch.bfloat16), (3, 1, 64, 128, torch.float16)])
def test_attention_of_chunks(lens, H, K, D, P, dtype):
    s = R.Setup(lens, H, K, D, P, dtype, seed=len(lens) + H)
    d = Device(s)
    out, lse = S.s3_paged_attention(d.cache, d.batch, d.q, d.ws, want_lse=True)
    d.fine()
    check(s, out, lse, *R.attention(s))


@pytest.mark.parametrize("window", [1, 17, 64, 100, 5000])
@pytest.mark.parametrize("lens", [[(1, 700), (1, 40)], [(90, 700), (3, 65)]])
def test_attention_window(window, lens):
    s = R.Setup(lens, 8, 2, 128, 64, seed=window)
    d = Device(s)
    out, lse = S.s3_paged_attention(d.cache, d.batch, d.q, d.ws, window=window, want_lse=True)
    d.fine()
    check(s, out, lse, *R.attention(s, window=window))


@pytest.mark.parametrize("lens", [[(1, 30), (4, 100)], [(100, 300)]])
def test_attention_not_causal(lens):
    s = R.Setup(lens, 8, 2, 128, 32, seed=5)
    d = Device(s)
    out, lse = S.s3_paged_attention(d.cache, d.batch, d.q, d.ws, causal=False, scale=0.05, want_lse=True)
    d.fine()
    check(s, out, lse, *R.attention(s, causal=False, scale=0.05))


@pytest.mark.parametrize("lens", [[(4, 2), (1, 0), (2, 2)], [(90, 40), (70, 0), (50, 50)]])
def test_rows_before_the_first_position_are_empty(lens):
    s = R.Setup(lens, 8, 2, 128, 16, seed=9)
    d = Device(s)
    out, lse = S.s3_paged_attention(d.cache, d.batch, d.q, d.ws, want_lse=True)
    d.fine()
    check(s, out, lse, *R.attention(s))


def some_lists(s, n, heads, per_token, seed, ascending=False):
    """Random distinct blocks with holes, blocks ahead of the row, past the sequence, and empty lists among them."""
    g = torch.Generator().manual_seed(seed)
    rows = list(s.rows()) if per_token else [(i, i, kv - 1) for i, (_, kv) in enumerate(s.lens)]
    out = torch.full((len(rows), heads, n), -1, dtype=torch.int32)
    for x, (_, i, pos) in enumerate(rows):
        top = s.lens[i][1] // s.P + 2                    # one or two past the last block too
        for h in range(heads):
            c = min(n, top) if (x + h) % 5 else 0        # every fifth list is empty
            pick = torch.randperm(top, generator=g)[:c]
            at = torch.randperm(n, generator=g)[:c]
            if ascending:
                pick, at = pick.sort().values, torch.arange(c)
            out[x, h, at] = pick.to(torch.int32)
    return out


@pytest.mark.parametrize("P,n", [(16, 1), (16, 9), (32, 5), (64, 6), (128, 3), (64, 40)])
@pytest.mark.parametrize("H,K,D,dtype", [(8, 2, 128, torch.bfloat16), (14, 2, 64, torch.float16), (20, 1, 128, torch.bfloat16), (2, 2, 128, torch.float16)])
@pytest.mark.parametrize("per_token", [True, False])
def test_attention_over_listed_blocks(P, n, H, K, D, dtype, per_token):
    lens = [(1, 500), (3, 64), (0, 90), (37, 333), (1, 1)]
    s = R.Setup(lens, H, K, D, P, dtype, seed=P + n)
    d = Device(s)
    for heads in {1, K}:
        lists = some_lists(s, n, heads, per_token, seed=n)
        out, lse = S.s3_block_attention(d.cache, d.batch, d.q, dev(lists), d.ws, per_token=per_token, want_lse=True)
        d.fine()
        check(s, out, lse, *R.attention(s, blocks=lists, per_token=per_token))


def test_all_blocks_listed_is_attention_over_everything():
    s = R.Setup([(40, 300)], 8, 2, 128, 16, seed=3)
    d = Device(s)
    lists = torch.arange(s.max_kv // 16 + 1, dtype=torch.int32, device="cuda").flip(0).view(1, 1, -1).contiguous()
    out, lse = S.s3_block_attention(d.cache, d.batch, d.q, lists, d.ws, per_token=False, window=33, want_lse=True)
    d.fine()
    check(s, out, lse, *R.attention(s, window=33))


@pytest.mark.parametrize("lens,H,K", [([(1, 9000)], 4, 2), ([(20, 9000)], 8, 2)])
def test_splits_are_joined(lens, H, K):
    """Enough keys for several splits, in both kernels; a key far above the others in one split only."""
    s = R.Setup(lens, H, K, 128, 64, seed=1)
    page, off = int(s.pages[0, 100]), 13
    s.k_cache[page, :, off] = (s.q[-1].view(K, H // K, 128).float().mean(1) * 6).to(s.dtype)
    d = Device(s)
    assert S.s3_kv_workspace_bytes(d.cache, d.batch, H) > 4096
    out, lse = S.s3_paged_attention(d.cache, d.batch, d.q, d.ws, want_lse=True)
    d.fine()
    check(s, out, lse, *R.attention(s))


@pytest.mark.parametrize("lens", [[(1, 300)], [(80, 300)]])
def test_scores_that_grow_along_the_keys(lens):
    """Every key tile raises the maximum far above the last one: the accumulator is rescaled each time."""
    s = R.Setup(lens, 4, 1, 128, 16, seed=2)
    for j in range(-(-300 // 16)):
        p = int(s.pages[0, j])
        c = min(16, 300 - 16 * j)
        s.k_cache[p, :, :c] = (s.k_cache[p, :, :c].float() * 0.1 + s.q[0, 0].float() * 0.05 * j).to(s.dtype)
    d = Device(s)
    out, lse = S.s3_paged_attention(d.cache, d.batch, d.q, d.ws, want_lse=True)
    d.fine()
    check(s, out, lse, *R.attention(s))


def test_infinite_scores_and_keys_out_of_sight():
    """An infinite key at a position that only the last rows may see: the others are not touched by it."""
    s = R.Setup([(60, 200)], 4, 1, 128, 16, seed=8)
    p, off = int(s.pages[0, 198 // 16]), 198 % 16
    s.k_cache[p, :, off] = float("inf")
    d = Device(s)
    out, _ = S.s3_paged_attention(d.cache, d.batch, d.q, d.ws)
    want, _ = R.attention(s)
    out = out.double().cpu()
    assert torch.isfinite(out[:58]).all()
    assert ((out - want)[:58].abs() <= EPS[s.dtype] * (want[:58].abs() + 1.2) + 1e-4).all()
    assert torch.isnan(out[58:]).any() == torch.isnan(want[58:]).any()


def test_strided_rows_pool_and_another_stream():
    """Queries as a slice of a fused projection, output with a row pitch, one pool for keys and values, calls on a side stream."""
    H, K, D, P = 8, 2, 128, 32
    s = R.Setup([(1, 100), (1, 555)], H, K, D, P, seed=4)
    pool = torch.full((s.n_pages, 2, K, P, D), float("nan"), dtype=s.dtype, device="cuda")
    pool[:, 0], pool[:, 1] = dev(s.k_cache), dev(s.v_cache)
    fused = torch.randn((s.T, H * D + 72), device="cuda").to(s.dtype)
    fused[:, 8:8 + H * D] = dev(s.q).view(s.T, H * D)
    q = fused[:, 8:8 + H * D].view(s.T, H, D)
    big = torch.full((s.T, H * D + 40), 7.0, dtype=s.dtype, device="cuda")
    d = Device(s)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    cache = S.KvCache(pool[:, 0], pool[:, 1])
    with torch.cuda.stream(side):
        out, lse = S.s3_paged_attention(cache, d.batch, q, d.ws, out=big[:, 16:16 + H * D].view(s.T, H, D), want_lse=True)
    torch.cuda.current_stream().wait_stream(side)
    d.fine()
    check(s, out, lse, *R.attention(s))
    assert (big[:, :16] == 7).all() and (big[:, 16 + H * D:] == 7).all()


def test_page_offsets_past_32_bits():
    """Pages more than 2^31 elements apart, and a cache of which only the far end is used."""
    K, P, D = 1, 16, 64
    stride = (1 << 30) + 64
    s = R.Setup([(1, 40), (30, 40)], 2, K, D, P, seed=6, spare=0)
    store = torch.empty(stride * (s.n_pages - 1) + 2 * K * P * D, dtype=s.dtype, device="cuda")
    k = store.as_strided((s.n_pages, K, P, D), (stride, P * D, D, 1))
    v = store.as_strided((s.n_pages, K, P, D), (stride, P * D, D, 1), K * P * D)
    k.copy_(dev(s.k_cache))
    v.copy_(dev(s.v_cache))
    assert stride * (s.n_pages - 1) > 2 ** 32
    d = Device(s)
    cache = S.KvCache(k, v)
    out, lse = S.s3_paged_attention(cache, d.batch, d.q, d.ws, want_lse=True)
    d.fine()
    check(s, out, lse, *R.attention(s))
    S.s3_kv_append(cache, d.batch, dev(s.k), dev(s.v), d.ws)
    d.fine()
    for t, i, pos in s.rows():
        page = int(s.pages[i, pos // P])
        assert torch.equal(k[page, :, pos % P].cpu(), s.k[t]) and torch.equal(v[page, :, pos % P].cpu(), s.v[t])


def test_bad_pages_and_lengths_are_reported_and_harmless():
    s = R.Setup([(1, 100), (40, 80)], 4, 2, 128, 16, seed=7)
    s.pages[0, 2], s.pages[1, 0] = -5, s.n_pages
    d = Device(s)
    before = d.k.clone()
    out, _ = S.s3_paged_attention(d.cache, d.batch, d.q, d.ws)
    assert torch.isfinite(out.float()).all()                     # the page reads as zeros
    with pytest.raises(S.S3Error) as e:
        S.s3_workspace_status(d.ws)
    assert e.value.code == S.S3_ERR_INVALID_ARG
    d.ws.zero_()
    s2 = R.Setup([(3, 16)], 4, 2, 128, 16, seed=7)
    s2.pages[0, 0] = s2.n_pages + 1
    d2 = Device(s2)
    before = d2.k.clone()
    S.s3_kv_append(d2.cache, d2.batch, dev(s2.k), dev(s2.v), d2.ws)
    with pytest.raises(S.S3Error):
        S.s3_workspace_status(d2.ws)
    assert torch.equal(d2.k.view(torch.int16), before.view(torch.int16))
    d3 = Device(s)
    d3.batch = S.KvBatch(d3.batch.cu_q, torch.tensor([100, 5000], dtype=torch.int32, device="cuda"), d3.batch.pages, s.T, s.max_q, s.max_kv)
    S.s3_paged_attention(d3.cache, d3.batch, d3.q, d3.ws)
    with pytest.raises(S.S3Error):
        S.s3_workspace_status(d3.ws)


# ------------------------------------------------------------------------------------------------ append
def tables(n, rot, theta=10000.0):
    a = torch.arange(n, dtype=torch.float64)[:, None] * theta ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)
    return a.cos().float(), a.sin().float()


@pytest.mark.parametrize("lens", [[(1, 1), (1, 64), (1, 65), (0, 30), (1, 200)], [(70, 70), (0, 5), (3, 66), (130, 150)], [(5, 3)]])
@pytest.mark.parametrize("H,K,D,P,dtype,rot,inter", [(8, 2, 128, 64, torch.bfloat16, 128, False), (4, 4, 64, 16, torch.float16, 32, True),
                                                     (6, 2, 128, 128, torch.float16, 48, False), (2, 1, 64, 32, torch.bfloat16, 64, True)])
def test_append(lens, H, K, D, P, dtype, rot, inter):
    s = R.Setup(lens, H, K, D, P, dtype, seed=P)
    code = torch.zeros((s.n_pages, K, D), dtype=torch.int8)
    scale = torch.full((s.n_pages, K), -3.0)
    d = Device(s, code, scale)
    cos, sin = tables(256, rot)
    rope = S.Rope(dev(cos), dev(sin), interleaved=inter)
    given = torch.randint(0, 256, (s.T,), generator=s.g).to(torch.int32)
    for positions in (None, given):
        q = S.s3_kv_append(d.cache, d.batch, dev(s.k), dev(s.v), d.ws, q=d.q, rope=rope, positions=None if positions is None else dev(positions))
        d.fine()
        q, kc, vc, cc, sc = q.cpu(), d.k.cpu(), d.v.cpu(), d.code.cpu(), d.scale.cpu()
        eps = EPS[dtype]
        touched = set()
        for t, i, pos in s.rows():
            row = int(given[t]) if positions is not None else max(pos, 0)
            c, sn = cos[row].double(), sin[row].double()
            want = R.rotate(s.q[t].double(), c, sn, rot, inter)
            assert ((q[t].double() - want).abs() <= eps * want.abs() + 2.0 ** -19).all()
            if pos < 0:
                continue
            page = int(s.pages[i, pos // P])
            want = R.rotate(s.k[t].double(), c, sn, rot, inter)
            got = kc[page, :, pos % P].double()
            assert ((got - want).abs() <= eps * want.abs() + 2.0 ** -19).all()
            assert torch.equal(got[:, rot:], want[:, rot:])
            assert torch.equal(vc[page, :, pos % P], s.v[t])
            s.k_cache[page, :, pos % P], s.v_cache[page, :, pos % P] = kc[page, :, pos % P], s.v[t]
            touched.add((i, pos // P))
        # nothing else was written
        assert torch.equal(kc.view(torch.int16), s.k_cache.view(torch.int16)) and torch.equal(vc.view(torch.int16), s.v_cache.view(torch.int16))
        seen = torch.zeros((s.n_pages,), dtype=torch.bool)
        for i, j in touched:
            page = int(s.pages[i, j])
            seen[page] = True
            for h in range(K):
                cw, sw = R.summary(s.k_cache[page, h, :min(P, lens[i][1] - j * P)])
                assert torch.equal(cc[page, h], cw) and float(sc[page, h]) == float(sw)
        assert (sc[~seen] == -3.0).all()


def test_append_without_rotation_queries_or_summaries_and_in_place():
    s = R.Setup([(3, 20), (40, 90)], 4, 2, 128, 16, seed=12)
    d = Device(s)
    assert S.s3_kv_append(d.cache, d.batch, dev(s.k), dev(s.v), d.ws) is None
    for t, i, pos in s.rows():
        page = int(s.pages[i, pos // 16])
        assert torch.equal(d.k[page, :, pos % 16].cpu(), s.k[t]) and torch.equal(d.v[page, :, pos % 16].cpu(), s.v[t])
    cos, sin = tables(128, 128)
    rope = S.Rope(dev(cos), dev(sin))
    apart = S.s3_kv_append(d.cache, d.batch, dev(s.k), dev(s.v), d.ws, q=d.q, rope=rope)
    q = d.q.clone()
    assert S.s3_kv_append(d.cache, d.batch, dev(s.k), dev(s.v), d.ws, q=q, rope=rope, q_out=q) is q
    assert torch.equal(q, apart)
    d.fine()
    far = torch.full((s.T,), 128, dtype=torch.int32, device="cuda")
    S.s3_kv_append(d.cache, d.batch, dev(s.k), dev(s.v), d.ws, rope=rope, positions=far)
    with pytest.raises(S.S3Error):
        S.s3_workspace_status(d.ws)


def test_summaries_after_a_rollback_and_of_wild_keys():
    """A sequence cut back and continued: the summary is that of what the page holds. NaN counts as 0, infinities as the limit."""
    s = R.Setup([(6, 60)], 2, 1, 128, 64, seed=13)
    s.k[2, 0, 5], s.k[3, 0, 6], s.k[3, 0, 7] = float("nan"), float("inf"), -1e30
    code = torch.zeros((s.n_pages, 1, 128), dtype=torch.int8)
    scale = torch.zeros((s.n_pages, 1))
    d = Device(s, code, scale)
    S.s3_kv_append(d.cache, d.batch, dev(s.k), dev(s.v), d.ws)
    page = int(s.pages[0, 0])
    held = d.k[page, 0, :60].cpu()
    cw, sw = R.summary(held)
    assert torch.equal(d.code[page, 0].cpu(), cw) and float(d.scale[page, 0]) == float(sw)
    back = S.KvBatch(torch.tensor([0, 1], dtype=torch.int32, device="cuda"), torch.tensor([55], dtype=torch.int32, device="cuda"),
                     d.batch.pages, 1, 1, 55)
    S.s3_kv_append(d.cache, back, dev(s.k[5:6]), dev(s.v[5:6]), d.ws)
    d.fine()
    cw, sw = R.summary(torch.cat([held[:54], s.k[5:6, 0]]))
    assert torch.equal(d.code[page, 0].cpu(), cw) and float(d.scale[page, 0]) == float(sw)


# ------------------------------------------------------------------------------------------------ selection
def summaries_of(s):
    code = torch.full((s.n_pages, s.K, s.D), 99, dtype=torch.int8)
    scale = torch.full((s.n_pages, s.K), float("nan"))
    for i, (_, kv) in enumerate(s.lens):
        for j in range(-(-kv // s.P)):
            page = int(s.pages[i, j])
            for h in range(s.K):
                code[page, h], scale[page, h] = R.summary(s.k_cache[page, h, :min(s.P, kv - j * s.P)])
    return code, scale


@pytest.mark.parametrize("lens", [[(1, 1), (1, 300), (0, 40), (1, 2000), (1, 64)], [(20, 1500), (3, 30), (2, 1)], [(4, 800)]])
@pytest.mark.parametrize("H,K,D,P,dtype", [(8, 2, 128, 16, torch.bfloat16), (14, 2, 64, 32, torch.float16), (4, 4, 128, 64, torch.bfloat16)])
@pytest.mark.parametrize("n,first,last", [(1, 0, 0), (4, 1, 2), (16, 0, 1), (33, 2, 0), (64, 1, 2)])
def test_selection(lens, H, K, D, P, dtype, n, first, last):
    s = R.Setup(lens, H, K, D, P, dtype, seed=P + n)
    code, scale = summaries_of(s)
    d = Device(s, code, scale)
    blocks = S.s3_block_select(d.cache, d.batch, d.q, n, d.ws, n_first=first, n_last=last)
    d.fine()
    assert torch.equal(blocks.cpu(), R.select(s, code, scale, n, first, last))


def test_selection_ties_and_zero_summaries():
    """Equal scores go to the lower block, over more candidates than the short list holds; all-zero queries tie everywhere."""
    s = R.Setup([(1, 16 * 900), (2, 16 * 500)], 4, 1, 128, 16, seed=21)
    code, scale = summaries_of(s)
    g = torch.Generator().manual_seed(3)
    pick = torch.randint(0, 3, (s.n_pages,), generator=g)
    for x in range(3):
        code[pick == x], scale[pick == x] = code[x].clone(), scale[x].clone().nan_to_num(0.5)
    s.q[1] = 0
    for n in (8, 16, 40):
        d = Device(s, code, scale)
        blocks = S.s3_block_select(d.cache, d.batch, d.q, n, d.ws, n_first=1, n_last=1)
        d.fine()
        assert torch.equal(blocks.cpu(), R.select(s, code, scale, n, 1, 1))


def test_selection_of_rows_before_the_first_position():
    s = R.Setup([(3, 1)], 4, 2, 128, 16, seed=2)
    code, scale = summaries_of(s)
    d = Device(s, code, scale)
    blocks = S.s3_block_select(d.cache, d.batch, d.q, 4, d.ws).cpu()
    assert (blocks[:2] == -1).all() and (blocks[2, :, 0] == 0).all() and (blocks[2, :, 1:] == -1).all()


# ------------------------------------------------------------------------------------------------ together, and refusals
def test_append_select_attend_step_by_step():
    """A prompt in chunks, then single tokens: what the cache, the summaries and the lists hold is what the next call reads."""
    H, K, D, P = 8, 2, 128, 16
    g = torch.Generator().manual_seed(5)
    n = 150
    cache = S.KvCache.zeros(12, K, P, D)
    pages = torch.randperm(12, generator=g).to(torch.int32)[:10].view(1, 10)
    cos, sin = tables(n, D)
    rope = S.Rope(dev(cos), dev(sin))
    q, k, v = (torch.randn((n, x, D), generator=g).bfloat16() for x in (H, K, K))
    done = 0
    for m in (70, 1, 33, 1, 1, 44):
        here = slice(done, done + m)
        done += m
        batch = S.KvBatch(torch.tensor([0, m], dtype=torch.int32, device="cuda"), torch.tensor([done], dtype=torch.int32, device="cuda"),
                          dev(pages), m, m, done)
        ws = S.new_workspace(S.s3_kv_workspace_bytes(cache, batch, H))
        rq = S.s3_kv_append(cache, batch, dev(k[here]), dev(v[here]), ws, q=dev(q[here]), rope=rope)
        blocks = S.s3_block_select(cache, batch, rq, 4, ws)
        out, lse = S.s3_block_attention(cache, batch, rq, blocks, ws, want_lse=True)
        full, full_lse = S.s3_paged_attention(cache, batch, rq, ws, want_lse=True)
        assert S.s3_workspace_status(ws) == 0
        s = R.Setup([(m, done)], H, K, D, P, seed=0, spare=2)
        s.pages, s.k_cache, s.v_cache, s.q = pages, cache.k.cpu(), cache.v.cpu(), rq.cpu()
        s.cols = 10
        want = R.select(s, cache.code.cpu(), cache.scale.cpu(), 4, 1, 2)
        assert torch.equal(blocks.cpu(), want)
        check(s, out, lse, *R.attention(s, blocks=want))
        check(s, full, full_lse, *R.attention(s))


def test_results_do_not_depend_on_the_run_or_on_a_captured_graph():
    s = R.Setup([(1, 3000), (1, 100)], 8, 2, 128, 64, seed=15)
    d = Device(s)
    a, la = S.s3_paged_attention(d.cache, d.batch, d.q, d.ws, want_lse=True)
    out, lse = torch.empty_like(a), torch.empty_like(la)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        S.s3_paged_attention(d.cache, d.batch, d.q, d.ws, out=out, lse=lse)
    for _ in range(2):
        out.zero_()
        graph.replay()
        assert torch.equal(out, a) and torch.equal(lse, la)
    d.fine()


def test_empty_batches_do_nothing():
    cache = S.KvCache.zeros(2, 2, 16, 64)
    e = torch.empty((0, 4, 64), dtype=torch.bfloat16, device="cuda")
    batch = S.KvBatch(torch.zeros(2, dtype=torch.int32, device="cuda"), torch.tensor([5], dtype=torch.int32, device="cuda"),
                      torch.zeros((1, 1), dtype=torch.int32, device="cuda"), 0, 0, 5)
    ws = S.new_workspace(S.s3_kv_workspace_bytes(cache, batch, 4))
    assert S.s3_paged_attention(cache, batch, e, ws)[0].shape == e.shape
    assert S.s3_block_select(cache, batch, e, 3, ws).shape == (0, 2, 3)
    S.s3_kv_append(cache, batch, e[:, :2], e[:, :2], ws, q=e)
    assert S.s3_workspace_status(ws) == 0


def refused(code, f, *a, **kw):
    with pytest.raises(S.S3Error) as e:
        f(*a, **kw)
    assert e.value.code == code


def test_refusals():
    s = R.Setup([(2, 40)], 8, 2, 128, 16, seed=1)
    d = Device(s)
    bad = S.KvBatch(d.batch.cu_q, d.batch.kv_len, d.batch.pages, s.T, s.T + 1, s.max_kv)
    refused(S.S3_ERR_INVALID_ARG, S.s3_paged_attention, d.cache, bad, d.q, d.ws)
    refused(S.S3_ERR_INVALID_ARG, S.s3_paged_attention, d.cache, d.batch, d.q[:, :7].contiguous(), d.ws)
    refused(S.S3_ERR_INVALID_ARG, S.s3_paged_attention, d.cache, d.batch, d.q, d.ws, scale=0.0)
    refused(S.S3_ERR_INVALID_ARG, S.s3_paged_attention, d.cache, d.batch, d.q, d.ws, scale=float("nan"))
    refused(S.S3_ERR_INVALID_ARG, S.s3_paged_attention, d.cache, d.batch, d.q, d.ws, window=-1)
    refused(S.S3_ERR_CAPACITY, S.s3_paged_attention, d.cache, d.batch, d.q, d.ws[:32])
    odd = torch.empty((2, 8 * 128 + 4), dtype=torch.bfloat16, device="cuda")
    refused(S.S3_ERR_INVALID_ARG, S.s3_paged_attention, d.cache, d.batch, odd[:, :1024].view(2, 8, 128), d.ws)
    refused(S.S3_ERR_INVALID_ARG, S.s3_paged_attention, d.cache, d.batch, odd.view(-1)[4:4 + 2048].view(2, 8, 128), d.ws)
    refused(S.S3_ERR_STATE, S.s3_block_select, d.cache, d.batch, d.q, 4, d.ws)
    lists = torch.zeros((2, 1, 513), dtype=torch.int32, device="cuda")
    refused(S.S3_ERR_UNSUPPORTED, S.s3_block_attention, d.cache, d.batch, d.q, lists, d.ws)
    refused(S.S3_ERR_INVALID_ARG, S.s3_block_attention, d.cache, d.batch, d.q, torch.zeros((2, 3, 4), dtype=torch.int32, device="cuda"), d.ws)
    c = Device(s, torch.zeros((s.n_pages, 2, 128), dtype=torch.int8), torch.zeros((s.n_pages, 2)))
    refused(S.S3_ERR_INVALID_ARG, S.s3_block_select, c.cache, c.batch, c.q, 2, c.ws, n_first=1, n_last=2)
    refused(S.S3_ERR_UNSUPPORTED, S.s3_block_select, c.cache, c.batch, c.q, 65, c.ws)
    t = torch.zeros((64, 12), device="cuda")
    refused(S.S3_ERR_UNSUPPORTED, S.s3_kv_append, d.cache, d.batch, dev(s.k), dev(s.v), d.ws, rope=S.Rope(t, t))
    for shape, dtype in (((2, 2, 24, 64), torch.bfloat16), ((2, 2, 16, 96), torch.bfloat16), ((2, 2, 16, 64), torch.float32)):
        x = torch.zeros(shape, dtype=dtype, device="cuda")
        refused(S.S3_ERR_UNSUPPORTED, S.KvCache, x, x)
    # a workspace for one split only where the call would use several
    s = R.Setup([(1, 4000)], 8, 2, 128, 16, seed=1)
    d = Device(s)
    refused(S.S3_ERR_CAPACITY, S.s3_paged_attention, d.cache, d.batch, d.q, d.ws[:512])


def on_gpu(s, blocks=None):
    """The 64-bit definition for one long sequence, on the GPU a key head at a time."""
    (n, kv), G = s.lens[0], s.H // s.K
    j, pos = torch.arange(kv, device="cuda"), torch.arange(kv - n, kv, device="cuda")[:, None]
    out, lse = torch.zeros((n, s.H, s.D), dtype=torch.float64), torch.zeros((n, s.H), dtype=torch.float64)
    for h in range(s.K):
        k, v = s.held(0, h, "k").cuda(), s.held(0, h, "v").cuda()
        for g in range(h * G, h * G + G):
            x = (dev(s.q[:, g]).double() @ k.T * s.scale).masked_fill(j > pos, -math.inf)
            lse[:, g] = torch.logsumexp(x, -1).cpu()
            out[:, g] = (torch.softmax(x, -1) @ v).cpu()
    return out, lse


@pytest.mark.parametrize("n,kv,H,K", [(1300, 5300, 32, 8), (1290, 9001, 28, 4)])
def test_a_chunk_late_in_a_prompt(n, kv, H, K):
    """Enough units for whole rounds before the shares, and cuts within units."""
    s = R.Setup([(n, kv)], H, K, 128, 64, seed=n)
    d = Device(s)
    out, lse = S.s3_paged_attention(d.cache, d.batch, d.q, d.ws, want_lse=True)
    d.fine()
    check(s, out, lse, *on_gpu(s))


@pytest.mark.parametrize("bound", [0, 3000])
def test_more_sequences_than_lanes(bound):
    """Batches of over 32 and over 64 sequences, empty ones among them; max_q and max_kv may be loose bounds."""
    for new in ([1] * 75, [(i * 7) % 41 for i in range(70)]):
        lens = [(q, q + (i * 37) % 300) for i, q in enumerate(new)]
        s = R.Setup(lens, 8, 2, 64, 16, seed=len(lens))
        s.max_kv += bound
        s.max_q = min(s.T, s.max_q + bound)
        wide = torch.full((len(lens), s.max_kv // 16 + s.cols), -7, dtype=torch.int32)
        wide[:, :s.cols] = s.pages
        s.pages, s.cols = wide, wide.shape[1]
        code, scale = summaries_of(s)
        d = Device(s, code, scale)
        out, lse = S.s3_paged_attention(d.cache, d.batch, d.q, d.ws, want_lse=True)
        d.fine()
        check(s, out, lse, *R.attention(s))
        blocks = S.s3_block_select(d.cache, d.batch, d.q, 5, d.ws)
        d.fine()
        assert torch.equal(blocks.cpu(), R.select(s, code, scale, 5, 1, 2))
        out, lse = S.s3_block_attention(d.cache, d.batch, d.q, blocks, d.ws, want_lse=True)
        d.fine()
        check(s, out, lse, *R.attention(s, blocks=blocks.cpu()))
        S.s3_kv_append(d.cache, d.batch, dev(s.k), dev(s.v), d.ws)
        d.fine()
        for t, i, pos in s.rows():
            assert torch.equal(d.k[int(s.pages[i, pos // 16]), :, pos % 16].cpu(), s.k[t])


def test_a_workspace_serves_smaller_batches():
    s = R.Setup([(300, 4000)], 16, 2, 128, 64, seed=3)
    d = Device(s)
    last = S.s3_kv_workspace_bytes(d.cache, d.batch, 16)
    for T, q, kv in ((300, 300, 4000), (299, 40, 3000), (64, 17, 500), (40, 3, 500), (9, 1, 64), (1, 1, 1)):
        b = S.KvBatch(d.batch.cu_q, d.batch.kv_len, d.batch.pages, T, q, kv)
        now = S.s3_kv_workspace_bytes(d.cache, b, 16)
        assert 0 < now <= last
        last = now


def test_example_runs_them_together():
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "evidence_attention.py")
    spec = importlib.util.spec_from_file_location("evidence_attention", path)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    question, answer, found = m.run(context=4096, chunk=1024)
    # the stretch asked about is one page of 64, and holds nearly all of the attention's weight
    assert found and question > 0.9 and min(answer) > 0.9


@pytest.mark.parametrize("lens", [[(300, 900)], [(130, 640), (0, 70), (260, 260), (1, 333), (90, 41)]])
@pytest.mark.parametrize("H,K,D,P,n,dtype,causal,window", [(8, 8, 128, 64, 9, torch.bfloat16, True, 0), (8, 2, 64, 16, 40, torch.float16, True, 0),
                                                           (8, 8, 128, 128, 6, torch.float16, True, 200), (14, 2, 128, 32, 12, torch.bfloat16, False, 0),
                                                           (6, 2, 128, 16, 24, torch.bfloat16, False, 150)])
def test_listed_blocks_that_cover_much_of_a_chunks_context(lens, H, K, D, P, n, dtype, causal, window):
    """Many rows whose lists are a good part of a short context. Blocks that no row lists hold NaN, their table entries no page."""
    s = R.Setup(lens, H, K, D, P, dtype, seed=P + n)
    for heads in {1, K}:
        lists = some_lists(s, n, heads, True, seed=n)
        skipped = lambda i, j: (7 * i + j) % 3 == 1
        for row, i, _ in s.rows():
            for b in range(s.cols + 1):
                if skipped(i, b):
                    lists[row][lists[row] == b] = -1
        t = R.Setup(lens, H, K, D, P, dtype, seed=P + n)
        for i, (_, kv) in enumerate(lens):
            for j in range(-(-kv // P)):
                if skipped(i, j):
                    page = int(t.pages[i, j])
                    t.k_cache[page], t.v_cache[page] = float("nan"), float("nan")
                    if j % 2:
                        t.pages[i, j] = 2**31 - 1 if j % 4 == 1 else -5
        d = Device(t)
        out, lse = S.s3_block_attention(d.cache, d.batch, d.q, dev(lists), d.ws, causal=causal, window=window, want_lse=True)
        d.fine()
        check(s, out, lse, *R.attention(s, causal=causal, window=window, blocks=lists))


def test_listed_blocks_of_a_chunk_whose_cached_positions_are_none():
    s = R.Setup([(200, 0)], 8, 8, 128, 16, seed=2)
    d = Device(s)
    lists = torch.zeros((s.T, 8, 20), dtype=torch.int32, device="cuda")
    lists += torch.arange(20, dtype=torch.int32, device="cuda")
    out, lse = S.s3_block_attention(d.cache, d.batch, d.q, lists, d.ws, want_lse=True)
    d.fine()
    assert (out == 0).all() and (lse == -math.inf).all()
