"""Paged key / value cache operators at the edges: narrow weights, wide windows, pages that a window has left behind, steps that
follow each other without a pause, misaligned arrays, every variant the host's plan can pick.

Tolerances are those of the tests beside it: eps = 2^-8 (bf16) or 2^-11 (f16); a result is a mean of values under weights rounded
to the type, each off by at most eps of itself, and is rounded once: |out - exact| <= eps (|out| + mean |v|) + 1e-4, the mean of |v|
under the exact weights. (f16 weights are lifted so that only those 2^-21 and more below the largest are subnormal; what
these lose is under 2^-32 each, 2^-15 of the largest weight for the 131072 keys here.)"""
import ctypes as C
import math

import pytest
import torch

import kv_reference as R
import paper_2601_17702_b200 as S
from paper_2601_17702_b200 import binding as B
from test_gpu_kv import Device, check, dev

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n,seqs", [(1, 600), (40, 300)])
@pytest.mark.parametrize("octaves", [18.5, 20.25, 23.5])
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_many_keys_far_below_the_largest_weight(n, seqs, octaves, dtype):
    """A strong first key and 131071 equal ones of weight 2^-octaves each, which together weigh 2^(17 - octaves). As many sequences,
    all over the same pages, as thread blocks run at a time or more: most of them are not cut into pieces."""
    s = R.Setup([(n, 131072)], 2, 1, 64, 128, dtype, seed=1, outside=0.0)
    s.scale = 1.0
    s.q.zero_()
    s.q[:, :, 0] = 8.0
    s.k_cache.zero_()
    s.v_cache.copy_((1 + torch.arange(64) / 64).to(dtype).expand_as(s.v_cache))
    first = int(s.pages[0, 0])
    s.k_cache[first, 0, 0, 0] = octaves * math.log(2.0) / 8
    s.v_cache[first, 0, 0] = 0
    want, want_lse = R.attention(s)
    cache = S.KvCache(dev(s.k_cache), dev(s.v_cache))
    batch = S.KvBatch(torch.arange(seqs + 1, dtype=torch.int32, device="cuda") * n, torch.full((seqs,), 131072, dtype=torch.int32, device="cuda"),
                      dev(s.pages.repeat(seqs, 1)), seqs * n, n, 131072)
    ws = S.new_workspace(S.s3_kv_workspace_bytes(cache, batch, 2))
    out, lse = S.s3_paged_attention(cache, batch, dev(s.q.repeat(seqs, 1, 1)), ws, scale=1.0, want_lse=True)
    assert S.s3_workspace_status(ws) == 0
    want, want_lse = want.repeat(seqs, 1, 1), want_lse.repeat(seqs, 1)
    check(s, out, lse, want, want_lse, mean_abs=want.abs())


@pytest.mark.parametrize("lens", [[(4, 2), (1, 30), (3, 0)], [(90, 40), (70, 70), (130, 125)]])
@pytest.mark.parametrize("window", [2**31 - 1, 2**31 - 30, 41])
def test_windows_up_to_the_largest_number(lens, window):
    """More new rows than positions: the first rows' positions are negative, and position - window passes 32 bits."""
    s = R.Setup(lens, 8, 2, 128, 16, seed=window % 97)
    d = Device(s)
    out, lse = S.s3_paged_attention(d.cache, d.batch, d.q, d.ws, window=window, want_lse=True)
    d.fine()
    check(s, out, lse, *R.attention(s, window=window))


def test_steps_that_follow_each_other_without_a_pause():
    """Launches overlap the one before them: append, select and attend on one cache, one list buffer and one workspace, step after step
    without waiting for the GPU, give what they give with a pause after every call."""
    H, K, D, P, n, steps = 8, 2, 128, 16, 3, 40
    g = torch.Generator().manual_seed(11)
    start = [400, 90, 250]
    q, k, v = (torch.randn((steps, n, x, D), generator=g).bfloat16().cuda() for x in (H, K, K))
    k[:, :, :, :40] *= 3.0
    held = torch.randn((120, K, P, D), generator=g).bfloat16().cuda()
    pages = torch.randperm(120, generator=g).to(torch.int32)[:n * 33].view(n, 33).cuda()
    cu = torch.arange(n + 1, dtype=torch.int32, device="cuda")
    lens = [torch.tensor([x + i + 1 for x in start], dtype=torch.int32, device="cuda") for i in range(steps)]

    def run(pause):
        cache = S.KvCache.zeros(120, K, P, D)
        cache.k.copy_(held)
        cache.v.copy_(held.flip(0))
        batch = [S.KvBatch(cu, lens[i], pages, n, 1, 33 * P) for i in range(steps)]
        ws = S.new_workspace(S.s3_kv_workspace_bytes(cache, batch[0], H))
        first = S.KvBatch(torch.tensor([0, 400, 490, 740], dtype=torch.int32, device="cuda"), torch.tensor(start, dtype=torch.int32, device="cuda"),
                          pages, 740, 400, 33 * P)
        prompt = torch.cat([held.flip(1).reshape(-1, K, D)[:740], held.flip(2).reshape(-1, K, D)[:740]], 1)
        S.s3_kv_append(cache, first, prompt[:, :K], prompt[:, K:], ws)
        lists = torch.full((n, K, 6), -7, dtype=torch.int32, device="cuda")
        out, seen = torch.empty((n, H, D), dtype=torch.bfloat16, device="cuda"), []
        kept = [(torch.empty_like(lists), torch.empty_like(out)) for _ in range(steps)]
        torch.cuda.synchronize()
        for i in range(steps):
            S.s3_kv_append(cache, batch[i], k[i], v[i], ws)
            torch.cuda.synchronize() if pause else None
            S.s3_block_select(cache, batch[i], q[i], 6, ws, blocks=lists)
            torch.cuda.synchronize() if pause else None
            S.s3_block_attention(cache, batch[i], q[i], lists, ws, out=out)
            torch.cuda.synchronize() if pause else None
            S.s3_block_select(cache, batch[i], q[i - 1], 6, ws, blocks=lists)      # the buffer is written again while the last call ends
            torch.cuda.synchronize() if pause else None
            S.s3_block_attention(cache, batch[i], q[i], lists, ws, out=kept[i][1])
            torch.cuda.synchronize() if pause else None
            S.s3_block_select(cache, batch[i], q[i], 6, ws, blocks=kept[i][0])
            torch.cuda.synchronize() if pause else None
        assert S.s3_workspace_status(ws) == 0
        return [x for pair in kept for x in pair] + [out, lists, cache.k, cache.v, cache.code, cache.scale]

    want = run(True)
    for _ in range(3):
        assert all(torch.equal(a, b) for a, b in zip(run(False), want))


def test_masks_of_one_call_are_not_those_of_the_next():
    """Per-token lists of a chunk as masks, the lists other ones in every call, through one workspace and without a pause."""
    s = R.Setup([(300, 900)], 8, 8, 128, 64, seed=31)
    d = Device(s)
    g = torch.Generator().manual_seed(5)
    lists = [dev(torch.stack([torch.randperm(15, generator=g)[:7] for _ in range(s.T * 8)]).view(s.T, 8, 7).to(torch.int32)) for _ in range(6)]
    want = []
    for x in lists:
        want.append(S.s3_block_attention(d.cache, d.batch, d.q, x, d.ws)[0])
        torch.cuda.synchronize()
    check(s, *S.s3_block_attention(d.cache, d.batch, d.q, lists[0], d.ws, want_lse=True), *R.attention(s, blocks=lists[0].cpu()))
    for _ in range(3):
        got = [S.s3_block_attention(d.cache, d.batch, d.q, x, d.ws)[0] for x in lists]
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    d.fine()


def test_misaligned_arrays_are_refused_before_any_launch():
    """A workspace that is a slice at an odd offset, and 4-byte arrays off their boundary, in every call."""
    s = R.Setup([(1, 4000), (30, 300)], 8, 2, 128, 16, seed=1, outside=0.0)
    d = Device(s, torch.zeros((s.n_pages, 2, 128), dtype=torch.int8), torch.zeros((s.n_pages, 2)))
    lists = torch.zeros((s.T, 2, 4), dtype=torch.int32, device="cuda")
    room = torch.zeros(d.ws.numel() + 64, dtype=torch.uint8, device="cuda")
    lib, code = B.lib(), S.S3_ERR_INVALID_ARG
    k, v, out, lse = dev(s.k), dev(s.v), torch.empty_like(d.q), torch.zeros((s.T + 1, 8), device="cuda")
    params = B.AttnParams(0.1, 1, 0, 0)

    def calls(ws=d.ws, batch=d.batch, lists=lists.data_ptr(), lse=lse.data_ptr(), positions=None):
        H, D = 8, 128
        at, n, st = ws.data_ptr(), ws.numel(), torch.cuda.current_stream().cuda_stream
        q, o, ref, c = d.q.data_ptr(), out.data_ptr(), C.byref(batch.desc), d.cache.handle
        cos = torch.ones((4000, 8), device="cuda")
        rope = S.Rope(cos, cos)
        return [lib.s3_kv_append(c, ref, rope.ref, positions, None, 0, 0, None, 0, k.data_ptr(), 2 * D, v.data_ptr(), 2 * D, at, n, st),
                lib.s3_block_select(c, ref, q, H * D, H, 4, 1, 1, lists, at, n, st),
                lib.s3_paged_attention(c, ref, q, H * D, H, C.byref(params), o, H * D, lse, at, n, st),
                lib.s3_block_attention(c, ref, q, H * D, H, lists, 4, 2, 1, C.byref(params), o, H * D, lse, at, n, st)]

    assert calls() == [0] * 4
    for off in (1, 2, 4, 8, 12, 17):
        assert calls(ws=room[off:]) == [code] * 4
    assert calls(ws=room[16:]) == [0] * 4 and calls(ws=room[48:]) == [0] * 4
    assert calls(lists=lists.data_ptr() + 2)[1::2] == [code] * 2
    assert calls(lse=lse.data_ptr() + 2)[2:] == [code] * 2
    assert calls(positions=lists.data_ptr() + 1)[0] == code
    for field in ("d_cu_q", "d_kv_len", "d_pages"):
        bad = S.KvBatch(d.batch.cu_q, d.batch.kv_len, d.batch.pages, s.T, s.max_q, s.max_kv)
        setattr(bad.desc, field, getattr(bad.desc, field) + 2)
        assert calls(batch=bad) == [code] * 4
    torch.cuda.synchronize()
    d.fine()


def left_behind(s, window):
    """The setup again, with the pages that no row's window reaches gone: NaN, and no page in the table."""
    t = R.Setup(s.lens, s.H, s.K, s.D, s.P, s.dtype, seed=s.seed)
    for i, (n, kv) in enumerate(s.lens):
        for j in range(max(kv - n - window + 1, 0) // s.P):
            page = int(t.pages[i, j])
            t.k_cache[page], t.v_cache[page] = float("nan"), float("nan")
            t.pages[i, j] = -1 if j % 2 else 2**31 - 1
    return t


@pytest.mark.parametrize("lens", [[(1, 700), (1, 333), (0, 40), (1, 20)], [(3, 1000)], [(90, 700), (3, 500)], [(300, 1500)]])
@pytest.mark.parametrize("D,P,window,dtype", [(128, 16, 33, torch.bfloat16), (64, 16, 100, torch.float16), (128, 64, 70, torch.bfloat16),
                                              (64, 128, 1, torch.float16), (128, 32, 200, torch.bfloat16)])
def test_pages_before_the_window_may_be_gone(lens, D, P, window, dtype):
    s = R.Setup(lens, 8, 2, D, P, dtype, seed=window)
    s.seed = window
    d = Device(left_behind(s, window))
    out, lse = S.s3_paged_attention(d.cache, d.batch, d.q, d.ws, window=window, want_lse=True)
    d.fine()
    check(s, out, lse, *R.attention(s, window=window))


@pytest.mark.parametrize("lens", [[(252, 700)] * 3, [(300, 1500)], [(1, 300), (2, 800)]])
@pytest.mark.parametrize("D,P,n,window,dtype", [(128, 16, 40, 90, torch.bfloat16), (64, 64, 12, 70, torch.float16), (128, 128, 6, 33, torch.float16)])
def test_listed_pages_before_the_window_may_be_gone(lens, D, P, n, window, dtype):
    """Per-token lists that name blocks behind the window too, as lists and as masks."""
    s = R.Setup(lens, 8, 8, D, P, dtype, seed=n)
    s.seed = n
    d = Device(left_behind(s, window))
    g = torch.Generator().manual_seed(n)
    lists = torch.full((s.T, 1, n), -1, dtype=torch.int32)
    for t, i, pos in s.rows():
        blocks = torch.randperm(pos // P + 1, generator=g)[:n]
        lists[t, 0, :len(blocks)] = blocks.to(torch.int32)
    out, lse = S.s3_block_attention(d.cache, d.batch, d.q, dev(lists), d.ws, window=window, want_lse=True)
    d.fine()
    check(s, out, lse, *R.attention(s, window=window, blocks=lists))


@pytest.mark.parametrize("n", [1, 80])
@pytest.mark.parametrize("offset", [3, 40, 70, 127])
@pytest.mark.parametrize("octaves", [6, 12, 14.5, 20, 40])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_one_key_far_above_the_others_anywhere_in_a_tile(n, offset, octaves, dtype):
    """Late tiles in which one key of either half rises over what the weights so far refer to, by less and by more than they hold."""
    s = R.Setup([(n, 1500)], 4, 1, 128, 16, dtype, seed=int(octaves) + offset)
    s.q *= 0.1
    s.q[:, :, 0] = 4.0
    s.k_cache[..., 0] = s.k_cache[..., 0].nan_to_num(0.0) * 0.1
    for at, more in ((640 + offset, 0.0), (1024 + offset, 3.0)):
        page, row = int(s.pages[0, at // 16]), at % 16
        s.k_cache[page, :, row] = 0
        s.k_cache[page, :, row, 0] = (octaves + more) * math.log(2.0) / (4 * s.scale)
    d = Device(s)
    out, lse = S.s3_paged_attention(d.cache, d.batch, d.q, d.ws, want_lse=True)
    d.fine()
    check(s, out, lse, *R.attention(s))


@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
def test_wild_keys_out_of_sight_of_few_rows(bad):
    """A key that only the last two of three rows may see."""
    s = R.Setup([(3, 200)], 4, 1, 128, 16, seed=8)
    s.k_cache[int(s.pages[0, 198 // 16]), :, 198 % 16] = bad
    d = Device(s)
    out, _ = S.s3_paged_attention(d.cache, d.batch, d.q, d.ws)
    want, _ = R.attention(s)
    out = out.double().cpu()
    assert ((out - want)[:1].abs() <= 2.0 ** -8 * (want[:1].abs() + 1.2) + 1e-4).all()
    assert torch.isnan(want[1:]).any() and torch.equal(torch.isnan(out[1:]), torch.isnan(want[1:]))


# ---- variants of the plan, each with its results -------------------------------------------------
def on_gpu(s, window=0, blocks=None):
    """The 64-bit definition on the GPU, a sequence and a query head at a time."""
    out = torch.zeros((s.T, s.H, s.D), dtype=torch.float64)
    lse = torch.full((s.T, s.H), -math.inf, dtype=torch.float64)
    G = s.H // s.K
    for i, (n, kv) in enumerate(s.lens):
        if n == 0 or kv == 0:
            continue
        rows = slice(s.cu[i], s.cu[i] + n)
        j, pos = torch.arange(kv, device="cuda"), torch.arange(kv - n, kv, device="cuda")[:, None]
        base = (j <= pos) & ((j > pos - window) if window else True)
        for h in range(s.K):
            k, v = s.held(i, h, "k").cuda(), s.held(i, h, "v").cuda()
            see = base
            if blocks is not None:
                lst = blocks[rows, h if blocks.shape[1] > 1 else 0].cuda().long()
                last = (kv - 1) // s.P
                listed = torch.zeros((n, last + 2), dtype=torch.bool, device="cuda")
                listed.scatter_(1, torch.where((lst >= 0) & (lst <= last), lst, last + 1), True)
                see = base & listed[:, j // s.P]
            some = see.any(1, keepdim=True)
            for g in range(h * G, h * G + G):
                x = (dev(s.q[rows, g]).double() @ k.T * s.scale).masked_fill(~see, -math.inf)
                lse[rows, g] = torch.logsumexp(x, -1).cpu()
                out[rows, g] = (torch.where(some, torch.softmax(x, -1), 0.0) @ v).cpu()
    return out, lse


def variant(s, n=0):
    """What the plan of this batch picks: (query tiles per item, masks, shares, whole rounds before them)."""
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    p = S.s3_attn_plan_describe(len(s.lens), s.T, s.max_q, s.max_kv, s.H, s.K, s.D, s.P, sms, s=n)
    tiles = 0 if not p.tile else 2 if p.tokens_per_item > 128 // (s.H // s.K) else 1
    return tiles, bool(p.masked), bool(p.shares), p.whole_rounds > 0


def lists_with_holes(s, n, heads, seed):
    """n distinct blocks in random places, some ahead of the row or past the sequence, every seventh list empty."""
    g = torch.Generator().manual_seed(seed)
    top = torch.tensor([s.lens[i][1] // s.P + 2 for _, i, _ in s.rows()])
    order = torch.rand((s.T, heads, int(top.max()) + n), generator=g).argsort(-1)[..., :n].to(torch.int32)
    order[order >= top[:, None, None]] = -1
    order[torch.arange(s.T) % 7 == 3, 0] = -1
    return order


@pytest.mark.parametrize("lens,H,K,D,P,dtype,window,want", [
    ([(1, 900), (1, 333)], 8, 2, 128, 16, torch.float16, 0, (0, False, True, False)),
    ([(2, 60), (1, 33), (0, 9)], 8, 2, 64, 16, torch.bfloat16, 0, (0, False, False, False)),
    ([(20, 120), (19, 77)], 8, 8, 64, 128, torch.bfloat16, 0, (1, False, False, False)),
    ([(270, 1621)], 8, 8, 128, 16, torch.float16, 0, (1, False, True, False)),
    ([(65, 65), (64, 131), (0, 3)] * 4, 28, 4, 128, 32, torch.bfloat16, 40, (2, False, False, False)),
    ([(270, 1621)], 8, 2, 64, 64, torch.float16, 300, (2, False, True, False)),
    ([(2401, 9700)], 28, 4, 128, 64, torch.bfloat16, 0, (2, False, True, False)),
    ([(2561, 10301)], 16, 16, 128, 64, torch.bfloat16, 0, (2, False, True, True)),
    ([(1299, 9401)], 32, 32, 64, 16, torch.float16, 3000, (2, False, True, True))])
def test_every_variant_over_the_whole_cache(lens, H, K, D, P, dtype, window, want):
    s = R.Setup(lens, H, K, D, P, dtype, seed=H + P)
    assert variant(s) == want
    d = Device(s)
    out, lse = S.s3_paged_attention(d.cache, d.batch, d.q, d.ws, window=window, want_lse=True)
    d.fine()
    check(s, out, lse, *on_gpu(s, window))


@pytest.mark.parametrize("lens,H,K,D,P,n,dtype,window,want", [
    ([(20, 200), (1, 40)], 8, 8, 128, 16, 4, torch.bfloat16, 0, (0, False, False, False)),
    ([(20, 200), (1, 40)], 8, 2, 64, 16, 60, torch.float16, 0, (0, False, True, False)),
    ([(20, 2000), (7, 310)], 20, 1, 128, 16, 20, torch.bfloat16, 0, (1, False, False, False)),
    ([(20, 4100)], 20, 1, 64, 16, 60, torch.float16, 100, (1, False, True, False)),
    ([(20, 25), (33, 90)], 8, 8, 64, 64, 40, torch.bfloat16, 0, (1, True, False, False)),
    ([(270, 1621)], 8, 8, 128, 16, 24, torch.float16, 200, (1, True, True, False)),
    ([(65, 65), (64, 131), (0, 3)] * 4, 28, 4, 128, 16, 24, torch.float16, 0, (2, True, False, False)),
    ([(65, 65), (64, 131), (0, 3)] * 4, 28, 4, 64, 16, 24, torch.bfloat16, 40, (2, True, False, False)),
    ([(252, 565), (251, 400), (0, 60), (252, 252), (3, 500)], 32, 8, 128, 128, 5, torch.bfloat16, 0, (2, True, False, False)),
    ([(423, 1840), (300, 1500), (77, 1840)], 32, 8, 128, 128, 16, torch.bfloat16, 0, (2, True, True, False)),
    ([(270, 1621)], 8, 2, 64, 64, 25, torch.float16, 500, (2, True, True, False)),
    ([(2601, 10405)], 16, 16, 128, 64, 30, torch.bfloat16, 0, (2, True, True, True)),
    ([(1300, 9402)], 32, 32, 64, 16, 60, torch.float16, 1500, (2, True, True, True))])
def test_every_variant_of_lists_per_token(lens, H, K, D, P, n, dtype, window, want):
    s = R.Setup(lens, H, K, D, P, dtype, seed=H + P + n)
    assert variant(s, n) == want
    d = Device(s)
    for heads in {1, K}:
        lists = lists_with_holes(s, n, heads, seed=n)
        out, lse = S.s3_block_attention(d.cache, d.batch, d.q, dev(lists), d.ws, window=window, want_lse=True)
        d.fine()
        check(s, out, lse, *on_gpu(s, window, lists))


def test_the_largest_batchs_workspace_serves_the_others():
    """Smaller batches in a workspace that a larger one has filled, each with the result that it gets in its own."""
    big = R.Setup([(300, 4000)], 16, 2, 128, 64, seed=3)
    d = Device(big)
    S.s3_paged_attention(d.cache, d.batch, d.q, d.ws)
    for lens in ([(299, 3000)], [(40, 2500), (3, 500)], [(17, 500)] * 3, [(3, 500)] * 3, [(1, 64)] * 9, [(1, 1)], [(1, 4000)]):
        s = R.Setup(lens, 16, 2, 128, 64, seed=len(lens), outside=0.0)
        e = Device(s)
        assert e.ws.numel() <= d.ws.numel()
        lists = dev(lists_with_holes(s, 5, 2, seed=1))
        for ws in (d.ws.fill_(0xFF), e.ws):
            ws[:S.S3_WS_HEADER_BYTES] = 0
            got = S.s3_paged_attention(e.cache, e.batch, e.q, ws, want_lse=True) + S.s3_block_attention(e.cache, e.batch, e.q, lists, ws, want_lse=True)
            assert S.s3_workspace_status(ws) == 0
            if ws is d.ws:
                first = got
        assert all(torch.equal(a, b) for a, b in zip(first, got))


@pytest.mark.parametrize("lens,n", [([(1, 3000), (1, 100)], 6), ([(300, 900)], 9), ([(20, 2000), (300, 1621)], 20)])
def test_a_captured_step_replays_on_new_inputs(lens, n):
    """Append, select and both attentions in one graph; replayed after the inputs changed in place, it gives what the calls give."""
    s = R.Setup(lens, 16, 4, 128, 64, seed=15, outside=0.0)
    d = Device(s, torch.zeros((s.n_pages, 4, 128), dtype=torch.int8), torch.zeros((s.n_pages, 4)))
    angle = torch.rand((4000, 64), device="cuda") * 6.28
    rope, k, v = S.Rope(angle.cos(), angle.sin()), dev(s.k), dev(s.v)
    lists = torch.empty((s.T, 4, n), dtype=torch.int32, device="cuda")
    rq, a, b = torch.empty_like(d.q), torch.empty_like(d.q), torch.empty_like(d.q)
    la, lb = (torch.empty((s.T, 16), device="cuda") for _ in range(2))

    def step():
        S.s3_kv_append(d.cache, d.batch, k, v, d.ws, q=d.q, rope=rope, q_out=rq)
        S.s3_block_select(d.cache, d.batch, rq, n, d.ws, blocks=lists)
        S.s3_block_attention(d.cache, d.batch, rq, lists, d.ws, out=a, lse=la)
        S.s3_paged_attention(d.cache, d.batch, rq, d.ws, out=b, lse=lb)

    def results():
        return [x.clone() for x in (rq, lists, a, la, b, lb, d.k, d.v, d.code, d.scale)]

    step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(3):
        for x in (k, v, d.q):
            x.copy_(x.roll(1, 0) * (1.5 if i == 1 else 1.0))
        step()
        want = results()
        for x in (rq, lists, a, la, b, lb):
            x.zero_()
        graph.replay()
        assert all(torch.equal(x, y) for x, y in zip(results(), want))
    d.fine()
