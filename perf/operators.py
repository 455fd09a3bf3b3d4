"""Workloads of the paged key/value cache operators: append with rotation and block summaries, block selection, attention
over a paged cache, attention over selected blocks. Head layouts are those of the key / query projections that the scan
configurations encode (32 query heads over 8 key heads of 128, 28 over 4), chunks and spans likewise (8192 and 2048 tokens,
64 positions). Synthetic values, seeded."""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
DEV = "cuda"
STEPS = 4096.0          # fixed-point steps per unit in which keys and queries are summed
FAR = 2047.0            # and the largest magnitude they count with


# ------------------------------------------------------------------------------------------------ cases
def _case(name, op, heads, kv_heads, dim, page, seqs, q, kv, ragged=False, dtype="bf16", s=0, lists="token", window=0,
          interleaved=False):
    return {"name": name, "op": op, "heads": heads, "kv_heads": kv_heads, "dim": dim, "page": page, "seqs": seqs, "q": q,
            "kv": kv, "ragged": ragged, "dtype": dtype, "s": s, "lists": lists, "window": window, "interleaved": interleaved}


def listed():
    return [
        # one decoding step of a small serving batch: a token per sequence, latency counts
        _case("append step 48", "append", 28, 4, 128, 64, 48, 1, 6000, ragged=True, dtype="f16"),
        # one streamed 8192-token chunk of a long prompt
        _case("append chunk 8192", "append", 32, 8, 128, 64, 1, 8192, 16384),
        # blocks for one token of each of 24 conversations with long contexts
        _case("select step 24x32k", "select", 32, 8, 128, 64, 24, 1, 32768, ragged=True, s=16),
        # blocks for every token of a 2048-token chunk late in a prompt
        _case("select chunk 2048x32k", "select", 32, 8, 128, 64, 1, 2048, 32768, s=16),
        # the smallest call: one sequence at the start of its answer
        _case("attend step 1x777", "attend", 28, 4, 128, 16, 1, 1, 777),
        # one sequence answering over the full 128K context
        _case("attend step 1x128k", "attend", 32, 8, 128, 64, 1, 1, 131072),
        # a serving batch of uneven lengths
        _case("attend step 64x8k", "attend", 28, 4, 128, 64, 64, 1, 8192, ragged=True, dtype="f16"),
        # prompts of uneven lengths, narrow heads, small pages
        _case("attend ragged 7x733", "attend", 16, 4, 64, 16, 7, 733, 3001, ragged=True),
        # a 2048-token chunk at the end of a 32K prompt
        _case("attend chunk 2048x32k", "attend", 32, 8, 128, 64, 1, 2048, 32768),
        # one decoding step over the selected blocks
        _case("blocks step 24x32k", "blocks", 32, 8, 128, 64, 24, 1, 32768, ragged=True, s=16),
        # every token of a chunk over its own selected blocks
        _case("blocks chunk 1024x32k", "blocks", 32, 8, 128, 64, 1, 1024, 32768, s=16),
        # questions of up to 64 tokens, each over the 16 evidence spans that the retrieval returned for it
        _case("blocks query 16x64", "blocks", 32, 8, 128, 64, 16, 64, 8192, ragged=True, s=16, lists="query"),
    ]


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["append", "select", "attend", "attend", "blocks", "blocks"])
    heads, kv_heads, dim = rng.choice([(32, 8, 128), (28, 4, 128), (16, 4, 64), (8, 8, 128), (16, 1, 128)])
    dtype = rng.choice(["bf16", "bf16", "f16"])
    page = rng.choice([16, 32, 64, 128]) if op != "select" else rng.choice([32, 64, 128])
    lists = rng.choice(["token", "query"])
    if rng.random() < 0.5:                                    # one decoding step of a batch
        seqs, q = _spread(rng, 1, 96), 1
        kv = _spread(rng, 300, min(131072, 800000 // seqs))
    else:                                                     # chunks
        q = _spread(rng, 2, 1600)
        seqs = max(1, min(_spread(rng, 1, 24), 2048 // q))
        kv = _spread(rng, max(300, q), max(q + 300, min(40000, (1 << 24) // (q * seqs))))
    if op == "append" and q > 1:
        q, seqs = _spread(rng, 2, 8192), 1
        kv = q + rng.randrange(0, 8192)
    s = min(rng.choice([4, 8, 16, 24]), 2048 // page) if op in ("select", "blocks") else 0
    window = rng.choice([0, 0, 0, 1024]) if op == "attend" else 0
    case = _case("", op, heads, kv_heads, dim, page, seqs, q, max(kv, q), rng.random() < 0.6, dtype, s, lists, window,
                 rng.random() < 0.3)
    del case["name"]
    return case


def _lengths(case):
    """New tokens and cached positions (the new ones included) of each sequence: the first has the largest of both."""
    n, q, kv = case["seqs"], case["q"], case["kv"]
    if not case["ragged"]:
        return [q] * n, [kv] * n
    part = [1.0 if i == 0 else math.modf(i * 0.6180339887)[0] for i in range(n)]
    back = [1.0 if i == 0 else math.modf(i * 0.4142135623)[0] for i in range(n)]
    new = [1 + int((q - 1) * p) for p in part]
    return new, [a + int((kv - q) * b) for a, b in zip(new, back)]


def _pairs(case):
    """Visible (query token, key) pairs."""
    total, w = 0, case["window"]
    for q, kv in zip(*_lengths(case)):
        lo, hi = kv - q + 1, kv
        total += (lo + hi) * q // 2
        if w and hi > w:
            a = max(lo, w + 1)
            total -= ((a - w) + (hi - w)) * (hi - a + 1) // 2
    return total


def work(case):
    new, kv = _lengths(case)
    T, H, K, D, P = sum(new), case["heads"], case["kv_heads"], case["dim"], case["page"]
    blocks = sum(-(-n // P) for n in kv)
    if case["op"] == "append":
        touched = sum((b - 1) // P - (b - a) // P + 1 for a, b in zip(new, kv))
        return {"bytes": 4 * T * (H + 2 * K) * D + T * D * 4 + touched * K * (D + 4), "flops": 4 * T * (H + K) * D}
    if case["op"] == "select":
        pairs = sum(sum(p // P + 1 for p in range(b - a, b)) for a, b in zip(new, kv))
        return {"bytes": 2 * T * H * D + blocks * K * (D + 4) + 4 * T * K * case["s"], "flops": 2 * pairs * K * D}
    io = 4 * T * H * D + 4 * T * H
    if case["op"] == "attend":
        w = case["window"]
        seen = sum(b if not w else min(b, w + a - 1) for a, b in zip(new, kv))
        return {"bytes": io + 4 * seen * K * D, "flops": 4 * _pairs(case) * H * D}
    s, hs = case["s"], K if case["lists"] == "token" else 1
    read, pairs, rows = 0, 0, 0
    for a, b in zip(new, kv):
        nb = -(-b // P)
        n = min(s, nb)
        if case["lists"] == "token":
            read += min(nb, a * n) * P
            pairs += sum(min((p // P) * P + P, s * P, p + 1) for p in range(b - a, b))
            rows += a
        else:
            read += min(n * P, b)
            pairs += a * min(n * P, b)
            rows += 1
    return {"bytes": io + 4 * read * K * D + 4 * rows * hs * s, "flops": 4 * pairs * H * D}


# ------------------------------------------------------------------------------------------------ inputs
def _summaries(k, length=None):
    """Codes (int8) and scales of the blocks' mean keys; k [..., positions, dim], length the positions that count."""
    f = torch.round(torch.nan_to_num(k.float(), nan=0.0).clamp(-FAR, FAR) * STEPS)
    if length is not None:
        f = f * (torch.arange(k.shape[-2], device=k.device)[:, None] < length[..., None, None])
    total = f.to(torch.int32).sum(-2, dtype=torch.int32)
    count = torch.full_like(total[..., :1], k.shape[-2]) if length is None else length[..., None]
    most = total.abs().amax(-1, keepdim=True)
    code = torch.round(total.float() * 127.0 / most.clamp(min=1).float()).to(torch.int8)
    return code, (most.float() / count.clamp(min=1).float())[..., 0]


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    dt = DTYPES[case["dtype"]]
    H, K, D, P = case["heads"], case["kv_heads"], case["dim"], case["page"]
    new, kv = _lengths(case)
    n, T = len(new), sum(new)
    most = -(-max(kv) // P)

    def normal(*shape):
        return torch.randn(shape, generator=g, device=DEV, dtype=torch.float32)

    # keys share a per-channel mean and have a few loud channels, as key projections do; values have a mean too
    mean = normal(K, 1, D) * 0.6
    gain = torch.exp(0.3 * normal(K, 1, D))
    n_pages = sum(-(-b // P) for b in kv) + 3
    k_cache = torch.empty((n_pages, K, P, D), device=DEV, dtype=dt)
    v_cache = torch.empty_like(k_cache)
    for a in range(0, n_pages, 512):
        b = min(n_pages, a + 512)
        # a block's keys have a direction in common, which is what makes some blocks matter more to a query than others
        k_cache[a:b] = ((normal(b - a, K, P, D) + 0.5 * normal(b - a, K, 1, D)) * gain + mean).to(dt)
        v_cache[a:b] = (normal(b - a, K, P, D) + 0.3 * mean).to(dt)
    order = torch.randperm(n_pages, generator=g, device=DEV).to(torch.int32)
    pages = torch.full((n, most), -1, device=DEV, dtype=torch.int32)
    at = 0
    for i, b in enumerate(kv):
        c = -(-b // P)
        pages[i, :c] = order[at:at + c]
        at += c
    cu = torch.zeros(n + 1, dtype=torch.int32)
    cu[1:] = torch.tensor(new).cumsum(0)
    # one fused projection output per token: the heads' queries, then keys, then values
    qkv = torch.cat([normal(T, H, D), (normal(T, K, D) * gain[:, 0] + mean[:, 0]), normal(T, K, D) + 0.3 * mean[:, 0]], 1)
    qkv = qkv.to(dt).reshape(T, (H + 2 * K) * D)
    st = {"case": case, "k_cache": k_cache, "v_cache": v_cache, "pages": pages, "cu": cu.to(DEV),
          "kv_len": torch.tensor(kv, device=DEV, dtype=torch.int32), "T": T, "max_q": max(new), "max_kv": max(kv),
          "q": qkv[:, :H * D].view(T, H, D), "k": qkv[:, H * D:(H + K) * D].view(T, K, D),
          "v": qkv[:, (H + K) * D:].view(T, K, D), "scale": D ** -0.5}
    if case["op"] in ("append", "select"):
        st["code"], st["mean_scale"] = _summaries(k_cache)
    if case["op"] == "append":
        angle = torch.arange(max(kv), dtype=torch.float64)[:, None] * 500000.0 ** (-torch.arange(0, D, 2, dtype=torch.float64) / D)
        st["cos"], st["sin"] = angle.cos().float().to(DEV), angle.sin().float().to(DEV)
    if case["op"] == "blocks":
        st["blocks"] = _some_blocks(case, st, new, kv, g)
    if own:
        import paper_2601_17702_b200 as S

        st["cache"] = S.KvCache(k_cache, v_cache, st.get("code"), st.get("mean_scale"))
        st["batch"] = S.KvBatch(st["cu"], st["kv_len"], pages, T, st["max_q"], st["max_kv"])
        st["ws"] = S.new_workspace(S.s3_kv_workspace_bytes(st["cache"], st["batch"], H))
        if case["op"] == "append":
            st["rope"] = S.Rope(st["cos"], st["sin"], interleaved=case["interleaved"])
    return st


def _some_blocks(case, st, new, kv, g):
    """Block lists of the form a selection returns: ascending, the first block and the token's own among them, -1 padded."""
    P, s, K = case["page"], case["s"], case["kv_heads"]
    if case["lists"] == "token":
        hs, own_block = K, torch.cat([torch.arange(b - a, b) for a, b in zip(new, kv)]).to(DEV) // P
    else:
        hs, own_block = 1, (torch.tensor(kv, device=DEV) - 1) // P
    top = int(own_block.max()) + 1
    w = torch.rand((own_block.numel(), hs, top), generator=g, device=DEV)
    j = torch.arange(top, device=DEV)
    w = torch.where(j == own_block[:, None, None], 3.0, torch.where(j == 0, 2.0, w))
    w = torch.where(j > own_block[:, None, None], -1.0, w)
    best, at = w.topk(min(s, top), -1)
    at = torch.where(best < 0, top, at).sort(-1).values
    at = torch.where(at == top, -1, at).to(torch.int32)
    return torch.nn.functional.pad(at, (0, s - at.shape[-1]), value=-1).contiguous()


# ------------------------------------------------------------------------------------------------ plain forms
def _token_rows(st):
    """Per new token: its sequence, its index there, its position."""
    t = torch.arange(st["T"], device=DEV)
    seq = torch.searchsorted(st["cu"][1:].long(), t, right=True)
    i = t - st["cu"].long()[seq]
    lens = (st["cu"][1:] - st["cu"][:-1]).long()
    return seq, i, st["kv_len"].long()[seq] - lens[seq] + i


def _rotate(x, cos, sin, interleaved):
    a, b = (x[..., 0::2], x[..., 1::2]) if interleaved else x.chunk(2, -1)
    lo, hi = a * cos - b * sin, b * cos + a * sin
    return torch.stack([lo, hi], -1).flatten(-2) if interleaved else torch.cat([lo, hi], -1)


def _append(st):
    c, dt = st["case"], st["q"].dtype
    P = c["page"]
    seq, _, pos = _token_rows(st)
    cos, sin = st["cos"][pos][:, None], st["sin"][pos][:, None]
    q = _rotate(st["q"].float(), cos, sin, c["interleaved"]).to(dt)
    k = _rotate(st["k"].float(), cos, sin, c["interleaved"]).to(dt)
    page = st["pages"].long()[seq, pos // P]
    st["k_cache"][page, :, pos % P] = k
    st["v_cache"][page, :, pos % P] = st["v"]
    # the summaries of the blocks the new tokens lie in
    kv = st["kv_len"].long()
    first = (kv - (st["cu"][1:] - st["cu"][:-1]).long()) // P
    j = first[:, None] + torch.arange((st["max_q"] + P - 2) // P + 1, device=DEV)
    j = torch.minimum(j, (kv[:, None] - 1) // P)
    touched = st["pages"].long().gather(1, j)
    code, scale = _summaries(st["k_cache"][touched], (kv[:, None] - j * P).clamp(max=P)[..., None].expand(-1, -1, c["kv_heads"]))
    st["code"][touched], st["mean_scale"][touched] = code, scale
    return {"q": q, "k": st["k_cache"], "v": st["v_cache"], "means": st["code"] * st["mean_scale"][..., None]}


def _select(st):
    c = st["case"]
    P, s, T, K = c["page"], c["s"], st["T"], c["kv_heads"]
    seq, _, pos = _token_rows(st)
    q = torch.round(st["q"].float().clamp(-FAR, FAR) * STEPS).to(torch.int32).view(T, K, -1, c["dim"]).sum(2, dtype=torch.int32)
    most = q.abs().amax(-1, keepdim=True).clamp(min=1)
    q = torch.round(q.float() * 127.0 / most.float())
    nb = st["pages"].shape[1]
    at = st["pages"].long().clamp(min=0)
    code, scale = st["code"][at].float(), st["mean_scale"][at]                     # [B, nb, K, D], [B, nb, K]
    if code.shape[0] == 1:                                                          # whole numbers below 2^24: exact
        dots = torch.einsum("tkd,nkd->tkn", q, code[0])
    else:
        padded = torch.zeros((code.shape[0], st["max_q"], K, c["dim"]), device=DEV)
        padded[seq, _token_rows(st)[1]] = q
        dots = torch.einsum("bqkd,bnkd->bqkn", padded, code)[seq, _token_rows(st)[1]]
    score = dots * scale[seq].transpose(1, 2)
    own_block = (pos // P)[:, None, None]
    j = torch.arange(nb, device=DEV)
    score = torch.where((j < 1) | (j > own_block - 2), torch.inf, score)            # the first block and the last two
    score = torch.where(j > own_block, -torch.inf, score)
    best, at = score.sort(dim=-1, descending=True, stable=True)                      # ties: the lowest block
    best, at = best[..., :s], at[..., :s]
    at = torch.where(best == -torch.inf, nb, at).sort(-1).values
    at = torch.where(at == nb, -1, at).to(torch.int32)
    return {"blocks": torch.nn.functional.pad(at, (0, s - at.shape[-1]), value=-1)}


def _attend(st):
    c, dt = st["case"], st["q"].dtype
    H, K, D, P = c["heads"], c["kv_heads"], c["dim"], c["page"]
    B, Q, G = st["pages"].shape[0], st["max_q"], H // K
    seq, i, pos = _token_rows(st)
    at = st["pages"].long().clamp(min=0)
    L = at.shape[1] * P
    k = st["k_cache"][at].transpose(1, 2).reshape(B, K, L, D).float()
    v = st["v_cache"][at].transpose(1, 2).reshape(B, K, L, D).float()
    q = torch.zeros((B, Q, H, D), device=DEV)
    q[seq, i] = st["q"].float()
    q = q.view(B, Q, K, G, D).permute(0, 2, 1, 3, 4).reshape(B, K, Q * G, D) * st["scale"]
    where = torch.full((B, Q), -1, device=DEV)
    where[seq, i] = pos
    j = torch.arange(L, device=DEV)
    seen = j <= where[..., None]                                                    # [B, Q, L]
    if c["window"]:
        seen &= j > where[..., None] - c["window"]
    seen = seen[:, None]
    if c["op"] == "blocks":
        listed_ = st["blocks"].long()
        rows, hs, _ = listed_.shape
        has = torch.zeros((rows, hs, at.shape[1] + 1), device=DEV, dtype=torch.bool)
        has.scatter_(2, torch.where(listed_ < 0, at.shape[1], listed_), True)
        has = has[..., :-1].repeat_interleave(P, -1)
        if c["lists"] == "token":
            mine = torch.zeros((B, Q, hs, L), device=DEV, dtype=torch.bool)
            mine[seq, i] = has
            seen = seen & mine.transpose(1, 2)
        else:
            seen = seen & has[:, :, None]
    score = torch.matmul(q, k.transpose(-1, -2))
    score.view(B, K, Q, G, L).masked_fill_(~seen[:, :, :, None], -torch.inf)
    most = score.amax(-1, keepdim=True)
    most = torch.where(most == -torch.inf, 0.0, most)
    score.sub_(most).exp_()
    total = score.sum(-1, keepdim=True)
    out = torch.matmul(score, v) / torch.where(total == 0, 1.0, total)
    lse = total.log() + most
    out = out.view(B, K, Q, G, D).transpose(1, 2).reshape(B, Q, H, D)[seq, i].to(dt)
    return {"out": out, "lse": lse.view(B, K, Q, G).transpose(1, 2).reshape(B, Q, H)[seq, i]}


def run(st):
    op = st["case"]["op"]
    if not own:
        return _append(st) if op == "append" else _select(st) if op == "select" else _attend(st)
    import paper_2601_17702_b200 as S

    c, cache, batch, ws = st["case"], st["cache"], st["batch"], st["ws"]
    if op == "append":
        q = S.s3_kv_append(cache, batch, st["k"], st["v"], ws, q=st["q"], rope=st["rope"])
        return {"q": q, "k": st["k_cache"], "v": st["v_cache"], "means": st["code"] * st["mean_scale"][..., None]}
    if op == "select":
        return {"blocks": S.s3_block_select(cache, batch, st["q"], c["s"], ws, n_first=1, n_last=2)}
    if op == "attend":
        out, lse = S.s3_paged_attention(cache, batch, st["q"], ws, scale=st["scale"], window=c["window"], want_lse=True)
    else:
        out, lse = S.s3_block_attention(cache, batch, st["q"], st["blocks"], ws, scale=st["scale"],
                                        per_token=c["lists"] == "token", want_lse=True)
    return {"out": out, "lse": lse}


# ------------------------------------------------------------------------------------------------ 64 bits
def exact(case, seed):
    if case["op"] == "select":
        return None                                           # whole numbers
    st = prepare(case, seed)
    new, kv = _lengths(case)
    H, K, D, P = case["heads"], case["kv_heads"], case["dim"], case["page"]
    G = H // K
    starts = [sum(new[:i]) for i in range(len(new))]
    if case["op"] == "append":
        q = st["q"].double()
        kc, vc = st["k_cache"].double(), st["v_cache"].double()
        means = st["code"].double() * st["mean_scale"].double()[..., None]
        half = torch.arange(D // 2, device=DEV)
        lo, hi = (2 * half, 2 * half + 1) if case["interleaved"] else (half, half + D // 2)
        table = st["pages"].tolist()
        for b, (a, n) in enumerate(zip(new, kv)):
            here = slice(starts[b], starts[b] + a)
            pos = torch.arange(n - a, n, device=DEV)
            turn = torch.complex(st["cos"][pos].double(), st["sin"][pos].double())[:, None]
            key = st["k"][here].double()
            for x in (q[here], key):
                z = torch.complex(x[..., lo], x[..., hi]) * turn
                x[..., lo], x[..., hi] = z.real, z.imag
            for j in range((n - a) // P, (n - 1) // P + 1):
                p0, p1 = max(j * P, n - a), min(j * P + P, n)
                page = table[b][j]
                kc[page, :, p0 - j * P:p1 - j * P] = key[p0 - (n - a):p1 - (n - a)].transpose(0, 1)
                vc[page, :, p0 - j * P:p1 - j * P] = st["v"][here].double()[p0 - (n - a):p1 - (n - a)].transpose(0, 1)
                # the summaries are of the keys as the cache holds them
                held = kc[page, :, :p1 - j * P].to(st["q"].dtype).double()
                total = torch.round(held.clamp(-FAR, FAR) * STEPS).sum(1)
                most = total.abs().amax(-1, keepdim=True)
                means[page] = torch.round(total * 127 / most.clamp(min=1)) * (most / (p1 - j * P))
        return {"q": q, "k": kc, "v": vc, "means": means}
    if 8 * _pairs(case) * H * D > 3e13:
        return None
    out = torch.zeros((st["T"], H, D), device=DEV, dtype=torch.float64)
    lse = torch.full((st["T"], H), -torch.inf, device=DEV, dtype=torch.float64)
    lists = st["blocks"].long() if case["op"] == "blocks" else None
    for b, (a, n) in enumerate(zip(new, kv)):
        held = st["pages"][b, :-(-n // P)].long()
        pos = torch.arange(n - a, n, device=DEV)[:, None]
        j = torch.arange(n, device=DEV)
        may = j <= pos
        if case["window"]:
            may &= j + case["window"] > pos
        for h in range(K):
            keys = st["k_cache"][held, h].reshape(-1, D)[:n].double()
            values = st["v_cache"][held, h].reshape(-1, D)[:n].double()
            see = may
            if lists is not None:
                mine = lists[starts[b]:starts[b] + a, h] if case["lists"] == "token" else lists[b, 0].expand(a, -1)
                hit = torch.zeros((a, held.numel()), device=DEV)
                hit.scatter_add_(1, mine.clamp(min=0), (mine >= 0).float())
                see = see & (hit[:, j // P] > 0)
            for g in range(h * G, h * G + G):
                x = st["q"][starts[b]:starts[b] + a, g].double() @ keys.T * D ** -0.5
                x = torch.where(see, x, -torch.inf)
                lse[starts[b]:starts[b] + a, g] = torch.logsumexp(x, -1)
                out[starts[b]:starts[b] + a, g] = torch.softmax(x, -1) @ values
    return {"out": out, "lse": lse}
