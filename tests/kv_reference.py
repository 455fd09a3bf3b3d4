"""Plain 64-bit definitions of the paged key / value cache operators, sequence by sequence and head by head, on the host."""
from __future__ import annotations

import math

import torch

STEPS, FAR = 4096.0, 2047.0


class Setup:
    """A batch over a fresh cache: lens = [(new rows, cached positions)], pages in random order, everything outside the
    sequences' positions filled with `outside` (NaN by default)."""

    def __init__(self, lens, H, K, D, P, dtype=torch.bfloat16, seed=0, outside=float("nan"), spare=3, table_pad=2, key_mean=0.4):
        g = torch.Generator().manual_seed(seed)
        self.lens, self.H, self.K, self.D, self.P, self.dtype, self.g = lens, H, K, D, P, dtype, g
        n = len(lens)
        blocks = [-(-kv // P) for _, kv in lens]
        self.n_pages = sum(blocks) + spare
        self.cols = max(blocks + [1]) + table_pad
        order = torch.randperm(self.n_pages, generator=g).tolist()
        self.pages = torch.full((n, self.cols), 2**31 - 1, dtype=torch.int32)        # entries past the length hold anything
        mean = torch.randn((K, 1, D), generator=g) * key_mean
        self.k_cache = torch.full((self.n_pages, K, P, D), outside).to(dtype)
        self.v_cache = torch.full((self.n_pages, K, P, D), outside).to(dtype)
        for i, (_, kv) in enumerate(lens):
            for j in range(blocks[i]):
                p = order.pop()
                self.pages[i, j] = p
                c = min(P, kv - j * P)
                self.k_cache[p, :, :c] = (torch.randn((K, c, D), generator=g) + 0.5 * torch.randn((K, 1, D), generator=g) + mean).to(dtype)
                self.v_cache[p, :, :c] = (torch.randn((K, c, D), generator=g) + 0.2 * mean).to(dtype)
        self.cu = [0]
        for q, _ in lens:
            self.cu.append(self.cu[-1] + q)
        self.T = self.cu[-1]
        self.q = torch.randn((self.T, H, D), generator=g).to(dtype)
        self.k = torch.randn((self.T, K, D), generator=g).to(dtype)
        self.v = torch.randn((self.T, K, D), generator=g).to(dtype)
        self.max_q = max([q for q, _ in lens] + [1])
        self.max_kv = max([kv for _, kv in lens] + [0])
        self.scale = D ** -0.5

    def rows(self):
        """(row, sequence, position) of every new row."""
        for i, (q, kv) in enumerate(self.lens):
            for r in range(q):
                yield self.cu[i] + r, i, kv - q + r

    def held(self, i, h, which):
        """Positions 0 .. kv of one head of a sequence in 64 bits."""
        kv = self.lens[i][1]
        c = self.k_cache if which == "k" else self.v_cache
        parts = [c[int(self.pages[i, j]), h, :min(self.P, kv - j * self.P)] for j in range(-(-kv // self.P))]
        return torch.cat(parts).double() if parts else torch.zeros((0, self.D), dtype=torch.float64)


def attention(s: Setup, causal=True, window=0, blocks=None, per_token=True, scale=None):
    """(out, lse) in 64 bits; rows that see nothing give 0 and -inf."""
    scale = s.scale if scale is None else scale
    out = torch.zeros((s.T, s.H, s.D), dtype=torch.float64)
    lse = torch.full((s.T, s.H), -math.inf, dtype=torch.float64)
    G = s.H // s.K
    for i, (n, kv) in enumerate(s.lens):
        if n == 0 or kv == 0:
            continue
        j = torch.arange(kv)
        pos = torch.arange(kv - n, kv)[:, None] if causal else torch.full((n, 1), kv - 1)
        base = j <= pos
        if window:
            base = base & (j > pos - window)
        for h in range(s.K):
            k, v = s.held(i, h, "k"), s.held(i, h, "v")
            see = base
            if blocks is not None:
                listed = torch.zeros((n, s.cols + 1), dtype=torch.bool)
                for r in range(n):
                    lst = (blocks[s.cu[i] + r] if per_token else blocks[i])[h if blocks.shape[1] > 1 else 0].tolist()
                    for b in lst:
                        if 0 <= b <= (kv - 1) // s.P:
                            listed[r, b] = True
                see = base & listed[:, j // s.P]
            for g in range(h * G, h * G + G):
                x = s.q[s.cu[i]:s.cu[i] + n, g].double() @ k.T * scale
                x = torch.where(see, x, -math.inf)
                some = see.any(1)
                w = torch.where(some[:, None], torch.softmax(x, -1), 0.0)
                out[s.cu[i]:s.cu[i] + n, g] = w @ v
                lse[s.cu[i]:s.cu[i] + n, g] = torch.logsumexp(x, -1)
    return out, lse


def rotate(x, cos, sin, rot, interleaved):
    """x [..., D] float64 by one table row."""
    y = x.clone()
    h = rot // 2
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if interleaved else (x[..., :h], x[..., h:rot])
    lo, hi = a * cos - b * sin, b * cos + a * sin
    if interleaved:
        y[..., 0:rot:2], y[..., 1:rot:2] = lo, hi
    else:
        y[..., :h], y[..., h:rot] = lo, hi
    return y


def summary(k):
    """(code, scale) of keys [positions, D] as the cache holds them: whole-number sums, the two roundings in fp32."""
    f = torch.nan_to_num(k.double(), nan=0.0, posinf=1e9, neginf=-1e9).clamp(-FAR, FAR) * STEPS
    total = torch.round(f).sum(0)
    most = total.abs().max()
    code = torch.round(total.float() * 127.0 / most.clamp(min=1).float()).to(torch.int8)
    return code, (most.float() / torch.tensor(float(k.shape[0]))).float()


def select(s: Setup, code, scale, n_sel, n_first, n_last):
    """Lists int32 [T, K, n_sel] from the host's copies of the summaries; integer scores, Python sorting."""
    G = s.H // s.K
    out = torch.full((s.T, s.K, n_sel), -1, dtype=torch.int32)
    for t, i, pos in s.rows():
        if pos < 0:
            continue
        for h in range(s.K):
            q = torch.round(s.q[t, h * G:(h + 1) * G].double().clamp(-FAR, FAR) * STEPS).sum(0)
            most = q.abs().max().clamp(min=1)
            c = torch.round(q.float() * 127.0 / most.float()).to(torch.int64)
            nb = pos // s.P + 1
            p = s.pages[i, :nb].long()
            dots = (code[p, h].to(torch.int64) * c).sum(-1)
            score = (dots.float() * scale[p, h]).tolist()
            key = [(0 if (j < n_first or j >= nb - n_last) else 1, -score[j], j) for j in range(nb)]
            forced_first = [(0, 0.0, j) if a == 0 else (a, b, j) for a, b, j in key]
            best = sorted(sorted(forced_first)[:n_sel], key=lambda z: z[2])
            for x, z in enumerate(best):
                out[t, h, x] = z[2]
    return out
