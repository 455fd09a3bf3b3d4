"""One attention layer answering from evidence: a long context is scanned chunk by chunk, a question attends to the evidence spans
that the inverted index returns for it, and the answer's tokens attend to the blocks that a cheap score picks for each.

    python examples/evidence_attention.py [--context 16384] [--chunk 2048]

Per chunk: projections (s3_sae_preact), append to the paged cache with rotation and block summaries (s3_kv_append), attention of
the chunk over everything before it (s3_paged_attention), and the scan itself: Top-k codes of the keys, postings, host index.
Question: span scores by co-activation, spans 64 wide = one page each, attention over them and the question's own block
(s3_block_attention, one list per sequence). Answer: s3_block_select + s3_block_attention per token. Synthetic weights and
hidden states; one stretch of the context is about what the question is about."""
from __future__ import annotations

import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2601_17702_b200 as S  # noqa: E402

HEADS, KV_HEADS, DIM, PAGE = 32, 8, 128, 64
D_MODEL, D_SAE, TOP_K = 1024, 4096, 16


class Layer:
    def __init__(self, max_tokens: int, seed: int = 0, device="cuda"):
        g = torch.Generator(device=device).manual_seed(seed)
        rand = lambda *shape: torch.randn(shape, generator=g, device=device)
        zeros = lambda n: torch.zeros(n, device=device)
        width = (HEADS + 2 * KV_HEADS) * DIM
        w = rand(D_MODEL, width) / math.sqrt(D_MODEL)
        w[:, :HEADS * DIM] = (w[:, HEADS * DIM:(HEADS + KV_HEADS) * DIM].view(D_MODEL, KV_HEADS, 1, DIM) * 1.5
                              + 0.5 * w[:, :HEADS * DIM].view(D_MODEL, KV_HEADS, -1, DIM)).reshape(D_MODEL, -1)   # queries that look for like keys
        self.proj = S.Sae(w.bfloat16(), zeros(width), zeros(D_MODEL))
        enc = rand(KV_HEADS * DIM, D_SAE) / math.sqrt(KV_HEADS * DIM)
        self.sae = S.Sae(enc.bfloat16(), zeros(D_SAE), zeros(KV_HEADS * DIM))
        pages = -(-max_tokens // PAGE)
        self.cache = S.KvCache.zeros(pages, KV_HEADS, PAGE, DIM)
        self.table = torch.randperm(pages, generator=g, device=device).to(torch.int32).view(1, pages)
        angle = torch.arange(max_tokens, dtype=torch.float64)[:, None] * 500000.0 ** (-torch.arange(0, DIM, 2, dtype=torch.float64) / DIM)
        self.rope = S.Rope(angle.cos().float().to(device), angle.sin().float().to(device))
        self.index = S.Index(1, D_SAE)
        self.n = 0
        self.device = device
        self.ws = S.new_workspace(1 << 20, device)

    def _room(self, n_bytes: int):
        if self.ws.numel() < n_bytes:
            self.ws = S.new_workspace(n_bytes, self.device)
        return self.ws

    def _qkv(self, h: torch.Tensor):
        """The heads' queries, keys and values as slices of one fused projection."""
        T = h.shape[0]
        out = torch.empty((T, self.proj.d_sae), dtype=torch.bfloat16, device=self.device)
        S.s3_sae_preact(self.proj, h, torch.bfloat16, out, self.ws)
        a, b = HEADS * DIM, (HEADS + KV_HEADS) * DIM
        return out[:, :a].view(T, HEADS, DIM), out[:, a:b].view(T, KV_HEADS, DIM), out[:, b:].view(T, KV_HEADS, DIM), out[:, a:b]

    def _codes(self, keys: torch.Tensor):
        T = keys.shape[0]
        ids = torch.empty((T, TOP_K), dtype=torch.int32, device=self.device)
        vals = torch.empty((T, TOP_K), dtype=torch.float32, device=self.device)
        S.s3_sae_encode_topk(self.sae, keys, TOP_K, ids, vals, self._room(self.sae.encode_workspace_bytes(T, TOP_K)))
        return ids, vals

    def _append(self, q, k, v):
        """The new tokens enter the cache; returns their batch and rotated queries."""
        T = q.shape[0]
        self.n += T
        i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device=self.device)
        batch = S.KvBatch(i32(0, T), i32(self.n), self.table, T, T, self.n)
        self._room(S.s3_kv_workspace_bytes(self.cache, batch, HEADS))
        return batch, S.s3_kv_append(self.cache, batch, k, v, self.ws, q=q, rope=self.rope)

    def scan_chunk(self, h: torch.Tensor) -> torch.Tensor:
        """Attention of a chunk of the context over all tokens so far; its keys' codes go to the index."""
        T, base = h.shape[0], self.n
        q, k, v, keys = self._qkv(h)
        ids, _ = self._codes(keys)
        row_ptr = torch.zeros(D_SAE + 1, dtype=torch.int32, device=self.device)
        pos = torch.zeros(T * TOP_K, dtype=torch.int32, device=self.device)
        S.s3_postings_build(ids, D_SAE, base, row_ptr, pos, self._room(S.s3_postings_workspace_bytes(T, TOP_K, D_SAE)))
        self.index.append(0, row_ptr, pos, T, TOP_K, base)
        self.index.stream_wait()
        batch, q = self._append(q, k, v)
        return S.s3_paged_attention(self.cache, batch, q, self.ws)[0]

    def ask(self, h: torch.Tensor, spans: int):
        """Attention of a question over its `spans` best evidence spans and its own tokens. Returns (output, the same over the whole
        cache, the spans)."""
        L = self.n
        assert L % PAGE == 0, "the question starts on a page of its own"
        q, k, v, keys = self._qkv(h)
        ids, vals = self._codes(keys)
        row_ptr, pos, _ = self.index.export_csr(0)
        top, _ = S.s3_coactivation_score_topspans([(row_ptr.to(self.device), pos.to(self.device))], D_SAE, L, ids[None, None], vals[None, None],
                                                  PAGE, PAGE, spans, 1.0, 0.0,
                                                  self._room(S.s3_score_workspace_bytes(1, h.shape[0], TOP_K, 1, L // PAGE, spans)))
        batch, q = self._append(q, k, v)
        own = torch.arange(L // PAGE, -(-self.n // PAGE), dtype=torch.int32, device=self.device)
        blocks = torch.cat([top[0], own]).view(1, 1, -1)
        out, _ = S.s3_block_attention(self.cache, batch, q, blocks, self.ws, per_token=False)
        return out, S.s3_paged_attention(self.cache, batch, q, self.ws)[0], top[0]

    def step(self, h: torch.Tensor, blocks: int):
        """One token of the answer over the blocks selected for it. Returns (output, the same over the whole cache, the blocks)."""
        q, k, v, _ = self._qkv(h)
        batch, q = self._append(q, k, v)
        chosen = S.s3_block_select(self.cache, batch, q, blocks, self.ws)
        out, _ = S.s3_block_attention(self.cache, batch, q, chosen, self.ws)
        return out, S.s3_paged_attention(self.cache, batch, q, self.ws)[0], chosen[0]


def run(context: int = 16384, chunk: int = 2048, spans: int = 16, steps: int = 4, seed: int = 0):
    """Returns the cosine of the evidence attention with attention over everything for the question and for the answer's tokens, and
    whether the stretch that the question is about is among its spans."""
    g = torch.Generator(device="cuda").manual_seed(seed + 1)
    layer = Layer(context + 1024, seed)
    h = torch.randn((context, D_MODEL), generator=g, device="cuda")
    where = context // 3 // PAGE * PAGE
    topic = torch.randn((1, D_MODEL), generator=g, device="cuda")
    h[where:where + PAGE] = 0.4 * h[where:where + PAGE] + topic
    for c in range(0, context, chunk):
        layer.scan_chunk(h[c:c + chunk].bfloat16())
    layer.index.sync()
    cosine = lambda a, b: float(torch.nn.functional.cosine_similarity(a.float().flatten(1), b.float().flatten(1)).mean())
    out, full, top = layer.ask((0.4 * torch.randn((24, D_MODEL), generator=g, device="cuda") + topic).bfloat16(), spans)
    question, found = cosine(out, full), where // PAGE in top.tolist()
    answer = []
    for _ in range(steps):
        out, full, chosen = layer.step((0.4 * torch.randn((1, D_MODEL), generator=g, device="cuda") + topic).bfloat16(), spans)
        answer.append(cosine(out, full))
    assert S.s3_workspace_status(layer.ws) == 0
    layer.index.close()
    return question, answer, found


if __name__ == "__main__":
    ap = argparse.ArgumentParser()
    ap.add_argument("--context", type=int, default=16384)
    ap.add_argument("--chunk", type=int, default=2048)
    a = ap.parse_args()
    question, answer, found = run(a.context, a.chunk)
    print(f"context of {a.context} tokens: the stretch asked about is {'among' if found else 'NOT among'} the evidence spans")
    print(f"question over 16 spans against the whole context: cosine {question:.4f}")
    print("answer over 16 selected blocks: cosine " + ", ".join(f"{x:.4f}" for x in answer))
