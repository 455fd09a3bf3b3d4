// What the kernels over a paged key / value cache share: the batch as they see it, the walk from a work item to its sequence,
// the launch parameters of the two attention kernels, and their PTX wrappers.
#pragma once

#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "s3_common.cuh"

namespace s3 {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kSumSteps = 4096.0f, kSumLimit = 2047.0f;   // fixed point of the summaries and of the summed queries

struct KvCacheState {
    s3_kv_cache_desc d;
    int page_shift;
    int box_rows;                                   // rows of one TMA box: min(page_size, 64)
    alignas(64) unsigned char map_k[128], map_v[128];
};

struct KvBatchDev {
    const int32_t* cu_q;
    const int32_t* kv_len;
    const int32_t* pages;
    int64_t ld_pages;
    int32_t n_seqs, T, max_q, max_kv;
};

// One sequence: rows [q0, q0 + n), kv cached positions; row r is at position kv - n + r.
struct SeqSpan {
    int q0, n, kv;
};

__device__ __forceinline__ SeqSpan load_seq(const KvBatchDev& b, int i, uint32_t* status)
{
    const int a0 = b.cu_q[i], a1 = b.cu_q[i + 1], len = b.kv_len[i];
    SeqSpan s;
    s.q0 = min(max(a0, 0), b.T);
    s.n = min(min(max(a1, s.q0), b.T) - s.q0, b.max_q);
    s.kv = min(max(len, 0), b.max_kv);
    if (status && (s.q0 != a0 || s.n != a1 - a0 || s.kv != len)) dev_set_error(status, DEV_BAD_BATCH);
    return s;
}

// Work item -> (sequence, item within it) when sequence i has count(i) items; run by a whole warp, every lane gets the
// result. False when there are fewer items.
template <class F>
__device__ __forceinline__ bool locate_item(int n_seqs, int item, F count, int& seq, int& idx)
{
    const int lane = threadIdx.x & 31;
    int base = 0;
    for (int i0 = 0; i0 < n_seqs; i0 += 32) {
        const int c = i0 + lane < n_seqs ? count(i0 + lane) : 0;
        int sum = c;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int up = __shfl_up_sync(0xffffffffu, sum, o);
            if (lane >= o) sum += up;
        }
        const uint32_t past = __ballot_sync(0xffffffffu, base + sum > item);
        if (past) {
            const int l = __ffs(past) - 1;
            seq = i0 + l;
            idx = item - (base + __shfl_sync(0xffffffffu, sum - c, l));
            return true;
        }
        base += __shfl_sync(0xffffffffu, sum, 31);
    }
    return false;
}

// The sequence of packed row t (the last one whose first row is <= t).
__device__ __forceinline__ int seq_of_row(const KvBatchDev& b, int t)
{
    int lo = 0, hi = b.n_seqs - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (b.cu_q[mid] <= t) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}

enum { LIST_NONE = 0, LIST_PER_TOKEN = 1, LIST_PER_SEQ = 2 };

// Launch parameters of the attention kernels. A thread block takes one (item, key head, split): an item is a run of
// tok_per_item new tokens of one sequence (with lists per token: one token), its query rows (token, head of the group)
// packed token by token; a split is a range of split_len virtual keys, counted from the first tile that the item sees. Virtual key v of an item is position
// block(v / page_size) * page_size + v % page_size, block(e) = e for the whole cache and = list[e] for a list.
struct AttnArgs {
    KvBatchDev b;
    int32_t n_heads, n_kv_heads, group, page_size, page_shift, box_rows, n_pages, head_dim;
    float scale, scale_log2;
    int32_t causal, window;
    const int32_t* lists;
    int32_t s, list_heads, list_mode;
    const void* q;
    int64_t ldq;
    void* out;
    int64_t ld_out;
    float* lse;
    float* part_o;              // [n_splits][T * n_heads][head_dim]
    float* part_lse;            // [n_splits][T * n_heads], base 2
    int32_t n_splits, split_len, tok_per_item, n_items, one_item_per_seq;
    uint32_t* status;
};

struct AttnItem {
    int seq, tok0, n_tok;       // first packed row, rows
    int pos0, kv;               // position of the first row, cached positions
    int list;                   // row of the lists
};

__device__ __forceinline__ bool attn_item(const AttnArgs& a, int item, AttnItem& it)
{
    if (a.list_mode == LIST_PER_TOKEN) {
        it.seq = seq_of_row(a.b, item);
        const SeqSpan s = load_seq(a.b, it.seq, a.status);
        it.tok0 = item;
        it.n_tok = item < s.q0 + s.n ? 1 : 0;
        it.kv = s.kv;
        it.pos0 = s.kv - s.n + (item - s.q0);
        it.list = item;
    } else {
        int idx = 0;
        if (a.one_item_per_seq) it.seq = item;
        else {
            const KvBatchDev& b = a.b;
            const int per = a.tok_per_item;
            if (!locate_item(b.n_seqs, item, [&](int i) { return (load_seq(b, i, nullptr).n + per - 1) / per; }, it.seq, idx)) return false;
        }
        const SeqSpan s = load_seq(a.b, it.seq, a.status);
        it.tok0 = s.q0 + idx * a.tok_per_item;
        it.n_tok = min(a.tok_per_item, s.n - idx * a.tok_per_item);
        it.kv = s.kv;
        it.pos0 = s.kv - s.n + idx * a.tok_per_item;
        it.list = it.seq;
    }
    if (!a.causal) it.pos0 = it.kv - 1;
    return it.n_tok > 0;
}

// ---- PTX wrappers -------------------------------------------------------------------------------
namespace kv {

constexpr uint32_t WAIT_LIMIT = 1u << 26;    // try_wait polls before a wait is declared dead (~1 s)

__device__ __forceinline__ uint32_t smem_u32(const void* p) { return static_cast<uint32_t>(__cvta_generic_to_shared(p)); }

__device__ __forceinline__ void mbar_init(uint64_t* bar, uint32_t count)
{
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(smem_u32(bar)), "r"(count) : "memory");
}
__device__ __forceinline__ void mbar_arrive(uint64_t* bar)
{
    asm volatile("{\n\t.reg .b64 st;\n\tmbarrier.arrive.shared::cta.b64 st, [%0];\n\t}" ::"r"(smem_u32(bar)) : "memory");
}
__device__ __forceinline__ void mbar_expect_tx(uint64_t* bar, uint32_t bytes)
{
    asm volatile("{\n\t.reg .b64 st;\n\tmbarrier.arrive.expect_tx.shared::cta.b64 st, [%0], %1;\n\t}" ::"r"(smem_u32(bar)), "r"(bytes)
                 : "memory");
}
// Bounded wait. Returns false if the wait ran out or another role already aborted (abort_flag null: not asked).
__device__ __forceinline__ bool mbar_wait(uint64_t* bar, uint32_t parity, volatile uint32_t* abort_flag)
{
    for (uint32_t it = 0; it < WAIT_LIMIT; ++it) {
        uint32_t ok;
        asm volatile(
            "{\n\t.reg .pred p;\n\t"
            "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
            "selp.u32 %0, 1, 0, p;\n\t}"
            : "=r"(ok)
            : "r"(smem_u32(bar)), "r"(parity)
            : "memory");
        if (ok) return true;
        if ((it & 1023u) == 1023u && abort_flag && *abort_flag) return false;
    }
    return false;
}

// Box of a 4-D map (column, row, head, page) into this block's shared memory; the column is 0 or 64, so every copy starts on a
// 16-byte boundary.
__device__ __forceinline__ void tma_load_4d(void* dst, const void* map, int c0, int c1, int c2, int c3, uint64_t* bar)
{
    asm volatile(
        "cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(
            smem_u32(dst)),
        "l"(reinterpret_cast<uint64_t>(map)), "r"(c0), "r"(c1), "r"(c2), "r"(c3), "r"(smem_u32(bar))
        : "memory");
}

__device__ __forceinline__ void fence_async_smem() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

__device__ __forceinline__ float ex2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

template <class T>
struct Half2Of;
template <>
struct Half2Of<__nv_bfloat16> {
    static constexpr bool is_bf16 = true;
    static __device__ __forceinline__ uint32_t pack(float lo, float hi)
    {
        uint32_t r;
        asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
        return r;
    }
    static __device__ __forceinline__ float lo(uint32_t v) { return __uint_as_float(v << 16); }
    static __device__ __forceinline__ float hi(uint32_t v) { return __uint_as_float(v & 0xffff0000u); }
};
template <>
struct Half2Of<__half> {
    static constexpr bool is_bf16 = false;
    static __device__ __forceinline__ uint32_t pack(float lo, float hi)
    {
        uint32_t r;
        asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
        return r;
    }
    static __device__ __forceinline__ float lo(uint32_t v) { return __half2float(__ushort_as_half(static_cast<unsigned short>(v & 0xffffu))); }
    static __device__ __forceinline__ float hi(uint32_t v) { return __half2float(__ushort_as_half(static_cast<unsigned short>(v >> 16))); }
};

__device__ __forceinline__ int fixed_of(float x)
{
    if (x != x) return 0;
    return __float2int_rn(__fmul_rn(fminf(fmaxf(x, -kSumLimit), kSumLimit), kSumSteps));
}

}  // namespace kv
}  // namespace s3
