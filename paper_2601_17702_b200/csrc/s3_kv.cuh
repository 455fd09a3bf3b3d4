// What the kernels over a paged key / value cache share: the batch as they see it, the walk from a work item to its sequence,
// the launch parameters of the two attention kernels, and their PTX wrappers.
#pragma once

#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <atomic>
#include <utility>

#include "s3_common.cuh"

namespace s3 {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kSumSteps = 4096.0f, kSumLimit = 2047.0f;   // fixed point of the summaries and of the summed queries

// Launch that may begin while the kernel before it in the stream ends (programmatic launch): its blocks set themselves up, and
// cudaGridDependencySynchronize() in the kernel waits for that kernel's end before anything it may have written is read, or
// anything it may still read is written. Worth about a microsecond per call where calls are short. What an earlier kernel may have
// written is read with ordinary loads: __ldg (ld.global.nc) asks for memory that nobody writes while the kernel lives, and these
// kernels live while the one before them still writes. Only the rotation tables are read that way.
template <class... Params, class... Args>
inline s3_status launch_overlapped(void (*kernel)(Params...), dim3 grid, int threads, size_t smem, cudaStream_t stream, Args&&... args)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    S3_CUDA_TRY(cudaLaunchKernelEx(&cfg, kernel, std::forward<Args>(args)...));
    return S3_OK;
}

// Lets a kernel use `bytes` of dynamic shared memory; asked once per kernel and device.
template <auto Kernel>
inline s3_status allow_smem(int bytes)
{
    static std::atomic<uint64_t> done{0};
    int dev = 0;
    S3_CUDA_TRY(cudaGetDevice(&dev));
    const uint64_t bit = dev < 64 ? uint64_t(1) << dev : 0;
    if (!(done.load(std::memory_order_relaxed) & bit)) {
        S3_CUDA_TRY(cudaFuncSetAttribute(Kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes));
        done.fetch_or(bit, std::memory_order_relaxed);
    }
    return S3_OK;
}

struct KvCacheState {
    s3_kv_cache_desc d;
    int page_shift;
    int box_rows;                                   // rows of one TMA box: min(page_size, 64)
    alignas(64) unsigned char map_k[128], map_v[128];     // (column, row, head, page), box 64 columns
    alignas(64) unsigned char wide_k[128], wide_v[128];   // (column of a half, row, half, head, page), box whole rows
    // 8-bit pages: map_k / map_v are of bytes, box whole rows; scales [page][head][row]
    float *k_scale, *v_scale;                       // null: 16-bit pages
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

constexpr int kMaxMaskWords = 128;      // 4096 blocks

enum { LIST_NONE = 0, LIST_PER_TOKEN = 1, LIST_PER_SEQ = 2 };

// Launch parameters of the attention kernels.
//
// An item is a run of tok_per_item new tokens of one sequence (with lists per token: one token); its query rows under one key
// head, (token, head of the group) packed token by token, are worked on together. Keys are counted virtually: virtual key v is
// position block(v / page_size) * page_size + v % page_size, block(e) = e for the whole cache and = list[e] for a list, and
// are taken in tiles from the first one that some row of the item sees.
//
// Lists per token have a second form, for chunks whose lists cover a good part of a short context: the keys are counted as for the
// whole cache, a bit per token and block says who may see it (masks), and blocks that no token of an item lists (unions) count as
// not there: they are neither looked up nor read. A key tile then serves an item's rows instead of a token's.
//
// The grid's thread blocks share the work in one of two ways, which the host chooses:
//   share = 0   unit u = (key head, item), whole, goes to block u mod grid; key head by key head, so that the blocks are at work on
//               the keys of one head or two, which the L2 cache holds when a token's list picks among many (1024 tokens x 16 of
//               512 blocks: 359 -> 333 us);
//   share > 0   the tiles of all units, laid end to end (key head by key head, item by item), are cut into equal shares of `share`
//               tiles or less, one per block, whatever the lengths are. A unit that a cut divides is worked on in pieces; a
//               piece's result goes to a slot of its block (each has at most two pieces: one that began before its share and
//               one that ends after it) and the join kernel adds the pieces up.
struct AttnArgs {
    KvBatchDev b;
    int32_t n_heads, n_kv_heads, group, page_size, page_shift, box_rows, n_pages, head_dim;
    float scale_log2;
    int32_t causal, window;
    // forms of the score, see s3_score_form, in base 2: cap2 > 0: cap2 tanh(dot score_in), else dot score_in
    float score_in, cap2;
    const float* slopes;        // null: none
    const int32_t* prefix;      // null: none
    const float *k_scale, *v_scale;     // 8-bit pages
    const int32_t* lists;
    int32_t s, list_heads, list_mode;
    uint32_t* masks;            // [T][list_heads][mask_words] or null
    uint32_t* unions;           // [item_number()][list_heads][mask_words]
    int32_t mask_words;
    const void* q;
    int64_t ldq;
    void* out;
    int64_t ld_out;
    float* lse;
    float* part_o;              // [2 * grid][rows_cap][head_dim]
    float* part_lse;            // [2 * grid][rows_cap], base 2
    int32_t* cuts;              // [grid][8]: the unit that the cut behind a block's share divides first, see Cut
    int32_t grid, share_min, whole_rounds, rows_cap, tok_per_item, n_items, one_item_per_seq;
    uint32_t* status;
    uint8_t* redo;              // [grid] or null: blocks whose results have to be made again, see FORM_BOUNDED in s3_attn_tile.cuh
};

struct AttnItem {
    int seq, tok0, n_tok;       // first packed row, rows
    int pos0, pos_last, kv;     // positions of the first and last row, cached positions
    int row0, prefix, end;      // first row's own position, positions open to all rows, positions that some row may see
    int list;                   // row of the lists
};

__device__ __forceinline__ AttnItem make_item(const AttnArgs& a, int seq, const SeqSpan& s, int idx)
{
    AttnItem it;
    it.seq = seq;
    it.tok0 = s.q0 + idx * a.tok_per_item;
    it.n_tok = max(min(a.tok_per_item, s.n - idx * a.tok_per_item), 0);
    it.kv = s.kv;
    it.pos0 = a.causal ? s.kv - s.n + idx * a.tok_per_item : s.kv - 1;
    it.pos_last = a.causal ? it.pos0 + it.n_tok - 1 : it.pos0;
    it.row0 = s.kv - s.n + idx * a.tok_per_item;
    it.prefix = a.prefix ? min(max(a.prefix[seq], 0), s.kv) : 0;
    it.end = it.pos_last < 0 ? it.pos_last + 1 : max(it.pos_last + 1, it.prefix);
    it.list = a.list_mode == LIST_PER_TOKEN ? it.tok0 : seq;
    return it;
}

// A number of its own for every item: first rows rise by tok_per_item within a sequence, and do not fall from one to the next.
__device__ __forceinline__ int item_number(const AttnArgs& a, const AttnItem& it) { return it.tok0 / a.tok_per_item + it.seq; }

// First position that some row of the item may see.
__device__ __forceinline__ int first_seen(const AttnArgs& a, const AttnItem& it)
{
    return a.window > 0 ? max(it.pos0 - a.window + 1, 0) : 0;
}

// Key tiles of an item, at least one (rows that see nothing still have a result to write).
template <int TILE>
__device__ __forceinline__ int item_tiles(const AttnArgs& a, const AttnItem& it)
{
    const int keys = a.list_mode == LIST_NONE ? it.end - (first_seen(a, it) & ~(TILE - 1)) : a.s << a.page_shift;
    return max((keys + TILE - 1) / TILE, 1);
}

__device__ __forceinline__ int seq_items(const AttnArgs& a, const SeqSpan& s)
{
    return (s.n + a.tok_per_item - 1) / a.tok_per_item;
}

// Item number -> item; a whole warp. False when there is no such item.
__device__ __forceinline__ bool attn_item(const AttnArgs& a, int item, AttnItem& it)
{
    int seq = item, idx = 0;
    if (a.list_mode == LIST_PER_TOKEN) {
        seq = seq_of_row(a.b, item);
        const SeqSpan s = load_seq(a.b, seq, a.status);
        if (item < s.q0 || item >= s.q0 + s.n) return false;
        it = make_item(a, seq, s, item - s.q0);
        return true;
    }
    if (!a.one_item_per_seq &&
        !locate_item(a.b.n_seqs, item, [&](int i) { return seq_items(a, load_seq(a.b, i, nullptr)); }, seq, idx)) return false;
    it = make_item(a, seq, load_seq(a.b, seq, a.status), idx);
    return it.n_tok > 0;
}

// sum of floor((a i + b) / m) for i in [0, n), with a n + b < 2^32, m > 0. Each step takes out the whole parts and swaps the roles of
// the two axes of the lattice, as in Euclid's algorithm.
__device__ __forceinline__ int64_t floor_sum(uint32_t n, uint32_t m, uint32_t a, uint32_t b)
{
    int64_t sum = 0;
    for (;;) {
        const uint32_t qa = a / m, qb = b / m;
        sum += static_cast<int64_t>(n) * (n - 1) / 2 * qa + static_cast<int64_t>(n) * qb;
        a -= qa * m;
        b -= qb * m;
        const uint32_t top = a * n + b;
        if (top < m) return sum;
        n = top / m;
        b = top - n * m;
        const uint32_t t = a;
        a = m;
        m = t;
    }
}

// Tiles of one key head over the items of sequence i.
template <int TILE>
__device__ __forceinline__ int64_t seq_tiles(const AttnArgs& a, int i, const SeqSpan& s)
{
    const int items = seq_items(a, s);
    if (items == 0) return 0;
    const int last = item_tiles<TILE>(a, make_item(a, i, s, items - 1));
    if (items == 1) return last;
    if (a.list_mode != LIST_NONE || !a.causal) return static_cast<int64_t>(items) * last;
    if (a.window == 0 && s.kv >= s.n && !a.prefix)          // all but the last item are full: item x ends before position kv - n + (x + 1) per
        return last + floor_sum(items - 1, TILE, a.tok_per_item, s.kv - s.n + a.tok_per_item + TILE - 1);
    int64_t sum = last;
    for (int x = 0; x < items - 1; ++x) sum += item_tiles<TILE>(a, make_item(a, i, s, x));
    return sum;
}

__device__ __forceinline__ int64_t divide(int64_t a, int64_t b)        // of non-negative numbers, mostly small ones
{
    return ((a | b) >> 32) == 0 ? static_cast<uint32_t>(a) / static_cast<uint32_t>(b) : a / b;
}

// Sequences of a batch, 32 at a time, one per lane: lengths and the tiles up to and with each.
struct SeqLanes {
    SeqSpan span;
    int64_t tiles, upto;
};

template <int TILE>
__device__ __forceinline__ SeqLanes load_lanes(const AttnArgs& a, int i0)
{
    const int lane = threadIdx.x & 31;
    SeqLanes q;
    q.span = SeqSpan{0, 0, 0};
    if (i0 + lane < a.b.n_seqs) q.span = load_seq(a.b, i0 + lane, a.status);
    q.tiles = seq_tiles<TILE>(a, i0 + lane, q.span);
    q.upto = q.tiles;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int64_t up = __shfl_up_sync(0xffffffffu, q.upto, o);
        if (lane >= o) q.upto += up;
    }
    return q;
}

// The item that holds tile number r of a key head, the number of its first tile and its tiles; a whole warp. `lanes` holds the
// first 32 sequences. False: no such tile.
template <int TILE>
__device__ __forceinline__ bool locate_tile(const AttnArgs& a, const SeqLanes& lanes, int64_t r, AttnItem& it, int64_t& first, int& n)
{
    const int lane = threadIdx.x & 31;
    if (a.list_mode == LIST_PER_TOKEN) {
        n = ((a.s << a.page_shift) + TILE - 1) / TILE;
        const int64_t item = divide(r, n);
        first = item * n;
        if (item >= a.b.T) return false;
        const int seq = seq_of_row(a.b, static_cast<int>(item));
        const SeqSpan s = load_seq(a.b, seq, a.status);
        it = make_item(a, seq, s, static_cast<int>(item) - s.q0);
        if (item < s.q0 || item >= s.q0 + s.n) it.n_tok = 0;
        return true;
    }
    SeqLanes q = lanes;
    int64_t base = 0;
    for (int i0 = 0; i0 < a.b.n_seqs; i0 += 32) {
        if (i0 > 0) q = load_lanes<TILE>(a, i0);
        const uint32_t past = __ballot_sync(0xffffffffu, base + q.upto > r);
        if (!past) {
            base += __shfl_sync(0xffffffffu, q.upto, 31);
            continue;
        }
        const int l = __ffs(past) - 1;
        base += __shfl_sync(0xffffffffu, q.upto - q.tiles, l);
        const SeqSpan s{__shfl_sync(0xffffffffu, q.span.q0, l), __shfl_sync(0xffffffffu, q.span.n, l), __shfl_sync(0xffffffffu, q.span.kv, l)};
        const int items = seq_items(a, s);
        if (items == 1) {
            first = base;
            n = static_cast<int>(__shfl_sync(0xffffffffu, q.tiles, l));
            it = make_item(a, i0 + l, s, 0);
            return true;
        }
        for (int x0 = 0; x0 < items; x0 += 32) {
            const int c = x0 + lane < items ? item_tiles<TILE>(a, make_item(a, i0 + l, s, x0 + lane)) : 0;
            int sum = c;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int up = __shfl_up_sync(0xffffffffu, sum, o);
                if (lane >= o) sum += up;
            }
            const uint32_t over = __ballot_sync(0xffffffffu, base + sum > r);
            if (over) {
                const int k = __ffs(over) - 1;
                n = __shfl_sync(0xffffffffu, c, k);
                first = base + __shfl_sync(0xffffffffu, sum - c, k);
                it = make_item(a, i0 + l, s, x0 + k);
                return true;
            }
            base += __shfl_sync(0xffffffffu, sum, 31);
        }
        return false;
    }
    return false;
}

// A piece of work of one thread block: tiles [t_lo, t_hi) of a unit; slot < 0: the whole unit.
struct Segment {
    AttnItem it;
    int head, t_lo, t_hi, v_base, slot;
};

// What a thread block leaves for the join: the unit that began in its share and went on behind it (n_tok 0: there is none) and
// the block that holds its last piece.
struct Cut {
    int32_t tok0, n_tok, head, last;
    int32_t unused[4];
};

// Walks a block's segments; every call by a whole warp.
template <int TILE>
struct Walk {
    int64_t per_head, share, at, end;       // share > 0: tile numbers; share 0: unit numbers
    int64_t unit, unit_end;                 // share > 0: units of the whole rounds before the shares
    int64_t origin;                         // and the tile number where the shares begin
    SeqLanes lanes;
    Cut cut;

    __device__ __forceinline__ void start(const AttnArgs& a)
    {
        share = 0;
        cut = Cut{0, 0, 0, 0, {0, 0, 0, 0}};
        if (a.share_min > 0) {
            if (a.list_mode == LIST_PER_TOKEN) per_head = static_cast<int64_t>(a.b.T) * (((a.s << a.page_shift) + TILE - 1) / TILE);
            else {
                lanes = load_lanes<TILE>(a, 0);
                per_head = __shfl_sync(0xffffffffu, lanes.upto, 31);
                for (int i0 = 32; i0 < a.b.n_seqs; i0 += 32) per_head += __shfl_sync(0xffffffffu, load_lanes<TILE>(a, i0).upto, 31);
            }
            const int64_t total = per_head * a.n_kv_heads;
            unit = blockIdx.x;
            unit_end = static_cast<int64_t>(a.whole_rounds) * a.grid;
            origin = 0;
            if (unit_end > 0) {                                       // one sequence: its items before the first that is shared
                const int64_t head = divide(unit_end, a.n_items);
                const SeqSpan s{__shfl_sync(0xffffffffu, lanes.span.q0, 0), __shfl_sync(0xffffffffu, lanes.span.n, 0), __shfl_sync(0xffffffffu, lanes.span.kv, 0)};
                const int before = min(static_cast<int>(unit_end - head * a.n_items), seq_items(a, s));
                int64_t sum = 0;
                for (int x = threadIdx.x & 31; x < before; x += 32) sum += item_tiles<TILE>(a, make_item(a, 0, s, x));
#pragma unroll
                for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
                origin = head * per_head + sum;
            }
            share = max(divide(max(total - origin, int64_t(0)) + a.grid - 1, a.grid), static_cast<int64_t>(a.share_min));
            at = origin + blockIdx.x * share;
            end = min(at + share, total);
        } else {
            at = blockIdx.x;
            end = static_cast<int64_t>(a.n_items) * a.n_kv_heads;
        }
    }
    __device__ __forceinline__ bool next(const AttnArgs& a, Segment& g)
    {
        while (share > 0 && unit < unit_end) {
            g.head = static_cast<int>(divide(unit, a.n_items));
            const bool some = attn_item(a, static_cast<int>(unit - static_cast<int64_t>(g.head) * a.n_items), g.it);
            unit += a.grid;
            if (!some) continue;
            g.t_lo = 0;
            g.t_hi = item_tiles<TILE>(a, g.it);
            g.slot = -1;
            g.v_base = a.list_mode == LIST_NONE ? first_seen(a, g.it) & ~(TILE - 1) : 0;
            return true;
        }
        while (at < end) {
            if (share == 0) {
                g.head = static_cast<int>(divide(at, a.n_items));
                const bool some = attn_item(a, static_cast<int>(at - static_cast<int64_t>(g.head) * a.n_items), g.it);
                at += a.grid;
                if (!some) continue;
                g.t_lo = 0;
                g.t_hi = item_tiles<TILE>(a, g.it);
                g.slot = -1;
            } else {
                int64_t first;
                int n;
                g.head = static_cast<int>(divide(at, per_head));
                const int64_t head_at = g.head * per_head;
                if (!locate_tile<TILE>(a, lanes, at - head_at, g.it, first, n)) return false;
                first += head_at;
                g.t_lo = static_cast<int>(at - first);
                g.t_hi = static_cast<int>(min(first + n, end) - first);
                const bool whole = g.t_lo == 0 && g.t_hi == n;
                g.slot = whole ? -1 : 2 * static_cast<int>(blockIdx.x) + (first + n > end ? 1 : 0);
                if (first + n > end && first >= origin + blockIdx.x * share)
                    cut = Cut{g.it.tok0, g.it.n_tok, g.head, static_cast<int32_t>(divide(first + n - 1 - origin, share)), {0, 0, 0, 0}};
                at = first + g.t_hi;
                if (g.it.n_tok <= 0) continue;
            }
            g.v_base = a.list_mode == LIST_NONE ? first_seen(a, g.it) & ~(TILE - 1) : 0;
            return true;
        }
        return false;
    }
    // Once all segments have been taken; one thread.
    __device__ __forceinline__ void leave_cut(const AttnArgs& a) const
    {
        if (share > 0) reinterpret_cast<Cut*>(a.cuts)[blockIdx.x] = cut;
    }
};

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

// Box of a 5-D map (column of a half, row, half, head, page): all columns of its rows, half by half.
__device__ __forceinline__ void tma_load_rows(void* dst, const void* map, int row, int head, int page, uint64_t* bar)
{
    asm volatile(
        "cp.async.bulk.tensor.5d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %2, %4, %5}], [%6];" ::"r"(
            smem_u32(dst)),
        "l"(reinterpret_cast<uint64_t>(map)), "r"(0), "r"(row), "r"(head), "r"(page), "r"(smem_u32(bar))
        : "memory");
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

// Untiled copy of bytes (a multiple of 16, both addresses on 16-byte boundaries) into this block's shared memory.
__device__ __forceinline__ void bulk_load(void* dst, const void* src, uint32_t bytes, uint64_t* bar)
{
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(smem_u32(dst)), "l"(src),
                 "r"(bytes), "r"(smem_u32(bar)) : "memory");
}

__device__ __forceinline__ void prefetch_map(const void* map)
{
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(map)) : "memory");
}
// Asks for the tables and lists of a launch, spread over its blocks' producer warps, so that the dependent reads (lengths, list,
// table, keys) do not each wait for memory.
__device__ __forceinline__ void prefetch_tables(const AttnArgs& a)
{
    const int64_t line = blockIdx.x * 32 + (threadIdx.x & 31);
    auto ask = [&](const int32_t* p, int64_t words) {
        if (line * 32 < words) asm volatile("prefetch.global.L2 [%0];" ::"l"(p + line * 32));
    };
    ask(a.b.pages, (a.b.n_seqs - 1) * a.b.ld_pages + ((a.b.max_kv + a.page_size - 1) >> a.page_shift));
    if (a.list_mode != LIST_NONE)
        ask(a.lists, static_cast<int64_t>(a.list_mode == LIST_PER_TOKEN ? a.b.T : a.b.n_seqs) * a.list_heads * a.s);
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
__device__ __forceinline__ float rcp(float x)
{
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float lg2(float x)
{
    float y;
    asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// tanh(z) / z = sum tanh_part<N>(i) z^2i, by the polynomial of degree N - 1 in z^2 whose largest relative error is smallest (found by the
// exchange of its extrema): N = 7 for |z| <= 1, off by 5e-8, N = 5 for |z| <= 1/2, off by 1.3e-8; evaluated in fp32 below 2e-7. No special
// function, and exact to the last bits for small z.
template <int N>
__device__ __forceinline__ constexpr float tanh_part(int i)
{
    if (N == 5) return i == 0 ? 9.999999869e-01f : i == 1 ? -3.333306939e-01f : i == 2 ? 1.332477932e-01f : i == 3 ? -5.298607529e-02f : 1.713500663e-02f;
    return i == 0 ? 9.999999502e-01f : i == 1 ? -3.333283915e-01f : i == 2 ? 1.332520408e-01f : i == 3 ? -5.345702956e-02f : i == 4 ? 2.028998042e-02f
         : i == 5 ? -6.203379098e-03f : 1.041022631e-03f;
}
// tanh(z) is that of seven terms for |z| <= 1, else by tanh(z) = 1 - 2 / (1 + e^2z), which is off by 2^-22: of little beside the result where |z| > 1, of all of it
// where z is small (a cap of 1e6 over scores of 2 takes every z there).
__device__ __forceinline__ float tanh_near(float z)
{
    const float w = z * z;
    float y = tanh_part<7>(6);
#pragma unroll
    for (int i = 5; i >= 0; --i) y = fmaf(y, w, tanh_part<7>(i));
    return y * z;
}
__device__ __forceinline__ float tanh_far(float z) { return fmaf(-2.0f, rcp(1.0f + ex2(2.0f * kLog2e * z)), 1.0f); }
__device__ __forceinline__ float tanh_any(float z) { return fabsf(z) <= 1.0f ? tanh_near(z) : tanh_far(z); }
// tanh of a few scores per lane; the vote saves the second form and changes no bit of the first.
template <int N>
__device__ __forceinline__ void tanh_of_few(float (&z)[N])
{
    bool far = false;
#pragma unroll
    for (int i = 0; i < N; ++i) far |= fabsf(z[i]) > 1.0f;
    if (__any_sync(0xffffffffu, far)) {
#pragma unroll
        for (int i = 0; i < N; ++i) z[i] = tanh_any(z[i]);
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) z[i] = tanh_near(z[i]);
    }
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

// 8-bit pages. Rows whose largest magnitude is below 2^-60 are held as zeros with scale 0, magnitudes beyond 2^60 (f16: 65504) count as that.
// So a value's scale lies within 2^-67 and 2^53 (f16: 2^-31 and 2^9) and may be part of its weight's exponent, 2^(score + log2 scale), without
// leaving fp32. A scale of 0 has no logarithm: its key enters with the smallest scale instead, which raises no reference that another value
// needs, and its codes count as 0, as do those of a scale that no append writes because it is smaller than the smallest.
constexpr float kLeastMagnitude = 8.673617379884035e-19f, kMostBf16 = 1.152921504606847e18f, kMostF16 = 65504.0f;
template <class T>
constexpr float kLeastScale = Half2Of<T>::is_bf16 ? 6.776263578034403e-21f : 4.656612873077393e-10f;       // 2^-67; 2^-24 / 127 > 2^-31

// Four codes (int8) of a word -> two pairs of the type, without rounding: the bytes are put into the low bits of a number whose last
// place is 1, which a subtraction takes off. f16 1024 + (code + 128) - 1152; bf16, whose last place at 128 is 1 and which
// has seven of them: (128 + low seven bits) - (128, or 256 for a negative code).
__device__ __forceinline__ uint32_t bytes_of(uint32_t a, uint32_t b, uint32_t pick)
{
    uint32_t r;
    asm("prmt.b32 %0, %1, %2, %3;" : "=r"(r) : "r"(a), "r"(b), "r"(pick));
    return r;
}
__device__ __forceinline__ uint32_t sub_f16x2(uint32_t a, uint32_t b)
{
    uint32_t r;
    asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ uint32_t sub_bf16x2(uint32_t a, uint32_t b)
{
    uint32_t r;
    asm("sub.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
template <class T>
__device__ __forceinline__ void widen(uint32_t codes, uint32_t& lo, uint32_t& hi)
{
    if constexpr (Half2Of<T>::is_bf16) {
        const uint32_t x = bytes_of(codes, 0x43434343u, 0x4140u), y = bytes_of(codes, 0x43434343u, 0x4342u);
        lo = sub_bf16x2(x & 0xff7fff7fu, x & 0xff80ff80u);
        hi = sub_bf16x2(y & 0xff7fff7fu, y & 0xff80ff80u);
    } else {
        const uint32_t u = codes ^ 0x80808080u;
        lo = sub_f16x2(bytes_of(u, 0x64646464u, 0x4140u), 0x64806480u);
        hi = sub_f16x2(bytes_of(u, 0x64646464u, 0x4342u), 0x64806480u);
    }
}

// Weights 2^(score - reference) go into the second product in the cache's type: the tensor cores take 16 bits there, and half the
// bytes of a 32-bit form; a weight is off by half a unit in its last place, like the values that it multiplies. A row's reference is
// its largest score less `lift` when it is set, and is set anew when a score exceeds it by `grow`. bf16 has the exponents of fp32, and
// any reference will do. f16 keeps all its bits only down to 2^-14: with weights of at most 1, 131071 keys of 2^-20.25 each lost 3 % of
// their share beside one strong key. Lifted to 2^7 and let grow to 2^15 (65504 is the largest number), weights down to 2^-21 of the
// largest keep all their bits, and what smaller ones lose is at most 2^-32 of it each. 2048 tokens over 32768 keys: 961 us with lift 7,
// 959 with 0, 1188 with 10 (tiles done over, because a score less far above the reference already leaves the range).
template <class T>
struct WeightRange {
    static constexpr float lift = 0.0f, grow = 8.0f;
    static constexpr float most = 14.0f;                 // weights may reach 2^most before a reference is looked at
};
template <>
struct WeightRange<__half> {
    static constexpr float lift = 7.0f, grow = 15.0f, most = 15.0f;
};

// rint(4096 clamp(x, -2047, 2047)), NaN -> 0: the conversion saturates and takes NaN to 0, the limit is a whole number of steps.
__device__ __forceinline__ int fixed_of(float x)
{
    constexpr int limit = static_cast<int>(kSumLimit * kSumSteps);
    return min(max(__float2int_rn(__fmul_rn(x, kSumSteps)), -limit), limit);
}

// rint(127 total / most) as two fp32 roundings (the product's and the quotient's) define it. The reciprocal is off by a few units
// in the last place, which shows only next to a half: there the quotient is taken.
__device__ __forceinline__ int code_of(int total, float most, float inv)
{
    const float x = __fmul_rn(__int2float_rn(total), 127.0f), r = x * inv, n = rintf(r);
    if (fabsf(fabsf(r - n) - 0.5f) > 1e-3f) return static_cast<int>(n);
    return static_cast<int>(rintf(__fdiv_rn(x, most)));
}

}  // namespace kv
}  // namespace s3
