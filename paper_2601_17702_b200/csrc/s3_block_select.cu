// Block selection: per new token and key head, the s blocks with the highest 8-bit score, the first and last ones included.
//
// A thread block takes up to TT tokens of one sequence and one key head. (1) The group's queries are summed in fixed point and
// coded to 8 bits, one warp per token. (2) The codes of 16 tokens are one operand of an 8-bit mma.sync (exact 32-bit sums) whose
// other operand, the codes of 8 blocks, goes from memory straight to registers: the two uint4 that a lane reads of its block's
// code and of its tokens' codes hold the same dimensions, and in which order a dot product takes them does not matter. (An 8-bit
// mma does 512 products per clock and scheduler, dp4a 64: 91 us per 2048 tokens x 8 heads x 512 blocks with dp4a.) The
// scores go to shared memory as order-preserving words (forced blocks highest, invisible ones 0). (3) A warp per token
// selects: each lane keeps two maxima, and the s-th largest of the 64 bounds the s-th largest score from below, so one pass
// collects the few candidates above it in block order, and each then counts how many are better. 33 to 64 candidates, or (large
// s, many equal scores) all scores, are bisected over their bits instead; ties always go to the lowest blocks.
// Bound by instructions (64 % of the issue slots): that 2048-token case now takes 35 us whole; 24 single tokens over up to 512
// blocks 9 us, which is latency.
#include "s3_kernels.cuh"
#include "s3_kv.cuh"

namespace s3 {
namespace {

using kv::Half2Of;

constexpr int SCORE_BYTES = 96 << 10;       // shared memory for scores: two thread blocks per SM
constexpr int MMA_TOKENS = 16;
constexpr int CAND = 64;                    // candidates per warp

struct SelectArgs {
    KvBatchDev b;
    const void* q;
    int64_t ldq;
    int n_heads, n_kv_heads, group, page_shift, n_pages;
    const int8_t* code;
    const float* scale;
    int s, n_first, n_last, nb_cap, one_item_per_seq;
    int32_t* blocks;
    uint32_t* status;
};

// Order-preserving word of fl32(dot) * scale. |dot| < 2^22: adding it to the bits of 1.5 * 2^23 converts it exactly, without the
// conversion unit; the multiply-add with +0 turns a -0 (scale 0) into the +0 that it equals.
__device__ __forceinline__ uint32_t order_of(int dot, float scale)
{
    const float x = __fmaf_rn(__fsub_rn(__int_as_float(0x4B400000 + dot), 12582912.0f), scale, 0.0f);
    const int b = __float_as_int(x);
    return static_cast<uint32_t>(b ^ ((b >> 31) | static_cast<int>(0x80000000u)));
}

// Largest v such that at least s of the n keys are >= v (n >= s).
template <class Get>
__device__ __forceinline__ uint32_t cut_of(int n, int s, Get get)
{
    const int lane = threadIdx.x & 31;
    uint32_t v = 0;
    for (int bit = 31; bit >= 0; --bit) {
        const uint32_t t = v | (1u << bit);
        int c = 0;
        for (int i = lane; i < n; i += 32) c += get(i) >= t;
        if (__reduce_add_sync(0xffffffffu, c) >= s) v = t;
    }
    return v;
}

// Writes the numbers of the s best of n entries in entry order: all above the cut, then the first ones at it.
template <class Get, class Num>
__device__ __forceinline__ void emit(int n, int s, uint32_t cut, Get get, Num num, int32_t* out)
{
    const int lane = threadIdx.x & 31;
    int above = 0;
    for (int i = lane; i < n; i += 32) above += get(i) > cut;
    int ties = s - __reduce_add_sync(0xffffffffu, above), done = 0;
    for (int i0 = 0; i0 < n; i0 += 32) {
        const uint32_t key = i0 + lane < n ? get(i0 + lane) : 0u;
        const uint32_t tie = __ballot_sync(0xffffffffu, i0 + lane < n && key == cut);
        const bool mine = i0 + lane < n && (key > cut || (key == cut && __popc(tie & ((1u << lane) - 1)) < ties));
        const uint32_t take = __ballot_sync(0xffffffffu, mine);
        if (mine) out[done + __popc(take & ((1u << lane) - 1))] = num(i0 + lane);
        done += __popc(take);
        ties = max(ties - __popc(tie), 0);
    }
}

__device__ __forceinline__ void select_row(const uint32_t* keys, int nb, int s, uint16_t* cand, int32_t* out)
{
    const int lane = threadIdx.x & 31;
    if (nb <= s) {
        for (int i = lane; i < s; i += 32) out[i] = i < nb ? i : -1;
        return;
    }
    {
        // four neighbouring blocks per lane and step; what a row holds past its blocks is ignored
        const uint4* keys4 = reinterpret_cast<const uint4*>(keys);
        auto four = [&](int i0) {
            uint4 k = keys4[(i0 >> 2) + lane];
            if (i0 + 128 > nb) {
                const int left = nb - i0 - 4 * lane;
                if (left < 1) k.x = 0;
                if (left < 2) k.y = 0;
                if (left < 3) k.z = 0;
                if (left < 4) k.w = 0;
            }
            return k;
        };
        uint32_t best_a = 0, best_b = 0;                               // of this lane's even and odd pairs of blocks
        for (int i0 = 0; i0 < nb; i0 += 128) {
            const uint4 k = four(i0);
            best_a = max(best_a, max(k.x, k.y));
            best_b = max(best_b, max(k.z, k.w));
        }
        // the s-th largest of the 64 maxima, rounded down to its upper 17 bits
        uint32_t bound = 0;
#pragma unroll
        for (int bit = 31; bit >= 15; --bit) {
            const uint32_t t = bound | (1u << bit);
            if (__popc(__ballot_sync(0xffffffffu, best_a >= t)) + __popc(__ballot_sync(0xffffffffu, best_b >= t)) >= s) bound = t;
        }
        bound = max(bound, 1u);
        // candidate number c of the row, in block order, ends up in lane c
        const uint32_t lower = (1u << lane) - 1;
        int n = 0;
        for (int i0 = 0; i0 < nb; i0 += 128) {
            const uint4 k = four(i0);
            const bool in[4] = {k.x >= bound, k.y >= bound, k.z >= bound, k.w >= bound};
            int at = n;
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                const uint32_t all = __ballot_sync(0xffffffffu, in[x]);
                at += __popc(all & lower);
                n += __popc(all);
            }
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                if (in[x] && at < CAND) cand[at] = static_cast<uint16_t>(i0 + 4 * lane + x);
                at += in[x];
            }
        }
        __syncwarp();
        const int num = lane < min(n, 32) ? cand[lane] : -1;
        const uint32_t key = num >= 0 ? keys[num] : 0u;
        __syncwarp();
        if (n >= s && n <= 32) {
            int better = 0;
#pragma unroll
            for (int c = 0; c < 32; ++c) {
                const uint32_t k = __shfl_sync(0xffffffffu, key, c);       // 0 past the last candidate
                better += k > key || (k == key && c < lane);
            }
            const bool take = lane < n && better < s;
            const uint32_t taken = __ballot_sync(0xffffffffu, take);
            if (take) out[__popc(taken & ((1u << lane) - 1))] = num;
            return;
        }
        if (n > 32 && n <= CAND) {
            auto get = [&](int i) { return keys[cand[i]]; };
            emit(n, s, cut_of(n, s, get), get, [&](int i) { return static_cast<int32_t>(cand[i]); }, out);
            __syncwarp();
            return;
        }
    }
    auto get = [&](int i) { return keys[i]; };
    emit(nb, s, cut_of(nb, s, get), get, [&](int i) { return i; }, out);
}

template <class T, int D, int TT, int THREADS>
__global__ void __launch_bounds__(THREADS, TT == 16 ? 5 : 2) select_kernel(const SelectArgs a)
{
    constexpr int W = D / 4, WARPS = THREADS / 32;            // 32-bit words of a code
    extern __shared__ __align__(16) unsigned char smem[];
    uint32_t* codes = reinterpret_cast<uint32_t*>(smem);      // [16][W], rows past the tokens zero
    uint32_t* keys = reinterpret_cast<uint32_t*>(smem + MMA_TOKENS * D);   // [TT][nb_cap]
    __shared__ uint16_t cand[WARPS][CAND];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int head = blockIdx.x % a.n_kv_heads, item = blockIdx.x / a.n_kv_heads;
    int seq = item, idx = 0;
    cudaTriggerProgrammaticLaunchCompletion();
    cudaGridDependencySynchronize();
    if (!a.one_item_per_seq) {
        const KvBatchDev& b = a.b;
        if (!locate_item(b.n_seqs, item, [&](int i) { return (load_seq(b, i, nullptr).n + TT - 1) / TT; }, seq, idx)) return;
    }
    const SeqSpan s = load_seq(a.b, seq, a.status);
    const int n_tok = min(TT, s.n - idx * TT);
    if (n_tok <= 0) return;
    const int tok0 = s.q0 + idx * TT, pos0 = s.kv - s.n + idx * TT;

    for (int tt = warp; tt < MMA_TOKENS; tt += WARPS) {
        if (tt >= n_tok) {
            if (lane < W) codes[tt * W + lane] = 0u;
            continue;
        }
        using H = Half2Of<T>;
        int q[4] = {0, 0, 0, 0};
        if (lane < W) {
            const T* src = static_cast<const T*>(a.q) + (tok0 + tt) * a.ldq + static_cast<int64_t>(head) * a.group * D + lane * 4;
            for (int g = 0; g < a.group; ++g) {
                const uint2 u = *reinterpret_cast<const uint2*>(src + g * D);
                q[0] += kv::fixed_of(H::lo(u.x)); q[1] += kv::fixed_of(H::hi(u.x));
                q[2] += kv::fixed_of(H::lo(u.y)); q[3] += kv::fixed_of(H::hi(u.y));
            }
        }
        const int most = __reduce_max_sync(0xffffffffu, max(max(abs(q[0]), abs(q[1])), max(abs(q[2]), abs(q[3]))));
        const float m = __int2float_rn(max(most, 1)), inv = 1.0f / m;
        uint32_t w = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int c = kv::code_of(q[i], m, inv);
            w |= (static_cast<uint32_t>(c) & 0xffu) << (8 * i);
        }
        if (lane < W) codes[tt * W + lane] = w;
    }
    __syncthreads();

    const int last = pos0 + n_tok - 1;
    const int nb = last < 0 ? 0 : (last >> a.page_shift) + 1;        // blocks that some token of the tile sees
    const int row = lane >> 2, quad = lane & 3;
    constexpr int Q = D / 64;                                         // uint4 per lane and row
    uint4 ta[Q], tb[Q];                                               // tokens row and row + 8
#pragma unroll
    for (int x = 0; x < Q; ++x) {
        ta[x] = *reinterpret_cast<const uint4*>(codes + row * W + (x * 4 + quad) * 4);
        tb[x] = TT > 8 ? *reinterpret_cast<const uint4*>(codes + (row + 8) * W + (x * 4 + quad) * 4) : make_uint4(0, 0, 0, 0);
    }
    const int32_t* table = a.b.pages + seq * a.b.ld_pages;
    const int8_t* my_code = a.code + head * D + quad * 16;            // of page 0
    const float* my_scale = a.scale + head;
    const int page_pitch = a.n_kv_heads * D;
    auto fetch = [&](int g, uint4 (&c)[Q], float& scale) {            // block 8 g + row
        const int j = g * 8 + row;
        scale = 0.0f;
#pragma unroll
        for (int x = 0; x < Q; ++x) c[x] = make_uint4(0, 0, 0, 0);
        if (j >= nb) return;
        const int page = table[j];
        if (static_cast<uint32_t>(page) >= static_cast<uint32_t>(a.n_pages)) {
            dev_set_error(a.status, DEV_BAD_PAGE);
            return;
        }
        const int8_t* src = my_code + static_cast<int64_t>(page) * page_pitch;
#pragma unroll
        for (int x = 0; x < Q; ++x) c[x] = *reinterpret_cast<const uint4*>(src + x * 64);
        scale = my_scale[static_cast<int64_t>(page) * a.n_kv_heads];
    };
    auto mma = [](int (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
        asm volatile("mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+r"(c[0]), "+r"(c[1]), "+r"(c[2]), "+r"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    };
    const int own_first = pos0 >> a.page_shift;                        // the tile's lowest own block
    uint4 next[Q];
    float next_scale;
    fetch(warp, next, next_scale);
    for (int g = warp; g * 8 < nb; g += WARPS) {
        uint4 c[Q];
#pragma unroll
        for (int x = 0; x < Q; ++x) c[x] = next[x];
        const float scale = next_scale;
        fetch(g + WARPS, next, next_scale);                            // the next group is on its way meanwhile
        int dot[4] = {0, 0, 0, 0};
#pragma unroll
        for (int x = 0; x < Q; ++x) {
            mma(dot, ta[x].x, tb[x].x, ta[x].y, tb[x].y, c[x].x, c[x].y);
            mma(dot, ta[x].z, tb[x].z, ta[x].w, tb[x].w, c[x].z, c[x].w);
        }
        const float s0 = __shfl_sync(0xffffffffu, scale, quad * 8), s1 = __shfl_sync(0xffffffffu, scale, quad * 8 + 4);
        uint32_t* to = keys + row * a.nb_cap + g * 8 + quad * 2;
        uint32_t key[4];
#pragma unroll
        for (int x = 0; x < 4; ++x) key[x] = order_of(dot[x], x & 1 ? s1 : s0);
        if (g * 8 < a.n_first || g * 8 + 7 > own_first - a.n_last || own_first < 0) {
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                const int own = (pos0 + row + (x >> 1) * 8) >> a.page_shift, j = g * 8 + quad * 2 + (x & 1);
                if (j < a.n_first || j > own - a.n_last) key[x] = 0xffffffffu;
                if (j > own) key[x] = 0u;                              // own < 0 at a negative position: nothing is visible
            }
        }
        if (row < TT) *reinterpret_cast<uint2*>(to) = make_uint2(key[0], key[1]);
        if (TT > 8) *reinterpret_cast<uint2*>(to + 8 * a.nb_cap) = make_uint2(key[2], key[3]);
    }
    __syncthreads();
    for (int tt = warp; tt < n_tok; tt += WARPS) {
        const int pos = pos0 + tt;
        select_row(keys + tt * a.nb_cap, pos < 0 ? 0 : (pos >> a.page_shift) + 1, a.s, cand[warp],
                   a.blocks + (static_cast<int64_t>(tok0 + tt) * a.n_kv_heads + head) * a.s);
    }
}

template <class T, int D, int TT, int THREADS>
s3_status launch_one(SelectArgs& a, cudaStream_t stream)
{
    const size_t smem = static_cast<size_t>(MMA_TOKENS) * D + static_cast<size_t>(TT) * a.nb_cap * 4;
    const s3_status allowed = allow_smem<select_kernel<T, D, TT, THREADS>>(200 << 10);
    if (allowed != S3_OK) return allowed;
    a.one_item_per_seq = a.b.max_q <= TT;
    const int64_t items = a.one_item_per_seq ? a.b.n_seqs : static_cast<int64_t>(a.b.T) / TT + a.b.n_seqs;
    S3_REQUIRE(items * a.n_kv_heads < (int64_t(1) << 31), S3_ERR_UNSUPPORTED, "the batch needs too many thread blocks");
    return launch_overlapped(select_kernel<T, D, TT, THREADS>, dim3(static_cast<unsigned>(items * a.n_kv_heads)), THREADS, smem, stream, a);
}

template <class T, int D>
s3_status launch_typed(SelectArgs& a, cudaStream_t stream)
{
    // Tokens per thread block: 16 share each code read, 4 or 1 where there are fewer of them, or where their scores do not fit. With 1, 4
    // and 16 (us, 32 heads over 8): 24 single tokens over 32K positions 8.3, 9.5, 10.7; 24 x 4 20.7, 10.0, 11.4; 8 x 8 over 8K 9.1, 5.6, 5.7;
    // 2048 over 32K 302, 65, 35. (64 single tokens over 8K 9.4, 6.4, 8.4: blocks of 1 take 512 threads.)
    const int room = SCORE_BYTES / (a.nb_cap * 4), want = a.b.max_q;
    if (room >= 16 && want > 4) return launch_one<T, D, 16, 256>(a, stream);
    if (room >= 4 && want > 1) return launch_one<T, D, 4, 256>(a, stream);
    return launch_one<T, D, 1, 512>(a, stream);
}

}  // namespace

s3_status launch_block_select(const KvCacheState& c, const KvBatchDev& b, const void* d_q, int64_t ldq, int n_heads, int s,
                              int n_first, int n_last, int32_t* d_blocks, uint32_t* d_status, cudaStream_t stream)
{
    SelectArgs a;
    a.b = b;
    a.q = d_q;
    a.ldq = ldq;
    a.n_heads = n_heads;
    a.n_kv_heads = c.d.n_kv_heads;
    a.group = n_heads / c.d.n_kv_heads;
    a.page_shift = c.page_shift;
    a.n_pages = c.d.n_pages;
    a.code = c.d.d_code;
    a.scale = c.d.d_scale;
    a.s = s;
    a.n_first = n_first;
    a.n_last = n_last;
    // words per row: whole steps of 128 blocks, and 8 more than a multiple of 32, so that 4 rows of a store fall into different banks
    a.nb_cap = (((b.max_kv + c.d.page_size - 1) >> c.page_shift) + 127) / 128 * 128 + 8;
    a.blocks = d_blocks;
    a.status = d_status;
    const bool wide = c.d.head_dim == 128;
    if (c.d.dtype == S3_BF16) return wide ? launch_typed<__nv_bfloat16, 128>(a, stream) : launch_typed<__nv_bfloat16, 64>(a, stream);
    return wide ? launch_typed<__half, 128>(a, stream) : launch_typed<__half, 64>(a, stream);
}

}  // namespace s3
