// Block selection: per new token and key head, the s blocks with the highest 8-bit score, the first and last ones included.
//
// A thread block takes TT tokens of one sequence and one key head. (1) The group's queries are summed in fixed point and coded
// to 8 bits, one warp per token. (2) Threads walk the sequence's blocks: a block's 8-bit summary is read once into registers
// and multiplied (dp4a, exact) with the codes of all TT tokens; the scores go to shared memory as order-preserving words
// (forced blocks highest, invisible ones 0). (3) A warp per token selects: the s-th largest of the 32 lanes' maxima bounds the
// s-th largest score from below, so one pass collects the few candidates above it in block order, and a bisection over their
// bits finds the exact cut; ties at the cut go to the lowest blocks. More than 32 blocks, or more candidates than the buffer
// holds, bisect over all scores instead.
#include "s3_kernels.cuh"
#include "s3_kv.cuh"

namespace s3 {
namespace {

using kv::Half2Of;

constexpr int CAND = 256;                   // candidates per warp
constexpr int SCORE_BYTES = 96 << 10;       // shared memory for scores: two thread blocks per SM

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

__device__ __forceinline__ uint32_t order_of(float x)
{
    const uint32_t b = __float_as_uint(x + 0.0f);        // -0 counts as 0
    return b & 0x80000000u ? ~b : b | 0x80000000u;
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
    if (s <= 32) {
        uint32_t best = 0;
        for (int i = lane; i < nb; i += 32) best = max(best, keys[i]);
        // the lanes' maxima in descending order over the lanes
#pragma unroll
        for (int size = 2; size <= 32; size <<= 1)
#pragma unroll
            for (int o = size >> 1; o > 0; o >>= 1) {
                const uint32_t other = __shfl_xor_sync(0xffffffffu, best, o);
                const bool keep_max = ((lane & o) == 0) == ((lane & size) == 0);
                best = keep_max ? max(best, other) : min(best, other);
            }
        const uint32_t bound = __shfl_sync(0xffffffffu, best, s - 1);
        int n = 0;
        for (int i0 = 0; i0 < nb && n <= CAND; i0 += 32) {
            const bool in = i0 + lane < nb && keys[i0 + lane] >= bound;
            const uint32_t m = __ballot_sync(0xffffffffu, in);
            const int at = n + __popc(m & ((1u << lane) - 1));
            if (in && at < CAND) cand[at] = static_cast<uint16_t>(i0 + lane);
            n += __popc(m);
        }
        __syncwarp();
        if (n <= CAND && bound > 0) {
            auto get = [&](int i) { return keys[cand[i]]; };
            const uint32_t cut = n == s ? bound : cut_of(n, s, get);
            emit(n, s, cut, get, [&](int i) { return static_cast<int32_t>(cand[i]); }, out);
            __syncwarp();
            return;
        }
    }
    auto get = [&](int i) { return keys[i]; };
    emit(nb, s, cut_of(nb, s, get), get, [&](int i) { return i; }, out);
}

template <class T, int D, int TT, int THREADS>
__global__ void __launch_bounds__(THREADS) select_kernel(const SelectArgs a)
{
    constexpr int W = D / 4;                                  // 32-bit words of a code
    extern __shared__ __align__(16) unsigned char smem[];
    uint32_t* codes = reinterpret_cast<uint32_t*>(smem);      // [TT][W]
    uint16_t* cand = reinterpret_cast<uint16_t*>(smem + TT * D);      // [warps][CAND]
    uint32_t* keys = reinterpret_cast<uint32_t*>(smem + TT * D + (THREADS / 32) * CAND * 2);   // [TT][nb_cap]
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int head = blockIdx.x % a.n_kv_heads, item = blockIdx.x / a.n_kv_heads;
    int seq = item, idx = 0;
    if (!a.one_item_per_seq) {
        const KvBatchDev& b = a.b;
        if (!locate_item(b.n_seqs, item, [&](int i) { return (load_seq(b, i, nullptr).n + TT - 1) / TT; }, seq, idx)) return;
    }
    const SeqSpan s = load_seq(a.b, seq, a.status);
    const int n_tok = min(TT, s.n - idx * TT);
    if (n_tok <= 0) return;
    const int tok0 = s.q0 + idx * TT, pos0 = s.kv - s.n + idx * TT;

    for (int tt = warp; tt < n_tok; tt += THREADS / 32) {
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
        const float m = __int2float_rn(max(most, 1));
        uint32_t w = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int c = static_cast<int>(rintf(__fdiv_rn(__fmul_rn(__int2float_rn(q[i]), 127.0f), m)));
            w |= (static_cast<uint32_t>(c) & 0xffu) << (8 * i);
        }
        if (lane < W) codes[tt * W + lane] = w;
    }
    __syncthreads();

    const int last = pos0 + n_tok - 1;
    const int nb = last < 0 ? 0 : (last >> a.page_shift) + 1;        // blocks that some token of the tile sees
    for (int j = threadIdx.x; j < nb; j += THREADS) {
        const int page = a.b.pages[seq * a.b.ld_pages + j];
        uint4 c[W / 4];
        float scale = 0.0f;
        if (page >= 0 && page < a.n_pages) {
            const int64_t at = static_cast<int64_t>(page) * a.n_kv_heads + head;
            const uint4* src = reinterpret_cast<const uint4*>(a.code + at * D);
#pragma unroll
            for (int i = 0; i < W / 4; ++i) c[i] = __ldg(src + i);
            scale = __ldg(a.scale + at);
        } else {
            dev_set_error(a.status, DEV_BAD_PAGE);
#pragma unroll
            for (int i = 0; i < W / 4; ++i) c[i] = make_uint4(0, 0, 0, 0);
        }
#pragma unroll 4
        for (int tt = 0; tt < TT; ++tt) {
            if (tt >= n_tok) break;
            const uint4* q4 = reinterpret_cast<const uint4*>(codes + tt * W);
            int d0 = 0, d1 = 0;
#pragma unroll
            for (int i = 0; i < W / 4; ++i) {
                const uint4 q = q4[i];
                d0 = __dp4a(static_cast<int>(c[i].x), static_cast<int>(q.x), d0);
                d1 = __dp4a(static_cast<int>(c[i].y), static_cast<int>(q.y), d1);
                d0 = __dp4a(static_cast<int>(c[i].z), static_cast<int>(q.z), d0);
                d1 = __dp4a(static_cast<int>(c[i].w), static_cast<int>(q.w), d1);
            }
            const int own = (pos0 + tt) >> a.page_shift;              // < 0 at a negative position: nothing is visible
            uint32_t key = order_of(__fmul_rn(__int2float_rn(d0 + d1), scale));
            if (j < a.n_first || j > own - a.n_last) key = 0xffffffffu;
            if (j > own) key = 0u;
            keys[tt * a.nb_cap + j] = key;
        }
    }
    __syncthreads();
    for (int tt = warp; tt < n_tok; tt += THREADS / 32) {
        const int pos = pos0 + tt;
        select_row(keys + tt * a.nb_cap, pos < 0 ? 0 : (pos >> a.page_shift) + 1, a.s, cand + warp * CAND,
                   a.blocks + (static_cast<int64_t>(tok0 + tt) * a.n_kv_heads + head) * a.s);
    }
}

template <class T, int D, int TT, int THREADS>
s3_status launch_one(SelectArgs& a, cudaStream_t stream)
{
    const size_t smem = static_cast<size_t>(TT) * D + (THREADS / 32) * CAND * 2 + static_cast<size_t>(TT) * a.nb_cap * 4;
    static bool raised[64] = {};                 // the attribute is kept per device; setting it twice does no harm
    int dev = 0;
    S3_CUDA_TRY(cudaGetDevice(&dev));
    if (dev >= 64 || !raised[dev]) {
        S3_CUDA_TRY(cudaFuncSetAttribute(select_kernel<T, D, TT, THREADS>, cudaFuncAttributeMaxDynamicSharedMemorySize, 200 << 10));
        if (dev < 64) raised[dev] = true;
    }
    a.one_item_per_seq = a.b.max_q <= TT;
    const int64_t items = a.one_item_per_seq ? a.b.n_seqs : static_cast<int64_t>(a.b.T) / TT + a.b.n_seqs;
    S3_REQUIRE(items * a.n_kv_heads < (int64_t(1) << 31), S3_ERR_UNSUPPORTED, "the batch needs too many thread blocks");
    select_kernel<T, D, TT, THREADS><<<static_cast<unsigned>(items * a.n_kv_heads), THREADS, smem, stream>>>(a);
    S3_CUDA_TRY(cudaGetLastError());
    return S3_OK;
}

template <class T, int D>
s3_status launch_typed(SelectArgs& a, cudaStream_t stream)
{
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
    a.nb_cap = ((b.max_kv + c.d.page_size - 1) >> c.page_shift) | 1;     // odd row pitch: rows start in different banks
    a.blocks = d_blocks;
    a.status = d_status;
    const bool wide = c.d.head_dim == 128;
    if (c.d.dtype == S3_BF16) return wide ? launch_typed<__nv_bfloat16, 128>(a, stream) : launch_typed<__nv_bfloat16, 64>(a, stream);
    return wide ? launch_typed<__half, 128>(a, stream) : launch_typed<__half, 64>(a, stream);
}

}  // namespace s3
