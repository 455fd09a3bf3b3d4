// Attention of a few query rows (at most 16 per item and key head) over a paged cache: decoding steps and lists per token.
//
//   out = sum_j p_j v_j / sum_j p_j,  p_j = 2^(scale log2e q.k_j - m)      one pass, running maximum m and sum
//
// Bound by reading keys and values once (HBM, or the L2 cache when neighbouring tokens list the same blocks). A thread block
// takes one (item, key head, split of the keys). Warp 4 copies 64-key tiles of K and V with TMA, page by page, into a ring of
// STAGES shared-memory slots; warps 0-3 take 16 keys of every tile each and keep their own m, sum and 16 x head_dim
// accumulator in registers, so the warps meet only at the end. Both products run on mma.sync m16n8k16 with the rows padded
// to 16: with this few rows per key the work is a copy, and the padding costs nothing that the memory would not.
// The four partial results, and then the splits (second kernel), are joined by their maxima and sums.
#include <type_traits>

#include "s3_kernels.cuh"
#include "s3_kv.cuh"

namespace s3 {
namespace {

using namespace kv;

constexpr int TILE = 64;                  // keys per tile
constexpr int STAGES = 3;
constexpr int WARPS = 4;                  // compute warps
constexpr int THREADS = 32 * (WARPS + 1);

struct Maps {
    alignas(64) unsigned char k[128], v[128];
};

template <int D>
__host__ __device__ constexpr int stage_bytes() { return 2 * TILE * D * 2; }
template <int D>
constexpr size_t smem_bytes() { return 1024 + static_cast<size_t>(STAGES) * stage_bytes<D>() + S3_MAX_BLOCK_LIST * 4; }

__device__ __forceinline__ void ldsm4(uint32_t (&r)[4], uint32_t addr)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldsm4_t(uint32_t (&r)[4], uint32_t addr)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
template <class T>
__device__ __forceinline__ void mma16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    if constexpr (std::is_same<T, __half>::value)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

template <class T, int D>
__global__ void __launch_bounds__(THREADS, 2) split_kernel(const __grid_constant__ Maps maps, const AttnArgs a)
{
    extern __shared__ unsigned char smem_raw[];
    unsigned char* ring = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    int* list = reinterpret_cast<int*>(ring + STAGES * stage_bytes<D>());
    __shared__ uint64_t full_bar[STAGES], empty_bar[STAGES];
    __shared__ uint32_t abort_word;
    __shared__ float red_m[WARPS][16], red_l[WARPS][16];
    volatile uint32_t* abort_flag = &abort_word;

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int split = blockIdx.x % a.n_splits, head = (blockIdx.x / a.n_splits) % a.n_kv_heads;
    const int item = blockIdx.x / a.n_splits / a.n_kv_heads;
    AttnItem it;
    if (!attn_item(a, item, it)) return;
    const int rows = it.n_tok * a.group;
    const int pos_last = a.causal ? it.pos0 + it.n_tok - 1 : it.pos0;
    const int seen_lo = a.window > 0 ? max(it.pos0 - a.window + 1, 0) : 0;     // positions some row of the item may see
    int v_lo = 0, v_hi = 0;
    if (a.list_mode == LIST_NONE) {
        v_lo = (seen_lo & ~(TILE - 1)) + split * a.split_len;
        v_hi = min(v_lo + a.split_len, pos_last + 1);
    } else {
        v_lo = split * a.split_len;
        v_hi = min((split + 1) * a.split_len, a.s << a.page_shift);
        const int hl = a.list_heads == 1 ? 0 : head;
        const int32_t* src = a.lists + (static_cast<int64_t>(it.list) * a.list_heads + hl) * a.s;
        for (int e = threadIdx.x; e < a.s; e += THREADS) {
            const int id = src[e];
            // a block all of whose positions are out of sight counts as not listed
            list[e] = id >= 0 && id <= (pos_last >> a.page_shift) && pos_last >= 0 && ((id + 1) << a.page_shift) > seen_lo ? id : -1;
        }
    }
    const int n_tiles = max(0, (v_hi - v_lo + TILE - 1) / TILE);
    if (threadIdx.x == 0) {
        for (int i = 0; i < STAGES; ++i) { mbar_init(&full_bar[i], 1); mbar_init(&empty_bar[i], WARPS); }
        abort_word = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncthreads();

    // First position of virtual key v (a multiple of 16), or -1 where no block is listed.
    auto pos_of = [&](int v) -> int {
        if (a.list_mode == LIST_NONE) return v;
        const int e = v >> a.page_shift;
        if (e >= a.s || list[e] < 0) return -1;
        return (list[e] << a.page_shift) + (v & (a.page_size - 1));
    };

    float o[D / 8][4];
    float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < D / 8; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) o[i][j] = 0.0f;

    int issued = 0;                            // tiles whose copies were started
    if (warp == WARPS) {
        // ---------------- producer ----------------
        if (lane == 0) {
            const int box = a.box_rows, per_tile = TILE / box;
            const int32_t* table = a.b.pages + it.seq * a.b.ld_pages;
            for (int t = 0; t < n_tiles; ++t) {
                const int st = t % STAGES;
                if (t >= STAGES && !mbar_wait(&empty_bar[st], ((t / STAGES) - 1) & 1, abort_flag)) {
                    dev_set_error(a.status, DEV_TIMEOUT_SMEM_EMPTY);
                    *abort_flag = 1;
                    break;
                }
                unsigned char* dst = ring + st * stage_bytes<D>();
                uint32_t bytes = 0;
                int page[TILE / 16], row[TILE / 16];
#pragma unroll
                for (int u = 0; u < TILE / 16; ++u) {
                    page[u] = -1;
                    row[u] = 0;
                    if (u >= per_tile) continue;
                    const int v = v_lo + t * TILE + u * box, pos = v < v_hi ? pos_of(v) : -1;
                    if (pos < 0 || pos >= it.kv) continue;
                    const int p = table[pos >> a.page_shift];
                    if (p < 0 || p >= a.n_pages) dev_set_error(a.status, DEV_BAD_PAGE);
                    page[u] = p < 0 || p >= a.n_pages ? a.n_pages : p;     // beyond the map: reads as zeros
                    row[u] = pos & (a.page_size - 1);
                    bytes += 2u * static_cast<uint32_t>(box) * D * 2;
                }
                issued = t + 1;
                if (bytes == 0) { mbar_arrive(&full_bar[st]); continue; }
                mbar_expect_tx(&full_bar[st], bytes);
#pragma unroll
                for (int u = 0; u < TILE / 16; ++u) {
                    if (page[u] < 0) continue;
#pragma unroll
                    for (int h = 0; h < D / 64; ++h) {
                        tma_load_4d(dst + h * TILE * 128 + u * box * 128, maps.k, h * 64, row[u], head, page[u], &full_bar[st]);
                        tma_load_4d(dst + TILE * D * 2 + h * TILE * 128 + u * box * 128, maps.v, h * 64, row[u], head, page[u], &full_bar[st]);
                    }
                }
            }
        }
    } else {
        // ---------------- compute ----------------
        const int r0 = lane >> 2, c0 = (lane & 3) * 2;
        uint32_t q[D / 16][4];
        int qpos[2];
        {
            const T* base = static_cast<const T*>(a.q) + static_cast<int64_t>(head) * a.group * D;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int row = r0 + 8 * i;
                const bool live = row < rows;
                const int tok = live ? row / a.group : 0, g = live ? row % a.group : 0;
                const T* src = base + static_cast<int64_t>(it.tok0 + tok) * a.ldq + g * D;
                qpos[i] = live ? (a.causal ? it.pos0 + tok : it.pos0) : -1;
#pragma unroll
                for (int k = 0; k < D / 16; ++k) {
                    q[k][i] = live ? *reinterpret_cast<const uint32_t*>(src + k * 16 + c0) : 0u;
                    q[k][2 + i] = live ? *reinterpret_cast<const uint32_t*>(src + k * 16 + 8 + c0) : 0u;
                }
            }
        }
        const int mi = lane >> 3, mr = lane & 7;
        const int k_row = warp * 16 + (mi >> 1) * 8 + mr, k_chunk = mi & 1;      // K: matrices (keys 0-7 | 8-15) x (d 0-7 | 8-15)
        const int v_row = warp * 16 + (mi & 1) * 8 + mr, v_chunk = mi >> 1;      // V: the same with the roles swapped, transposed
        bool ok = true;
        for (int t = 0; t < n_tiles; ++t) {
            const int st = t % STAGES;
            ok = mbar_wait(&full_bar[st], (t / STAGES) & 1, abort_flag);
            if (!__all_sync(0xffffffffu, ok)) {
                ok = false;
                if (lane == 0) { dev_set_error(a.status, DEV_TIMEOUT_TMA_FULL); *abort_flag = 1; }
                break;
            }
            const int v = v_lo + t * TILE + warp * 16;
            const int pos = v < v_hi ? pos_of(v) : -1;
            if (pos >= 0 && pos <= pos_last) {
                unsigned char* tile = ring + st * stage_bytes<D>();
                const uint32_t ks = smem_u32(tile), vs = ks + TILE * D * 2;
                if (pos + 16 > it.kv) {
                    // values past the last position may hold anything: zero their rows
                    const int first = max(it.kv - pos, 0);
                    for (int x = lane; x < (16 - first) * (D / 64) * 8; x += 32) {
                        const int rr = first + x / ((D / 64) * 8), c = x % ((D / 64) * 8);
                        *reinterpret_cast<uint4*>(tile + TILE * D * 2 + (c >> 3) * TILE * 128 + (warp * 16 + rr) * 128 + (c & 7) * 16) =
                            make_uint4(0, 0, 0, 0);
                    }
                    fence_async_smem();
                    __syncwarp();
                }
                float sc[2][4] = {{0, 0, 0, 0}, {0, 0, 0, 0}};
#pragma unroll
                for (int k = 0; k < D / 16; ++k) {
                    uint32_t b[4];
                    const int c = k * 2 + k_chunk;
                    ldsm4(b, ks + (c >> 3) * TILE * 128 + k_row * 128 + (((c & 7) ^ (k_row & 7)) << 4));
                    mma16816<T>(sc[0], q[k], b[0], b[1]);
                    mma16816<T>(sc[1], q[k], b[2], b[3]);
                }
                const bool edge = pos + 15 > it.pos0 || (a.window > 0 && pos <= pos_last - a.window);
                float mx[2] = {-INFINITY, -INFINITY};
#pragma unroll
                for (int n = 0; n < 2; ++n)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int i = j >> 1, kp = pos + n * 8 + c0 + (j & 1);
                        sc[n][j] *= a.scale_log2;
                        if (edge && (kp > qpos[i] || (a.window > 0 && kp <= qpos[i] - a.window))) sc[n][j] = -INFINITY;
                        mx[i] = fmaxf(mx[i], sc[n][j]);
                    }
                float f[2], ref[2];
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    mx[i] = fmaxf(mx[i], __shfl_xor_sync(0xffffffffu, mx[i], 1));
                    mx[i] = fmaxf(mx[i], __shfl_xor_sync(0xffffffffu, mx[i], 2));
                    mx[i] = fmaxf(mx[i], m[i]);
                    ref[i] = mx[i] == -INFINITY ? 0.0f : mx[i];
                    f[i] = ex2(m[i] - ref[i]);
                    m[i] = mx[i];
                    l[i] *= f[i];
                }
                uint32_t p[4];
#pragma unroll
                for (int n = 0; n < 2; ++n) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        sc[n][j] = ex2(sc[n][j] - ref[j >> 1]);
                        l[j >> 1] += sc[n][j];
                    }
                    p[2 * n] = Half2Of<T>::pack(sc[n][0], sc[n][1]);
                    p[2 * n + 1] = Half2Of<T>::pack(sc[n][2], sc[n][3]);
                }
                if (__any_sync(0xffffffffu, f[0] != 1.0f || f[1] != 1.0f)) {
#pragma unroll
                    for (int i = 0; i < D / 8; ++i) { o[i][0] *= f[0]; o[i][1] *= f[0]; o[i][2] *= f[1]; o[i][3] *= f[1]; }
                }
#pragma unroll
                for (int k = 0; k < D / 16; ++k) {
                    uint32_t b[4];
                    const int c = k * 2 + v_chunk;
                    ldsm4_t(b, vs + (c >> 3) * TILE * 128 + v_row * 128 + (((c & 7) ^ (v_row & 7)) << 4));
                    mma16816<T>(o[2 * k], p, b[0], b[1]);
                    mma16816<T>(o[2 * k + 1], p, b[2], b[3]);
                }
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(&empty_bar[st]);
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            l[i] += __shfl_xor_sync(0xffffffffu, l[i], 1);
            l[i] += __shfl_xor_sync(0xffffffffu, l[i], 2);
            if ((lane & 3) == 0) { red_m[warp][r0 + 8 * i] = m[i]; red_l[warp][r0 + 8 * i] = l[i]; }
        }
    }
    // every copy has landed and been read (or waited for): the ring becomes the meeting place of the four accumulators
    __syncthreads();
    if (*abort_flag) {
        if (threadIdx.x == WARPS * 32)         // no copy may be in flight when the block leaves
            for (int i = max(0, issued - STAGES); i < issued; ++i) mbar_wait(&full_bar[i % STAGES], (i / STAGES) & 1, nullptr);
        __syncthreads();
        return;
    }
    constexpr int PITCH = D + 4;
    float* acc = reinterpret_cast<float*>(ring);                       // [WARPS][16][PITCH]
    static_assert(WARPS * 16 * PITCH * 4 <= STAGES * stage_bytes<D>(), "the accumulators fit the ring");
    if (warp < WARPS) {
        const int r0 = lane >> 2, c0 = (lane & 3) * 2;
#pragma unroll
        for (int i = 0; i < D / 8; ++i) {
            *reinterpret_cast<float2*>(&acc[(warp * 16 + r0) * PITCH + i * 8 + c0]) = make_float2(o[i][0], o[i][1]);
            *reinterpret_cast<float2*>(&acc[(warp * 16 + r0 + 8) * PITCH + i * 8 + c0]) = make_float2(o[i][2], o[i][3]);
        }
    }
    __syncthreads();
    constexpr int VEC = D / 4;
    for (int x = threadIdx.x; x < rows * VEC; x += THREADS) {
        const int row = x / VEC, c = (x % VEC) * 4;
        float top = red_m[0][row];
#pragma unroll
        for (int w = 1; w < WARPS; ++w) top = fmaxf(top, red_m[w][row]);
        const float ref = top == -INFINITY ? 0.0f : top;
        float sum = 0.0f;
        float4 y = make_float4(0, 0, 0, 0);
#pragma unroll
        for (int w = 0; w < WARPS; ++w) {
            const float f = ex2(red_m[w][row] - ref);
            sum += f * red_l[w][row];
            const float4 z = *reinterpret_cast<const float4*>(&acc[(w * 16 + row) * PITCH + c]);
            y.x += f * z.x; y.y += f * z.y; y.z += f * z.z; y.w += f * z.w;
        }
        const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
        y.x *= inv; y.y *= inv; y.z *= inv; y.w *= inv;
        const int tok = it.tok0 + row / a.group, h = head * a.group + row % a.group;
        const int64_t out_row = static_cast<int64_t>(tok) * a.n_heads + h;
        const float lse2 = sum == 0.0f ? -INFINITY : top + log2f(sum);
        if (a.n_splits == 1) {
            T* dst = static_cast<T*>(a.out) + static_cast<int64_t>(tok) * a.ld_out + h * D + c;
            *reinterpret_cast<uint2*>(dst) = make_uint2(Half2Of<T>::pack(y.x, y.y), Half2Of<T>::pack(y.z, y.w));
            if (c == 0 && a.lse) a.lse[out_row] = lse2 / kLog2e;
        } else {
            const int64_t part = static_cast<int64_t>(split) * a.b.T * a.n_heads + out_row;
            if (sum != 0.0f) *reinterpret_cast<float4*>(a.part_o + part * D + c) = y;
            if (c == 0) a.part_lse[part] = lse2;
        }
    }
}

// Joins the splits of every row: weights 2^(lse_i - max). A warp per row.
template <class T, int D>
__global__ void __launch_bounds__(128) join_kernel(const AttnArgs a)
{
    cudaGridDependencySynchronize();
    const int lane = threadIdx.x & 31;
    const int64_t row = static_cast<int64_t>(blockIdx.x) * 4 + (threadIdx.x >> 5), rows = static_cast<int64_t>(a.b.T) * a.n_heads;
    if (row >= rows) return;
    float top = -INFINITY;
    for (int i = lane; i < a.n_splits; i += 32) top = fmaxf(top, a.part_lse[i * rows + row]);
#pragma unroll
    for (int x = 16; x > 0; x >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, x));
    constexpr int N = D / 32;                    // consecutive values per lane
    float y[N];
#pragma unroll
    for (int j = 0; j < N; ++j) y[j] = 0.0f;
    float sum = 0.0f;
    const bool some = top > -INFINITY;
    for (int i = 0; some && i < a.n_splits; ++i) {
        const float part = a.part_lse[i * rows + row];
        if (part == -INFINITY) continue;         // nothing was written there
        const float f = ex2(part - top);
        sum += f;
        const float* src = a.part_o + (i * rows + row) * D + lane * N;
        if constexpr (N == 4) {
            const float4 z = *reinterpret_cast<const float4*>(src);
            y[0] += f * z.x; y[1] += f * z.y; y[2] += f * z.z; y[3] += f * z.w;
        } else {
            const float2 z = *reinterpret_cast<const float2*>(src);
            y[0] += f * z.x; y[1] += f * z.y;
        }
    }
    const float inv = some ? 1.0f / sum : 0.0f;
    const int64_t tok = row / a.n_heads, h = row % a.n_heads;
    T* dst = static_cast<T*>(a.out) + tok * a.ld_out + h * D + lane * N;
#pragma unroll
    for (int j = 0; j < N; j += 2) *reinterpret_cast<uint32_t*>(dst + j) = Half2Of<T>::pack(y[j] * inv, y[j + 1] * inv);
    if (lane == 0 && a.lse) a.lse[row] = some ? (top + log2f(sum)) / kLog2e : -INFINITY;
}

template <class T, int D>
s3_status launch_split(const KvCacheState& c, const AttnArgs& a, cudaStream_t stream)
{
    static bool raised[64] = {};                 // the attribute is kept per device; setting it twice does no harm
    int dev = 0;
    S3_CUDA_TRY(cudaGetDevice(&dev));
    if (dev >= 64 || !raised[dev]) {
        S3_CUDA_TRY(cudaFuncSetAttribute(split_kernel<T, D>, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem_bytes<D>())));
        if (dev < 64) raised[dev] = true;
    }
    Maps maps;
    memcpy(maps.k, c.map_k, sizeof(maps.k));
    memcpy(maps.v, c.map_v, sizeof(maps.v));
    const int64_t blocks = static_cast<int64_t>(a.n_items) * a.n_kv_heads * a.n_splits;
    S3_REQUIRE(blocks < (int64_t(1) << 31), S3_ERR_UNSUPPORTED, "the batch needs too many thread blocks");
    split_kernel<T, D><<<static_cast<unsigned>(blocks), THREADS, smem_bytes<D>(), stream>>>(maps, a);
    S3_CUDA_TRY(cudaGetLastError());
    return S3_OK;
}

template <class T, int D>
s3_status launch_join_typed(const AttnArgs& a, cudaStream_t stream)
{
    const int64_t rows = static_cast<int64_t>(a.b.T) * a.n_heads;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>((rows + 3) / 4));
    cfg.blockDim = dim3(128);
    cfg.stream = stream;
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;      // its launch overlaps the kernel before it
    attr.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    S3_CUDA_TRY(cudaLaunchKernelEx(&cfg, join_kernel<T, D>, a));
    return S3_OK;
}

}  // namespace

s3_status launch_attn_split(const KvCacheState& c, const AttnArgs& a, cudaStream_t stream)
{
    const bool wide = c.d.head_dim == 128;
    if (c.d.dtype == S3_BF16) return wide ? launch_split<__nv_bfloat16, 128>(c, a, stream) : launch_split<__nv_bfloat16, 64>(c, a, stream);
    return wide ? launch_split<__half, 128>(c, a, stream) : launch_split<__half, 64>(c, a, stream);
}

s3_status launch_attn_join(const KvCacheState& c, const AttnArgs& a, cudaStream_t stream)
{
    const bool wide = c.d.head_dim == 128;
    if (c.d.dtype == S3_BF16) return wide ? launch_join_typed<__nv_bfloat16, 128>(a, stream) : launch_join_typed<__nv_bfloat16, 64>(a, stream);
    return wide ? launch_join_typed<__half, 128>(a, stream) : launch_join_typed<__half, 64>(a, stream);
}

}  // namespace s3
