// Append to a paged key / value cache: rotation of keys and queries, copies into the pages, summaries of the touched blocks.
//
// One launch, two kinds of thread blocks. The first n_touched * n_kv_heads blocks take one (page that holds a new token, key
// head): they rotate and write the page's new keys, copy its new values and, when the cache has summaries, add the fixed-point
// keys of ALL the page's positions < kv_len (new ones from registers, earlier ones read back) in 32-bit integers. A summary is
// therefore a function of what the page holds: appending the same positions again, or again after a rollback, needs no
// record of earlier sums and no atomics. The remaining blocks rotate 32 query rows each.
// Bound by memory traffic with little work in flight per thread: the kernel is kept to 64 registers, eight thread blocks per SM
// (8192 tokens of 32 + 8 + 8 heads: 40 us when that was chosen, against 49 at 96 registers with four rows' reads issued at once).
// A thread owns 8 rotation pairs (two 16-byte vectors) of a row, so both halves of a pair are in its registers.
//
// Products and sums of the rotation are rounded one by one (no fused multiply-add): the rotated key, and with it every
// summary, has the same bits wherever the formula is evaluated in fp32.
#include "s3_kernels.cuh"
#include "s3_kv.cuh"

namespace s3 {
namespace {

using kv::Half2Of;

constexpr int THREADS = 128;
constexpr int Q_ROWS = 32;                 // query rows per thread block

struct AppendArgs {
    KvBatchDev b;
    const float* cosv;
    const float* sinv;
    int n_pos, rot_dim, interleaved;
    const int32_t* positions;
    const void *q, *k, *v;
    void* q_out;
    int64_t ldq, ld_qo, ldk, ldv;
    int n_heads, n_kv_heads, page_size, page_shift, n_pages;
    void *kc, *vc;
    int64_t k_page, v_page;
    int8_t* code;
    float* scale;
    int one_page_per_seq, n_kv_blocks;
    uint32_t* status;
};

// The two vectors of pair p: element offsets and whether they rotate.
__device__ __forceinline__ void pair_of(const AppendArgs& a, int p, int& e0, int& e1, bool& turn)
{
    turn = p * 16 < a.rot_dim;
    if (turn && !a.interleaved) {
        e0 = p * 8;
        e1 = a.rot_dim / 2 + p * 8;
    } else {
        e0 = p * 16;
        e1 = e0 + 8;
    }
}

template <class T>
__device__ __forceinline__ void rotate(const AppendArgs& a, int p, bool turn, int64_t angle_row, uint4& u0, uint4& u1)
{
    if (!turn) return;
    using H = Half2Of<T>;
    const float* cosv = a.cosv + angle_row * (a.rot_dim / 2) + p * 8;
    const float* sinv = a.sinv + angle_row * (a.rot_dim / 2) + p * 8;
    auto turned = [](float lo, float hi, float c, float s, float& r0, float& r1) {
        r0 = __fsub_rn(__fmul_rn(lo, c), __fmul_rn(hi, s));
        r1 = __fadd_rn(__fmul_rn(hi, c), __fmul_rn(lo, s));
    };
    uint32_t w0[4] = {u0.x, u0.y, u0.z, u0.w}, w1[4] = {u1.x, u1.y, u1.z, u1.w};
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        const float4 c = __ldg(reinterpret_cast<const float4*>(cosv) + half), s = __ldg(reinterpret_cast<const float4*>(sinv) + half);
        float r0, r1, r2, r3;
        if (a.interleaved) {
            uint32_t (&w)[4] = half ? w1 : w0;                         // four pairs within one vector
            turned(H::lo(w[0]), H::hi(w[0]), c.x, s.x, r0, r1);
            w[0] = H::pack(r0, r1);
            turned(H::lo(w[1]), H::hi(w[1]), c.y, s.y, r0, r1);
            w[1] = H::pack(r0, r1);
            turned(H::lo(w[2]), H::hi(w[2]), c.z, s.z, r0, r1);
            w[2] = H::pack(r0, r1);
            turned(H::lo(w[3]), H::hi(w[3]), c.w, s.w, r0, r1);
            w[3] = H::pack(r0, r1);
        } else {
            uint32_t &x = w0[2 * half], &y = w1[2 * half], &z = w0[2 * half + 1], &v = w1[2 * half + 1];
            turned(H::lo(x), H::lo(y), c.x, s.x, r0, r1);
            turned(H::hi(x), H::hi(y), c.y, s.y, r2, r3);
            x = H::pack(r0, r2);
            y = H::pack(r1, r3);
            turned(H::lo(z), H::lo(v), c.z, s.z, r0, r1);
            turned(H::hi(z), H::hi(v), c.w, s.w, r2, r3);
            z = H::pack(r0, r2);
            v = H::pack(r1, r3);
        }
    }
    u0 = make_uint4(w0[0], w0[1], w0[2], w0[3]);
    u1 = make_uint4(w1[0], w1[1], w1[2], w1[3]);
}

__device__ __forceinline__ int64_t angle_row_of(const AppendArgs& a, int t, int pos)
{
    const int p = a.positions ? a.positions[t] : pos;
    if (p < 0 || p >= a.n_pos) {
        dev_set_error(a.status, DEV_BAD_POSITION);
        return p < 0 ? 0 : a.n_pos - 1;
    }
    return p;
}

template <class T>
__device__ __forceinline__ void add_fixed(const uint4& u, int (&sum)[16], int at)
{
    using H = Half2Of<T>;
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        sum[at + 2 * i] += kv::fixed_of(H::lo(w[i]));
        sum[at + 2 * i + 1] += kv::fixed_of(H::hi(w[i]));
    }
}

template <class T, int D>
__global__ void __launch_bounds__(THREADS, 8) append_kernel(const AppendArgs a)
{
    constexpr int PAIRS = D / 16, ROWS = THREADS / PAIRS;    // threads per row, rows per pass
    const int p = threadIdx.x % PAIRS, r = threadIdx.x / PAIRS;
    int e0, e1;
    bool turn;
    pair_of(a, p, e0, e1, turn);
    cudaTriggerProgrammaticLaunchCompletion();
    cudaGridDependencySynchronize();

    if (static_cast<int>(blockIdx.x) >= a.n_kv_blocks) {
        // ---------------- queries ----------------
        const int64_t rows = static_cast<int64_t>(a.b.T) * a.n_heads;
        const int64_t first = static_cast<int64_t>(blockIdx.x - a.n_kv_blocks) * Q_ROWS;
        constexpr int N = Q_ROWS / ROWS;
        uint4 u0[N], u1[N];
        T* dst[N];
        int tok[N];
#pragma unroll
        for (int i = 0; i < N; ++i) {                                  // all reads first
            const int64_t row = first + i * ROWS + r;
            tok[i] = row < rows ? static_cast<int>(row / a.n_heads) : -1;
            if (tok[i] < 0) continue;
            const int h = static_cast<int>(row - static_cast<int64_t>(tok[i]) * a.n_heads);
            const T* src = static_cast<const T*>(a.q) + tok[i] * a.ldq + h * D;
            dst[i] = static_cast<T*>(a.q_out) + tok[i] * a.ld_qo + h * D;
            u0[i] = *reinterpret_cast<const uint4*>(src + e0);
            u1[i] = *reinterpret_cast<const uint4*>(src + e1);
        }
        int64_t angle[N];
#pragma unroll
        for (int i = 0; i < N; ++i) {
            angle[i] = 0;
            if (tok[i] < 0 || a.rot_dim == 0) continue;
            if (i > 0 && tok[i] == tok[i - 1]) { angle[i] = angle[i - 1]; continue; }
            int pos = 0;
            if (!a.positions) {
                const SeqSpan s = load_seq(a.b, seq_of_row(a.b, tok[i]), a.status);
                pos = max(s.kv - s.n + (tok[i] - s.q0), 0);            // a row before the first position is not stored: any angle
            }
            angle[i] = angle_row_of(a, tok[i], pos);
        }
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if (tok[i] < 0) continue;
            rotate<T>(a, p, turn, angle[i], u0[i], u1[i]);
            *reinterpret_cast<uint4*>(dst[i] + e0) = u0[i];
            *reinterpret_cast<uint4*>(dst[i] + e1) = u1[i];
        }
        return;
    }

    // ---------------- keys, values, summary of one (page, head) ----------------
    __shared__ int part[THREADS / 32][D];
    __shared__ int most[D / 32];
    const int head = blockIdx.x % a.n_kv_heads, item = blockIdx.x / a.n_kv_heads;
    int seq = item, idx = 0;
    if (!a.one_page_per_seq) {
        const KvBatchDev& b = a.b;
        const int shift = a.page_shift;
        const bool found = locate_item(b.n_seqs, item, [&](int i) {
            const SeqSpan s = load_seq(b, i, nullptr);
            return s.n == 0 || s.kv == 0 ? 0 : ((s.kv - 1) >> shift) - (max(s.kv - s.n, 0) >> shift) + 1;
        }, seq, idx);
        if (!found) return;
    }
    const SeqSpan s = load_seq(a.b, seq, a.status);
    if (s.n == 0 || s.kv == 0) return;
    const int start = s.kv - s.n;                                   // position of the first new row, may be negative
    const int block = (max(start, 0) >> a.page_shift) + idx;
    const int base = block << a.page_shift;
    const int end = min(s.kv - base, a.page_size);                  // positions of the block that exist
    const int fresh = max(start - base, 0);                         // the first of them that is new
    const int page = a.b.pages[seq * a.b.ld_pages + block];
    if (page < 0 || page >= a.n_pages) {
        if (threadIdx.x == 0) dev_set_error(a.status, DEV_BAD_PAGE);
        return;
    }
    T* kc = static_cast<T*>(a.kc) + page * a.k_page + static_cast<int64_t>(head) * a.page_size * D;
    T* vc = static_cast<T*>(a.vc) + page * a.v_page + static_cast<int64_t>(head) * a.page_size * D;
    int sum[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) sum[i] = 0;
    const int t_base = s.q0 + base - start;                         // row of the new token at position `base`
    for (int x = (a.code ? 0 : fresh) + r; x < end; x += ROWS) {
        const bool held = x < fresh;
        const int64_t t = t_base + x;
        const T* src = held ? kc + x * D : static_cast<const T*>(a.k) + t * a.ldk + head * D;
        uint4 u0 = *reinterpret_cast<const uint4*>(src + e0), u1 = *reinterpret_cast<const uint4*>(src + e1);
        if (!held) {
            const T* val = static_cast<const T*>(a.v) + t * a.ldv + head * D;
            const uint4 v0 = *reinterpret_cast<const uint4*>(val + p * 16), v1 = *reinterpret_cast<const uint4*>(val + p * 16 + 8);
            if (turn) rotate<T>(a, p, turn, angle_row_of(a, t_base + x, base + x), u0, u1);
            *reinterpret_cast<uint4*>(kc + x * D + e0) = u0;
            *reinterpret_cast<uint4*>(kc + x * D + e1) = u1;
            *reinterpret_cast<uint4*>(vc + x * D + p * 16) = v0;
            *reinterpret_cast<uint4*>(vc + x * D + p * 16 + 8) = v1;
        }
        if (a.code) {
            add_fixed<T>(u0, sum, 0);
            add_fixed<T>(u1, sum, 8);
        }
    }
    if (!a.code) return;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
#pragma unroll
    for (int i = 0; i < 16; ++i)
#pragma unroll
        for (int o = PAIRS; o < 32; o <<= 1) sum[i] += __shfl_xor_sync(0xffffffffu, sum[i], o);
    if (lane < PAIRS)
#pragma unroll
        for (int i = 0; i < 8; ++i) { part[warp][e0 + i] = sum[i]; part[warp][e1 + i] = sum[8 + i]; }
    __syncthreads();
    int total = 0;
    const int d = threadIdx.x;
    if (d < D) {
#pragma unroll
        for (int w = 0; w < THREADS / 32; ++w) total += part[w][d];
        const int m = __reduce_max_sync(0xffffffffu, abs(total));
        if (lane == 0) most[warp] = m;
    }
    __syncthreads();
    if (d < D) {
        int m = most[0];
#pragma unroll
        for (int w = 1; w < D / 32; ++w) m = max(m, most[w]);
        const int64_t at = static_cast<int64_t>(page) * a.n_kv_heads + head;
        const float most_f = __int2float_rn(max(m, 1));
        a.code[at * D + d] = static_cast<int8_t>(kv::code_of(total, most_f, 1.0f / most_f));
        if (d == 0) a.scale[at] = __fdiv_rn(__int2float_rn(m), __int2float_rn(end));
    }
}

}  // namespace

s3_status launch_kv_append(const KvCacheState& c, const KvBatchDev& b, const s3_rope* rope, const int32_t* d_positions,
                           const void* d_q, int64_t ldq, int n_heads, void* d_q_out, int64_t ld_qo, const void* d_k, int64_t ldk,
                           const void* d_v, int64_t ldv, uint32_t* d_status, cudaStream_t stream)
{
    AppendArgs a;
    a.b = b;
    a.cosv = rope ? rope->d_cos : nullptr;
    a.sinv = rope ? rope->d_sin : nullptr;
    a.n_pos = rope ? rope->n_pos : 0;
    a.rot_dim = rope ? rope->rot_dim : 0;
    a.interleaved = rope ? rope->interleaved != 0 : 0;
    a.positions = d_positions;
    a.q = d_q; a.k = d_k; a.v = d_v;
    a.q_out = d_q_out;
    a.ldq = ldq; a.ld_qo = ld_qo; a.ldk = ldk; a.ldv = ldv;
    a.n_heads = n_heads;
    a.n_kv_heads = c.d.n_kv_heads;
    a.page_size = c.d.page_size;
    a.page_shift = c.page_shift;
    a.n_pages = c.d.n_pages;
    a.kc = c.d.d_k; a.vc = c.d.d_v;
    a.k_page = c.d.k_page_stride; a.v_page = c.d.v_page_stride;
    a.code = c.d.d_code;
    a.scale = c.d.d_scale;
    a.status = d_status;
    // Pages a sequence of n new rows can touch: (n + page_size - 2) / page_size + 1. When that is one (a decoding step) item =
    // sequence; otherwise the items are counted along the batch (at most T / page_size + 2 per sequence).
    a.one_page_per_seq = (b.max_q + c.d.page_size - 2) / c.d.page_size + 1 == 1;
    const int64_t items = a.one_page_per_seq ? b.n_seqs : static_cast<int64_t>(b.T) / c.d.page_size + 2 * static_cast<int64_t>(b.n_seqs);
    const int64_t kv_blocks = items * c.d.n_kv_heads;
    const int64_t q_blocks = d_q ? (static_cast<int64_t>(b.T) * n_heads + Q_ROWS - 1) / Q_ROWS : 0;
    S3_REQUIRE(kv_blocks + q_blocks < (int64_t(1) << 31), S3_ERR_UNSUPPORTED, "the batch needs too many thread blocks");
    a.n_kv_blocks = static_cast<int>(kv_blocks);
    const dim3 grid(static_cast<unsigned>(kv_blocks + q_blocks));
    const bool wide = c.d.head_dim == 128;
    if (c.d.dtype == S3_BF16)
        return wide ? launch_overlapped(append_kernel<__nv_bfloat16, 128>, grid, THREADS, 0, stream, a)
                    : launch_overlapped(append_kernel<__nv_bfloat16, 64>, grid, THREADS, 0, stream, a);
    return wide ? launch_overlapped(append_kernel<__half, 128>, grid, THREADS, 0, stream, a)
                : launch_overlapped(append_kernel<__half, 64>, grid, THREADS, 0, stream, a);
}

}  // namespace s3
