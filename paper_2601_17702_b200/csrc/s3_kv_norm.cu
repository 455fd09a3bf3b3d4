// Append to a paged key / value cache with a norm per head before the rotation, and to pages that hold 8 bits; rows read back.
//
//   y[d] = x[d] / sqrt(mean_d x[d]^2 + eps) weight[d],  rotated pairs of y,  one rounding;  8 bits: code[d] = rint(127 y[d] / max |y|)
//
// Laid out like the plain append: the first n_touched * n_kv_heads blocks take one (page that holds a new token, key head) with its keys,
// values and, when the cache has them, its summary; the rest take query rows, two to a thread. D / 16 threads own a row, 16 elements each: both
// halves of every rotation pair are in one thread, the norm and the largest magnitude cross the row's threads by shuffles, so a row is
// read once and written once. Bound by memory traffic, as the plain append is.
//
// 16-bit rows are worked on in fp32. Keys that become codes are worked on in 64 bits: a code changes where 127 y / max crosses a half, and
// in fp32 the order of the norm's sum would decide some 30 of a million codes; in 64 bits a code is in effect a function of the formula.
// The 64-bit pipe has half the rate of the 32-bit one here and the key heads are few, so it hides behind the copies.
#include "s3_kernels.cuh"
#include "s3_kv.cuh"

namespace s3 {
namespace {

using kv::Half2Of;

constexpr int THREADS = 128;
constexpr int Q_PASSES = 2;                // query rows per thread

struct NormAppendArgs {
    KvBatchDev b;
    const float *cosv, *sinv;
    int n_pos, rot_dim, interleaved;
    const float *q_weight, *k_weight;      // null: no norm
    int per_head;
    float eps;
    const int32_t* positions;
    const void *q, *k, *v;
    void* q_out;
    int64_t ldq, ld_qo, ldk, ldv;
    int n_heads, n_kv_heads, page_size, page_shift, n_pages;
    void *kc, *vc;
    int64_t k_page, v_page;
    float *k_scale, *v_scale;
    int8_t* code;
    float* scale;
    int one_page_per_seq, n_kv_blocks;
    uint32_t* status;
};

// A thread's 16 elements of a row: two runs of eight, e0 and e1. Where the head is rotated by halves they are the two sides of eight
// pairs, else consecutive.
struct Place {
    int e0, e1;
    bool turn;
};

__device__ __forceinline__ Place place_of(const NormAppendArgs& a, int p)
{
    const bool turn = p * 16 < a.rot_dim;
    if (turn && !a.interleaved) return Place{p * 8, a.rot_dim / 2 + p * 8, true};
    return Place{p * 16, p * 16 + 8, turn};
}

template <class T>
__device__ __forceinline__ void unpack(const uint4& u, float* x)
{
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { x[2 * i] = Half2Of<T>::lo(w[i]); x[2 * i + 1] = Half2Of<T>::hi(w[i]); }
}
template <class T>
__device__ __forceinline__ uint4 packed(const float* x)
{
    using H = Half2Of<T>;
    return make_uint4(H::pack(x[0], x[1]), H::pack(x[2], x[3]), H::pack(x[4], x[5]), H::pack(x[6], x[7]));
}

__device__ __forceinline__ float root(float x) { return sqrtf(x); }
__device__ __forceinline__ double root(double x) { return sqrt(x); }

// The row's norm, in the precision of F; a row's threads are LANES neighbours of a warp.
template <int D, int LANES, class F>
__device__ __forceinline__ void normed(F (&x)[16], const float* weight, const Place& at, float eps)
{
    F sum = 0;
#pragma unroll
    for (int i = 0; i < 16; ++i) sum += x[i] * x[i];
#pragma unroll
    for (int o = 1; o < LANES; o <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    F add = F(eps);
    if constexpr (sizeof(F) == 4) {
        // rows of numbers beyond 2^60, whose squares leave fp32: again, by 2^-70
        const bool over = !(sum <= 3.4028235e38f);
        if (__any_sync(0xffffffffu, over)) {
            const F by = over ? 8.470329472543003e-22f : 1.0f;
            F again = 0;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                x[i] *= by;
                again += x[i] * x[i];
            }
#pragma unroll
            for (int o = 1; o < LANES; o <<= 1) again += __shfl_xor_sync(0xffffffffu, again, o);
            sum = again;
            add *= by * by;
        }
    }
    const F inv = F(1) / root(sum / F(D) + add);
#pragma unroll
    for (int i = 0; i < 16; i += 4) {
        const float4 w = *reinterpret_cast<const float4*>(weight + (i < 8 ? at.e0 + i : at.e1 + i - 8));
        x[i] *= inv * F(w.x);
        x[i + 1] *= inv * F(w.y);
        x[i + 2] *= inv * F(w.z);
        x[i + 3] *= inv * F(w.w);
    }
}

// Pair i of the eight: (x[i], x[8 + i]), or interleaved (x[2 i], x[2 i + 1]). In fp32 products and sums are rounded one by one, as in the
// plain append.
__device__ __forceinline__ void turned(float& lo, float& hi, float c, float s)
{
    const float r = __fsub_rn(__fmul_rn(lo, c), __fmul_rn(hi, s));
    hi = __fadd_rn(__fmul_rn(hi, c), __fmul_rn(lo, s));
    lo = r;
}
__device__ __forceinline__ void turned(double& lo, double& hi, float c, float s)
{
    const double r = lo * c - hi * s;
    hi = hi * c + lo * s;
    lo = r;
}
template <class F>
__device__ __forceinline__ void rotated(const NormAppendArgs& a, F (&x)[16], int p, int64_t angle_row)
{
    const float* cosv = a.cosv + angle_row * (a.rot_dim / 2) + p * 8;
    const float* sinv = a.sinv + angle_row * (a.rot_dim / 2) + p * 8;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        const float4 c = __ldg(reinterpret_cast<const float4*>(cosv) + half), s = __ldg(reinterpret_cast<const float4*>(sinv) + half);
        const float cs[4] = {c.x, c.y, c.z, c.w}, sn[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int k = 4 * half + i;
            if (a.interleaved) turned(x[2 * k], x[2 * k + 1], cs[i], sn[i]);
            else turned(x[k], x[8 + k], cs[i], sn[i]);
        }
    }
}

__device__ __forceinline__ int64_t angle_row_of(const NormAppendArgs& a, int t, int pos)
{
    const int p = a.positions ? a.positions[t] : pos;
    if (p < 0 || p >= a.n_pos) {
        dev_set_error(a.status, DEV_BAD_POSITION);
        return p < 0 ? 0 : a.n_pos - 1;
    }
    return p;
}

// What counts of a number that is to be held in 8 bits.
template <class T, class F>
__device__ __forceinline__ F counted(F x)
{
    constexpr F most = Half2Of<T>::is_bf16 ? kv::kMostBf16 : kv::kMostF16;
    return x != x ? F(0) : x > most ? most : x < -most ? -most : x;
}

__device__ __forceinline__ int low_word(float x) { return __float_as_int(x); }
__device__ __forceinline__ int low_word(double x) { return __double2loint(x); }

// Codes and scale of a row, 16 elements in each of LANES threads. The division itself is taken only next to a half, where the product with
// the reciprocal may fall on the other side; values of 16 bits may lie exactly on a half, and ties go to the even code.
// fp32 is enough for rows that come in 16 bits: 127 x is exact, and the quotient of a number of 18 bits by one of 11 is either a half or
// further from it than fp32 rounds.
template <class T, int LANES, class F>
__device__ __forceinline__ float coded(F (&x)[16], uint32_t (&w)[4])
{
    F most = 0;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        x[i] = counted<T>(x[i]);
        const F m = x[i] < 0 ? -x[i] : x[i];
        most = m > most ? m : most;
    }
#pragma unroll
    for (int o = 1; o < LANES; o <<= 1) {
        const F other = __shfl_xor_sync(0xffffffffu, most, o);
        most = other > most ? other : most;
    }
    const bool some = most >= F(kv::kLeastMagnitude);
    const F inv = some ? F(127) / most : F(0);
    constexpr F near = sizeof(F) == 8 ? F(1e-9) : F(1e-3);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        uint32_t word = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            // the sum with 1.5 times the number whose last place is 1 is rounded to a whole number, which its low bits hold
            constexpr F whole = sizeof(F) == 8 ? F(6755399441055744.0) : F(12582912.0);
            const F r = x[4 * i + j] * inv, t = r + whole, off = r - (t - whole);
            int c = low_word(t);
            if ((off < 0 ? -off : off) > F(0.5) - near && some) c = low_word(x[4 * i + j] * F(127) / most + whole);
            word |= (static_cast<uint32_t>(c) & 0xffu) << (8 * j);
        }
        w[i] = word;
    }
    return some ? static_cast<float>(most / F(127)) : 0.0f;
}

__device__ __forceinline__ void add_codes(uint32_t word, float scale, int* sum)
{
#pragma unroll
    for (int j = 0; j < 4; ++j) sum[j] += kv::fixed_of(__fmul_rn(static_cast<float>(static_cast<int8_t>(word >> (8 * j))), scale));
}
template <class T>
__device__ __forceinline__ void add_fixed(const uint4& u, int* sum)
{
    float x[8];
    unpack<T>(u, x);
#pragma unroll
    for (int i = 0; i < 8; ++i) sum[i] += kv::fixed_of(x[i]);
}

template <class T, int D, bool I8>
__global__ void __launch_bounds__(THREADS, 8) append_norm_kernel(const NormAppendArgs a)
{
    constexpr int LANES = D / 16, ROWS = THREADS / LANES;    // threads per row, rows per pass
    const int p = threadIdx.x % LANES, r = threadIdx.x / LANES;
    const Place at = place_of(a, p);
    cudaTriggerProgrammaticLaunchCompletion();
    cudaGridDependencySynchronize();

    if (static_cast<int>(blockIdx.x) >= a.n_kv_blocks) {
        // ---------------- queries ----------------
        const int64_t rows = static_cast<int64_t>(a.b.T) * a.n_heads;
        const int64_t first = static_cast<int64_t>(blockIdx.x - a.n_kv_blocks) * (ROWS * Q_PASSES);
        constexpr int N = Q_PASSES;
        uint4 u0[N], u1[N];
        int tok[N], head[N];
#pragma unroll
        for (int i = 0; i < N; ++i) {                                  // all reads first
            const int64_t row = first + i * ROWS + r;
            tok[i] = row < rows ? static_cast<int>(row / a.n_heads) : -1;
            head[i] = static_cast<int>(row - static_cast<int64_t>(tok[i]) * a.n_heads);
            u0[i] = u1[i] = make_uint4(0, 0, 0, 0);                    // a row that is not there goes through the shuffles as zeros
            if (tok[i] < 0) continue;
            const T* src = static_cast<const T*>(a.q) + tok[i] * a.ldq + head[i] * D;
            u0[i] = *reinterpret_cast<const uint4*>(src + at.e0);
            u1[i] = *reinterpret_cast<const uint4*>(src + at.e1);
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
            float x[16];
            unpack<T>(u0[i], x);
            unpack<T>(u1[i], x + 8);
            if (a.q_weight) normed<D, LANES>(x, a.q_weight + (a.per_head && tok[i] >= 0 ? head[i] * D : 0), at, a.eps);
            if (tok[i] < 0) continue;
            if (at.turn) rotated(a, x, p, angle[i]);
            T* dst = static_cast<T*>(a.q_out) + tok[i] * a.ld_qo + head[i] * D;
            *reinterpret_cast<uint4*>(dst + at.e0) = packed<T>(x);
            *reinterpret_cast<uint4*>(dst + at.e1) = packed<T>(x + 8);
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
    const int64_t page_head = static_cast<int64_t>(page) * a.n_kv_heads + head;
    const int64_t k_at = page * a.k_page + static_cast<int64_t>(head) * a.page_size * D, v_at = page * a.v_page + static_cast<int64_t>(head) * a.page_size * D;
    const float* weight = a.k_weight ? a.k_weight + (a.per_head ? head * D : 0) : nullptr;
    int sum[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) sum[i] = 0;
    const int t_base = s.q0 + base - start;                         // row of the new token at position `base`
    const int from = a.code ? 0 : fresh;
    for (int x0 = from; x0 < end; x0 += ROWS) {                      // every thread takes part in the shuffles
        const int x = x0 + r;
        const bool here = x < end, held = here && x < fresh, add = here && !held;
        const int64_t t = t_base + x;
        uint4 u0 = make_uint4(0, 0, 0, 0), u1 = u0, v0 = u0, v1 = u0;
        if (add) {
            const T* src = static_cast<const T*>(a.k) + t * a.ldk + head * D;
            const T* val = static_cast<const T*>(a.v) + t * a.ldv + head * D;
            u0 = *reinterpret_cast<const uint4*>(src + at.e0);
            u1 = *reinterpret_cast<const uint4*>(src + at.e1);
            v0 = *reinterpret_cast<const uint4*>(val + p * 16);
            v1 = *reinterpret_cast<const uint4*>(val + p * 16 + 8);
        }
        const int64_t angle = add && at.turn ? angle_row_of(a, t_base + x, base + x) : 0;
        if constexpr (I8) {
            int8_t *kc = static_cast<int8_t*>(a.kc) + k_at + x * D, *vc = static_cast<int8_t*>(a.vc) + v_at + x * D;
            float f[16];
            double y[16];
            uint32_t w[4], z[4];
            unpack<T>(u0, f);
            unpack<T>(u1, f + 8);
#pragma unroll
            for (int i = 0; i < 16; ++i) y[i] = f[i];
            if (weight) normed<D, LANES>(y, weight, at, a.eps);
            if (at.turn) rotated(a, y, p, angle);
            float scale = coded<T, LANES>(y, w);
            unpack<T>(v0, f);
            unpack<T>(v1, f + 8);
            const float v_scale = coded<T, LANES>(f, z);
            if (add) {
                *reinterpret_cast<uint2*>(kc + at.e0) = make_uint2(w[0], w[1]);
                *reinterpret_cast<uint2*>(kc + at.e1) = make_uint2(w[2], w[3]);
                *reinterpret_cast<uint4*>(vc + p * 16) = make_uint4(z[0], z[1], z[2], z[3]);
                if (p == 0) {
                    a.k_scale[(page_head << a.page_shift) + x] = scale;
                    a.v_scale[(page_head << a.page_shift) + x] = v_scale;
                }
            } else if (held) {
                const uint2 lo = *reinterpret_cast<const uint2*>(kc + at.e0), hi = *reinterpret_cast<const uint2*>(kc + at.e1);
                w[0] = lo.x; w[1] = lo.y; w[2] = hi.x; w[3] = hi.y;
                scale = a.k_scale[(page_head << a.page_shift) + x];
            }
            if (a.code && here) {
#pragma unroll
                for (int i = 0; i < 4; ++i) add_codes(w[i], scale, sum + 4 * i);
            }
        } else {
            T *kc = static_cast<T*>(a.kc) + k_at + x * D, *vc = static_cast<T*>(a.vc) + v_at + x * D;
            float f[16];
            unpack<T>(u0, f);
            unpack<T>(u1, f + 8);
            if (weight) normed<D, LANES>(f, weight, at, a.eps);
            if (at.turn) rotated(a, f, p, angle);
            u0 = packed<T>(f);
            u1 = packed<T>(f + 8);
            if (add) {
                *reinterpret_cast<uint4*>(kc + at.e0) = u0;
                *reinterpret_cast<uint4*>(kc + at.e1) = u1;
                *reinterpret_cast<uint4*>(vc + p * 16) = v0;
                *reinterpret_cast<uint4*>(vc + p * 16 + 8) = v1;
            } else if (held) {
                u0 = *reinterpret_cast<const uint4*>(kc + at.e0);
                u1 = *reinterpret_cast<const uint4*>(kc + at.e1);
            }
            if (a.code && here) {
                add_fixed<T>(u0, sum);
                add_fixed<T>(u1, sum + 8);
            }
        }
    }
    if (!a.code) return;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
#pragma unroll
    for (int i = 0; i < 16; ++i)
#pragma unroll
        for (int o = LANES; o < 32; o <<= 1) sum[i] += __shfl_xor_sync(0xffffffffu, sum[i], o);
    if (lane < LANES) {
#pragma unroll
        for (int i = 0; i < 8; ++i) { part[warp][at.e0 + i] = sum[i]; part[warp][at.e1 + i] = sum[8 + i]; }
    }
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
        const float most_f = __int2float_rn(max(m, 1));
        a.code[page_head * D + d] = static_cast<int8_t>(kv::code_of(total, most_f, 1.0f / most_f));
        if (d == 0) a.scale[page_head] = __fdiv_rn(__int2float_rn(m), __int2float_rn(end));
    }
}

// Rows of the batch as the cache holds them: D / 16 threads per (row, key head), keys and values. A copy with a product; the rows' addresses
// are found thread by thread.
struct ReadArgs {
    KvBatchDev b;
    int n_kv_heads, page_size, page_shift, n_pages;
    const void *kc, *vc;
    int64_t k_page, v_page;
    const float *k_scale, *v_scale;
    void *k, *v;
    int64_t ldk, ldv;
    uint32_t* status;
};

template <class T, int D, bool I8>
__device__ __forceinline__ void read_row(const void* pages, int64_t from, float scale, bool there, T* dst)
{
    uint4 y0 = make_uint4(0, 0, 0, 0), y1 = y0;
    if (there) {
        if constexpr (I8) {
            const uint4 u = *reinterpret_cast<const uint4*>(static_cast<const int8_t*>(pages) + from);
            const uint32_t w[4] = {u.x, u.y, u.z, u.w};
            float x[16];
#pragma unroll
            for (int i = 0; i < 4; ++i) {                              // (a conversion of each code takes four times as long)
                using B = Half2Of<__nv_bfloat16>;
                uint32_t lo, hi;
                kv::widen<__nv_bfloat16>(w[i], lo, hi);
                x[4 * i] = B::lo(lo) * scale;
                x[4 * i + 1] = B::hi(lo) * scale;
                x[4 * i + 2] = B::lo(hi) * scale;
                x[4 * i + 3] = B::hi(hi) * scale;
            }
            y0 = packed<T>(x);
            y1 = packed<T>(x + 8);
        } else {
            y0 = *reinterpret_cast<const uint4*>(static_cast<const T*>(pages) + from);
            y1 = *reinterpret_cast<const uint4*>(static_cast<const T*>(pages) + from + 8);
        }
    }
    *reinterpret_cast<uint4*>(dst) = y0;
    *reinterpret_cast<uint4*>(dst + 8) = y1;
}

template <class T, int D, bool I8>
__global__ void __launch_bounds__(THREADS) read_kernel(const ReadArgs a)
{
    constexpr int LANES = D / 16;
    cudaTriggerProgrammaticLaunchCompletion();
    cudaGridDependencySynchronize();
    const int64_t i = static_cast<int64_t>(blockIdx.x) * THREADS + threadIdx.x, row_head = i / LANES;
    if (row_head >= static_cast<int64_t>(a.b.T) * a.n_kv_heads) return;
    const int p = static_cast<int>(i % LANES), t = static_cast<int>(row_head / a.n_kv_heads);
    const int head = static_cast<int>(row_head - static_cast<int64_t>(t) * a.n_kv_heads);
    const int seq = seq_of_row(a.b, t);
    const SeqSpan s = load_seq(a.b, seq, a.status);
    const int pos = s.kv - s.n + (t - s.q0);
    bool there = t < s.q0 + s.n && pos >= 0 && pos < s.kv;
    int page = 0;
    if (there) {
        page = a.b.pages[seq * a.b.ld_pages + (pos >> a.page_shift)];
        if (page < 0 || page >= a.n_pages) {
            dev_set_error(a.status, DEV_BAD_PAGE);
            there = false;
            page = 0;
        }
    }
    const int row = pos & (a.page_size - 1);
    const int64_t in_page = (static_cast<int64_t>(head) * a.page_size + row) * D + p * 16, scale_at = ((static_cast<int64_t>(page) * a.n_kv_heads + head) << a.page_shift) + row;
    if (a.k) read_row<T, D, I8>(a.kc, page * a.k_page + in_page, I8 && there ? a.k_scale[scale_at] : 0.0f, there, static_cast<T*>(a.k) + t * a.ldk + head * D + p * 16);
    if (a.v) read_row<T, D, I8>(a.vc, page * a.v_page + in_page, I8 && there ? a.v_scale[scale_at] : 0.0f, there, static_cast<T*>(a.v) + t * a.ldv + head * D + p * 16);
}

template <class T, int D>
s3_status launch_append(const KvCacheState& c, const NormAppendArgs& a, dim3 grid, cudaStream_t stream)
{
    return c.k_scale ? launch_overlapped(append_norm_kernel<T, D, true>, grid, THREADS, 0, stream, a)
                     : launch_overlapped(append_norm_kernel<T, D, false>, grid, THREADS, 0, stream, a);
}
template <class T, int D>
s3_status launch_read(const KvCacheState& c, const ReadArgs& a, dim3 grid, cudaStream_t stream)
{
    return c.k_scale ? launch_overlapped(read_kernel<T, D, true>, grid, THREADS, 0, stream, a)
                     : launch_overlapped(read_kernel<T, D, false>, grid, THREADS, 0, stream, a);
}

}  // namespace

s3_status launch_kv_append_norm(const KvCacheState& c, const KvBatchDev& b, const s3_head_norm* norm, const s3_rope* rope, const int32_t* d_positions,
                                const void* d_q, int64_t ldq, int n_heads, void* d_q_out, int64_t ld_qo, const void* d_k, int64_t ldk,
                                const void* d_v, int64_t ldv, uint32_t* d_status, cudaStream_t stream)
{
    NormAppendArgs a;
    a.b = b;
    a.cosv = rope ? rope->d_cos : nullptr;
    a.sinv = rope ? rope->d_sin : nullptr;
    a.n_pos = rope ? rope->n_pos : 0;
    a.rot_dim = rope ? rope->rot_dim : 0;
    a.interleaved = rope ? rope->interleaved != 0 : 0;
    a.q_weight = norm ? norm->d_q_weight : nullptr;
    a.k_weight = norm ? norm->d_k_weight : nullptr;
    a.per_head = norm ? norm->per_head != 0 : 0;
    a.eps = norm ? norm->eps : 0.0f;
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
    a.k_scale = c.k_scale; a.v_scale = c.v_scale;
    a.code = c.d.d_code;
    a.scale = c.d.d_scale;
    a.status = d_status;
    // items as for the plain append
    a.one_page_per_seq = (b.max_q + c.d.page_size - 2) / c.d.page_size + 1 == 1;
    const int64_t items = a.one_page_per_seq ? b.n_seqs : static_cast<int64_t>(b.T) / c.d.page_size + 2 * static_cast<int64_t>(b.n_seqs);
    const int64_t kv_blocks = items * c.d.n_kv_heads;
    const int q_rows = THREADS / (c.d.head_dim / 16) * Q_PASSES;
    const int64_t q_blocks = d_q ? (static_cast<int64_t>(b.T) * n_heads + q_rows - 1) / q_rows : 0;
    S3_REQUIRE(kv_blocks + q_blocks < (int64_t(1) << 31), S3_ERR_UNSUPPORTED, "the batch needs too many thread blocks");
    a.n_kv_blocks = static_cast<int>(kv_blocks);
    const dim3 grid(static_cast<unsigned>(kv_blocks + q_blocks));
    const bool wide = c.d.head_dim == 128;
    if (c.d.dtype == S3_BF16) return wide ? launch_append<__nv_bfloat16, 128>(c, a, grid, stream) : launch_append<__nv_bfloat16, 64>(c, a, grid, stream);
    return wide ? launch_append<__half, 128>(c, a, grid, stream) : launch_append<__half, 64>(c, a, grid, stream);
}

s3_status launch_kv_read(const KvCacheState& c, const KvBatchDev& b, void* d_k, int64_t ldk, void* d_v, int64_t ldv, uint32_t* d_status, cudaStream_t stream)
{
    const ReadArgs a{b, c.d.n_kv_heads, c.d.page_size, c.page_shift, c.d.n_pages, c.d.d_k, c.d.d_v, c.d.k_page_stride, c.d.v_page_stride,
                     c.k_scale, c.v_scale, d_k, d_v, ldk, ldv, d_status};
    const int64_t threads = static_cast<int64_t>(b.T) * c.d.n_kv_heads * (c.d.head_dim / 16), blocks = (threads + THREADS - 1) / THREADS;
    S3_REQUIRE(blocks < (int64_t(1) << 31), S3_ERR_UNSUPPORTED, "the batch needs too many thread blocks");
    const dim3 grid(static_cast<unsigned>(blocks));
    const bool wide = c.d.head_dim == 128;
    if (c.d.dtype == S3_BF16) return wide ? launch_read<__nv_bfloat16, 128>(c, a, grid, stream) : launch_read<__nv_bfloat16, 64>(c, a, grid, stream);
    return wide ? launch_read<__half, 128>(c, a, grid, stream) : launch_read<__half, 64>(c, a, grid, stream);
}

}  // namespace s3
