// Attention of a few query rows (at most 16 per item and key head) over a paged cache: decoding steps and lists per token.
//
//   out = sum_j p_j v_j / sum_j p_j,  p_j = 2^(scale log2e q.k_j - m)      one pass, running reference m and sum
//
// Bound by reading keys and values once (HBM, or the L2 cache when tokens list the same blocks). Two persistent thread blocks
// per SM walk the work (units of one item and one key head, or pieces of them). Warp 4 reads a unit's lengths, list and table entries, copies its
// query rows and then its 64-key tiles of K and V (TMA, page by page) into a ring of shared-memory slots, and goes on to the next
// unit while the others still compute: a unit's start (four dependent reads before the first key arrives, about 5 us with one
// thread block per unit) and its end (joining the warps) hide behind the copies.
// Warps 0-3 take 16 keys of every tile each and keep their own reference, sum and accumulator in registers, so the warps meet
// only at the end of a unit. Both products are taken transposed, S^T = K Q^T and O^T = V^T P^T (mma.sync m16n8k16): the 16-wide
// side of the instruction holds keys and dimensions, the 8-wide side the query rows, of which a group of 4 or 7 fills most.
// P^T changes its fragment form in registers (movmatrix). The reference moves only when a score exceeds it by 2^8 (f16: 2^15, see
// WeightRange), which one warp vote decides; weights stay inside either type. With this few rows per key the work is a copy.
// Measured on a B200 whose copies run at 6.53 TB/s: one token of 4 x 8 heads over 131072 keys 92 us (5.9 TB/s); 64 tokens over up to
// 8192 keys 94 us; 1024 tokens over 16 of 512 blocks each 327 us, where the 4.3 GB through the SMs' read ports bound (245 us at 64 bytes
// per clock and SM), 93 % of them hits in L2.
#include <string.h>

#include <type_traits>

#include "s3_kernels.cuh"
#include "s3_kv.cuh"

namespace s3 {
namespace {

using namespace kv;

constexpr int TILE = 64;                  // keys per tile
constexpr int WARPS = 4;                  // compute warps
constexpr int THREADS = 32 * (WARPS + 1);

struct Maps {
    alignas(64) unsigned char k[128], v[128];
};

// What the producer tells the compute warps about a unit.
struct UnitInfo {
    int rows, n_tiles, tok0, pos0, pos_last, kv, head, slot;       // rows 0: no more units
};

// NT: groups of 8 query rows. Two thread blocks per SM have 113 KB of shared memory each.
template <int D, int NT>
struct Layout {
    static constexpr int STAGE = 2 * TILE * D * 2;
    static constexpr int STAGES = (D == 128 ? 3 : 6) - (NT == 2 ? 1 : 0) * (D == 128 ? 1 : 2);
    static constexpr int PITCH = D + 4;                              // floats; rows of two lanes of a quad fall 8 banks apart
    static constexpr int Q_PITCH = D * 2 + 16;                       // bytes
    static constexpr int SLOTS = STAGES * STAGE;                     // two accumulators on their way to another warp
    static constexpr int SLOT = NT * 8 * PITCH * 4;
    static constexpr int Q = SLOTS + 2 * SLOT;
    static constexpr int TOTAL = Q + 2 * NT * 8 * Q_PITCH;
    static_assert(TOTAL + 1024 + 1024 <= 114 * 1024, "two thread blocks per SM");
};

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
__device__ __forceinline__ uint32_t transpose8(uint32_t x)
{
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
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
// Untiled copy of bytes (a multiple of 16, both addresses on 16-byte boundaries) into this block's shared memory.
__device__ __forceinline__ void bulk_load(void* dst, const void* src, uint32_t bytes, uint64_t* bar)
{
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(smem_u32(dst)), "l"(src),
                 "r"(bytes), "r"(smem_u32(bar)) : "memory");
}

template <class T, int D, int NT>
__global__ void __launch_bounds__(THREADS, 2) split_kernel(const __grid_constant__ Maps maps, const __grid_constant__ AttnArgs a)
{
    using L = Layout<D, NT>;
    using Range = WeightRange<T>;
    constexpr int STAGES = L::STAGES;
    extern __shared__ __align__(1024) unsigned char ring[];           // swizzled tiles start on 1024-byte boundaries
    __shared__ uint64_t full_bar[STAGES], empty_bar[STAGES], unit_full[2], unit_empty[2];
    __shared__ uint64_t from2, from3, from1, free0, free1;            // accumulators 2 -> 0, 3 -> 1, 1 -> 0; slots free again
    __shared__ UnitInfo infos[2];
    __shared__ int pos16[STAGES][4];                                  // first position of each 16 keys of a tile, -1: none
    __shared__ float red_m[2][NT * 8], red_l[2][NT * 8];
    __shared__ uint32_t abort_word;
    volatile uint32_t* abort_flag = &abort_word;

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    cudaTriggerProgrammaticLaunchCompletion();       // the join's blocks may take their places; they wait for this grid's end
    if (threadIdx.x == 0) {
        for (int i = 0; i < STAGES; ++i) { mbar_init(&full_bar[i], 1); mbar_init(&empty_bar[i], WARPS); }
        for (int i = 0; i < 2; ++i) { mbar_init(&unit_full[i], 1); mbar_init(&unit_empty[i], WARPS); }
        mbar_init(&from1, 1); mbar_init(&from2, 1); mbar_init(&from3, 1); mbar_init(&free0, 1); mbar_init(&free1, 1);
        abort_word = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }

    // token and head of a query row, row < 16: an integer division costs some 100 clocks
    const uint32_t group_inv = (65536u + a.group - 1) / a.group;
    auto token_of = [&](int row) { return static_cast<int>(row * group_inv >> 16); };
    auto head_of = [&](int row) { return row - token_of(row) * a.group; };
    auto give_up = [&](uint32_t code) {
        if (lane == 0) { dev_set_error(a.status, code); *abort_flag = 1; }
    };

    if (warp == WARPS) {
        // ---------------- producer ----------------
        const int box = a.box_rows, per_tile = TILE / box, group_tiles = 32 / per_tile;
        const int lane_tile = lane / per_tile, lane_box = lane % per_tile;
        int tiles = 0, units = 0;                                     // pushed so far
        bool ok = true;
        prefetch_tables(a);
        if (lane == 0) {
            prefetch_map(maps.k);
            prefetch_map(maps.v);
        }
        Walk<TILE> walk;
        Segment g;
        cudaGridDependencySynchronize();
        walk.start(a);
        // A lane per box: the lanes read the table entries of the next 32 boxes together, one group ahead of the copies, so that
        // no copy waits for its page number. The next segment is looked up while the ring is full.
        auto look_up = [&](const Segment& of, int t, int& page, int& pos) {       // this lane's box of tile t + lane_tile
            const int v = of.v_base + (of.t_lo + t + lane_tile) * TILE + lane_box * box;
            page = pos = -1;
            if (t + lane_tile >= of.t_hi - of.t_lo) return;
            if (a.list_mode == LIST_NONE) pos = v <= of.it.pos_last && v + box > first_seen(a, of.it) ? v : -1;      // boxes before the window are not there
            else if (v < a.s << a.page_shift) {
                const int id = a.lists[(static_cast<int64_t>(of.it.list) * a.list_heads + (a.list_heads == 1 ? 0 : of.head)) * a.s + (v >> a.page_shift)];
                // a block all of whose positions are out of sight counts as not listed
                if (id >= 0 && of.it.pos_last >= 0 && id <= (of.it.pos_last >> a.page_shift) && ((id + 1) << a.page_shift) > first_seen(a, of.it))
                    pos = (id << a.page_shift) + (v & (a.page_size - 1));
            }
            if (pos < 0 || pos >= of.it.kv) { pos = -1; return; }
            const int p = a.b.pages[of.it.seq * a.b.ld_pages + (pos >> a.page_shift)];
            page = p < 0 || p >= a.n_pages ? a.n_pages : p;            // beyond the map: reads as zeros
        };
        Segment ahead;
        int page, pos, next_page = -1, next_pos = -1;
        bool some = walk.next(a, g);
        if (some) look_up(g, 0, next_page, next_pos);
        __syncthreads();                                              // the barriers exist; the first reads ran meanwhile
        while (ok && some) {
            const AttnItem& it = g.it;
            const int head = g.head, pos_last = it.pos_last, n_tiles = g.t_hi - g.t_lo, rows = it.n_tok * a.group;
            const int ub = units & 1;
            if (units >= 2 && !__all_sync(0xffffffffu, mbar_wait(&unit_empty[ub], ((units >> 1) - 1) & 1, abort_flag))) {
                give_up(DEV_TIMEOUT_SMEM_EMPTY);
                break;
            }
            if (lane == 0) {
                infos[ub] = UnitInfo{rows, n_tiles, it.tok0, it.pos0, pos_last, it.kv, head, g.slot};
                mbar_expect_tx(&unit_full[ub], static_cast<uint32_t>(rows) * D * 2);
            }
            __syncwarp();
            if (lane < rows) {
                const T* src = static_cast<const T*>(a.q) + static_cast<int64_t>(it.tok0 + token_of(lane)) * a.ldq + (head * a.group + head_of(lane)) * D;
                bulk_load(ring + L::Q + (ub * NT * 8 + lane) * L::Q_PITCH, src, D * 2, &unit_full[ub]);
            }
            ++units;

            for (int t0 = 0; t0 < n_tiles && ok; t0 += group_tiles) {
                page = next_page;
                pos = next_pos;
                if (page == a.n_pages) dev_set_error(a.status, DEV_BAD_PAGE);
                const bool last_group = t0 + group_tiles >= n_tiles;
                if (!last_group) look_up(g, t0 + group_tiles, next_page, next_pos);
                for (int t = t0; t < min(n_tiles, t0 + group_tiles); ++t) {
                    const int st = tiles % STAGES, round = tiles / STAGES;
                    if (round > 0 && !__all_sync(0xffffffffu, mbar_wait(&empty_bar[st], (round - 1) & 1, abort_flag))) {
                        give_up(DEV_TIMEOUT_SMEM_EMPTY);
                        ok = false;
                        break;
                    }
                    const bool here = lane_tile == t - t0, mine = here && page >= 0;
                    if (here) {
                        const int units16 = box / 16;
#pragma unroll
                        for (int x = 0; x < TILE / 16; ++x) {
                            const int at = pos + 16 * x;               // whole 16-key units that no row can see are skipped
                            if (x < units16) pos16[st][lane_box * units16 + x] = mine && at <= pos_last && at < it.kv ? at : -1;
                        }
                    }
                    const uint32_t boxes = __popc(__ballot_sync(0xffffffffu, mine));
                    __syncwarp();
                    if (lane == 0) {
                        if (boxes) mbar_expect_tx(&full_bar[st], boxes * 2u * static_cast<uint32_t>(box) * D * 2);
                        else mbar_arrive(&full_bar[st]);
                    }
                    ++tiles;
                    __syncwarp();
                    if (mine) {
                        // a box holds its rows' first halves, then their second ones
                        unsigned char* dst = ring + st * L::STAGE + lane_box * box * D * 2;
                        const int row = pos & (a.page_size - 1);
                        tma_load_rows(dst, maps.k, row, head, page, &full_bar[st]);
                        tma_load_rows(dst + TILE * D * 2, maps.v, row, head, page, &full_bar[st]);
                    }
                    if (last_group && t == min(t0 + STAGES - 1, n_tiles - 1)) {
                        some = walk.next(a, ahead);
                        if (some) look_up(ahead, 0, next_page, next_pos);
                    }
                }
            }
            g = ahead;
        }
        if (lane == 0) walk.leave_cut(a);
        const int ub = units & 1;
        if (ok && units >= 2 && !__all_sync(0xffffffffu, mbar_wait(&unit_empty[ub], ((units >> 1) - 1) & 1, abort_flag)))
            give_up(DEV_TIMEOUT_SMEM_EMPTY);
        else if (ok && lane == 0) {
            infos[ub].rows = 0;
            mbar_arrive(&unit_full[ub]);
        }
        if (__any_sync(0xffffffffu, *abort_flag != 0) && lane == 0) {  // no copy may be in flight when the block leaves
            for (int i = max(0, tiles - STAGES); i < tiles; ++i) mbar_wait(&full_bar[i % STAGES], (i / STAGES) & 1, nullptr);
            for (int i = max(0, units - 2); i < units; ++i) mbar_wait(&unit_full[i & 1], (i >> 1) & 1, nullptr);
        }
    } else {
        // ---------------- compute ----------------
        cudaGridDependencySynchronize();                              // it writes where the kernel before may still read
        __syncthreads();
        const int quad = lane & 3, r8 = lane >> 2;                    // this thread's query rows: 2 quad, 2 quad + 1 (+ 8 nt)
        const int mi = lane >> 3, mr = lane & 7;
        const int k_row = warp * 16 + (mi & 1) * 8 + mr, k_chunk = mi >> 1;       // K as A: (keys 0-7 | 8-15) x (d 0-7), then d 8-15
        const int v_row = warp * 16 + (mi >> 1) * 8 + mr, v_chunk = mi & 1;       // V^T as A: (d 0-7 | 8-15) x (keys 0-7), then 8-15
        // where this lane's rows are in a tile of boxes, and how far apart a row's halves
        const int box = a.box_rows, half_pitch = box * 128;
        const uint32_t k_off = k_row / box * (box * D * 2) + k_row % box * 128, v_off = v_row / box * (box * D * 2) + v_row % box * 128;
        float* slot0 = reinterpret_cast<float*>(ring + L::SLOTS);
        float* slot1 = reinterpret_cast<float*>(ring + L::SLOTS + L::SLOT);
        int tiles = 0;
        for (int units = 0;; ++units) {
            const int ub = units & 1;
            if (!__all_sync(0xffffffffu, mbar_wait(&unit_full[ub], (units >> 1) & 1, abort_flag))) {
                give_up(DEV_TIMEOUT_TMA_FULL);
                break;
            }
            const UnitInfo info = infos[ub];
            if (info.rows == 0) break;
            uint32_t q[NT][D / 16][2];
            int qpos[NT][2];
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                const unsigned char* src = ring + L::Q + (ub * NT * 8 + n * 8 + r8) * L::Q_PITCH + quad * 4;
                const bool live = n * 8 + r8 < info.rows;
#pragma unroll
                for (int k = 0; k < D / 16; ++k) {
                    q[n][k][0] = live ? *reinterpret_cast<const uint32_t*>(src + k * 32) : 0u;
                    q[n][k][1] = live ? *reinterpret_cast<const uint32_t*>(src + k * 32 + 16) : 0u;
                }
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const int row = n * 8 + quad * 2 + i;
                    qpos[n][i] = row >= info.rows ? -1 : a.causal ? info.pos0 + token_of(row) : info.pos0;
                }
            }
            float o[NT][D / 16][4], m[NT][2], l[NT][2];
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                m[n][0] = m[n][1] = -INFINITY;
                l[n][0] = l[n][1] = 0.0f;
#pragma unroll
                for (int i = 0; i < D / 16; ++i)
#pragma unroll
                    for (int j = 0; j < 4; ++j) o[n][i][j] = 0.0f;
            }
            bool ok = true;
            for (int t = 0; t < info.n_tiles; ++t, ++tiles) {
                const int st = tiles % STAGES;
                ok = __all_sync(0xffffffffu, mbar_wait(&full_bar[st], (tiles / STAGES) & 1, abort_flag));
                if (!ok) break;
                const int pos = pos16[st][warp];
                if (pos >= 0) {
                    unsigned char* tile = ring + st * L::STAGE;
                    const uint32_t ks = smem_u32(tile), vs = ks + TILE * D * 2;
                    if (pos + 16 > info.kv) {
                        // values past the last position may hold anything: zero their rows
                        const int first = info.kv - pos;
                        for (int x = lane; x < (16 - first) * (D / 8); x += 32) {
                            const int rr = warp * 16 + first + x / (D / 8), c = x % (D / 8);
                            *reinterpret_cast<uint4*>(tile + TILE * D * 2 + rr / box * (box * D * 2) + (c >> 3) * half_pitch + rr % box * 128 +
                                                      (c & 7) * 16) = make_uint4(0, 0, 0, 0);
                        }
                        fence_async_smem();
                        __syncwarp();
                    }
                    float sc[NT][4];
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int j = 0; j < 4; ++j) sc[n][j] = 0.0f;
#pragma unroll
                    for (int k = 0; k < D / 16; ++k) {
                        uint32_t x[4];
                        const int c = k * 2 + k_chunk;
                        ldsm4(x, ks + k_off + (c >> 3) * half_pitch + (((c & 7) ^ (k_row & 7)) << 4));
#pragma unroll
                        for (int n = 0; n < NT; ++n) mma16816<T>(sc[n], x, q[n][k][0], q[n][k][1]);
                    }
                    const bool edge = pos + 15 > info.pos0 || (a.window > 0 && pos <= info.pos_last - a.window);
                    bool grow = false;
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const int i = j & 1, kp = pos + r8 + (j >> 1) * 8;
                            sc[n][j] *= a.scale_log2;
                            if (edge && (kp > qpos[n][i] || (a.window > 0 && kp <= qpos[n][i] - a.window))) sc[n][j] = -INFINITY;
                            grow |= sc[n][j] > m[n][i] + Range::grow;
                        }
                    if (__any_sync(0xffffffffu, grow)) {
#pragma unroll
                        for (int n = 0; n < NT; ++n) {
                            float f[2];
#pragma unroll
                            for (int i = 0; i < 2; ++i) {
                                float top = fmaxf(fmaxf(sc[n][i], sc[n][2 + i]) - Range::lift, m[n][i]);
                                top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 4));
                                top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 8));
                                top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 16));
                                f[i] = m[n][i] == -INFINITY ? 0.0f : ex2(m[n][i] - top);
                                m[n][i] = top;
                                l[n][i] *= f[i];
                            }
#pragma unroll
                            for (int k = 0; k < D / 16; ++k) {
                                o[n][k][0] *= f[0]; o[n][k][1] *= f[1];
                                o[n][k][2] *= f[0]; o[n][k][3] *= f[1];
                            }
                        }
                    }
                    uint32_t p[NT][2];
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            sc[n][j] = ex2(sc[n][j] - (m[n][j & 1] == -INFINITY ? 0.0f : m[n][j & 1]));
                            l[n][j & 1] += sc[n][j];
                        }
                        p[n][0] = transpose8(Half2Of<T>::pack(sc[n][0], sc[n][1]));
                        p[n][1] = transpose8(Half2Of<T>::pack(sc[n][2], sc[n][3]));
                    }
#pragma unroll
                    for (int k = 0; k < D / 16; ++k) {
                        uint32_t x[4];
                        const int c = k * 2 + v_chunk;
                        ldsm4_t(x, vs + v_off + (c >> 3) * half_pitch + (((c & 7) ^ (v_row & 7)) << 4));
#pragma unroll
                        for (int n = 0; n < NT; ++n) mma16816<T>(o[n][k], x, p[n][0], p[n][1]);
                    }
                }
                __syncwarp();
                if (lane == 0) mbar_arrive(&empty_bar[st]);
            }
            if (!ok) {
                give_up(DEV_TIMEOUT_TMA_FULL);
                break;
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(&unit_empty[ub]);              // its description and query rows have been read
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int x = 4; x < 32; x <<= 1) l[n][i] += __shfl_xor_sync(0xffffffffu, l[n][i], x);

            // ---- the four accumulators: 2 -> 0 and 3 -> 1, then 1 -> 0 ----
            // One copy of the code for both steps: it runs once per unit, and what a short call waits for here is instructions.
            auto wait = [&](uint64_t* bar, uint32_t parity) {
                ok = __all_sync(0xffffffffu, mbar_wait(bar, parity, abort_flag));
                if (!ok) give_up(DEV_TIMEOUT_ACC_FULL);
                return ok;
            };
            const uint32_t now = units & 1;                           // every barrier here completes once per unit
#pragma unroll 1
            for (int step = 0; step < 2 && ok; ++step) {
                const int x = step == 0 ? warp & 1 : 1;               // slot
                float* slot = x == 0 ? slot0 : slot1;
                auto at = [&](int n, int k, int j) -> float& {
                    return slot[(n * 8 + quad * 2 + (j & 1)) * L::PITCH + k * 16 + (j >> 1) * 8 + r8];
                };
                if (step == 0 ? warp >= 2 : warp == 1) {
                    if (step == 0 && units > 0 && !wait(x == 0 ? &free0 : &free1, now ^ 1)) break;
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
#pragma unroll
                        for (int k = 0; k < D / 16; ++k)
#pragma unroll
                            for (int j = 0; j < 4; ++j) at(n, k, j) = o[n][k][j];
                        if (r8 == 0)
#pragma unroll
                            for (int i = 0; i < 2; ++i) { red_m[x][n * 8 + quad * 2 + i] = m[n][i]; red_l[x][n * 8 + quad * 2 + i] = l[n][i]; }
                    }
                    __syncwarp();
                    if (lane == 0) mbar_arrive(step == 1 ? &from1 : x == 0 ? &from2 : &from3);
                } else if (step == 0 ? warp < 2 : warp == 0) {
                    if (!wait(step == 1 ? &from1 : x == 0 ? &from2 : &from3, now)) break;
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        float f[2], g[2];
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            const float m2 = red_m[x][n * 8 + quad * 2 + i], top = fmaxf(m[n][i], m2), ref = top == -INFINITY ? 0.0f : top;
                            f[i] = ex2(m[n][i] - ref);
                            g[i] = ex2(m2 - ref);
                            m[n][i] = top;
                            l[n][i] = l[n][i] * f[i] + red_l[x][n * 8 + quad * 2 + i] * g[i];
                        }
#pragma unroll
                        for (int k = 0; k < D / 16; ++k)
#pragma unroll
                            for (int j = 0; j < 4; ++j) o[n][k][j] = o[n][k][j] * f[j & 1] + at(n, k, j) * g[j & 1];
                    }
                    __syncwarp();
                    if (step == 1 && lane == 0) mbar_arrive(&free1);
                }
            }
            if (!ok) break;
            if (warp == 0) {
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const float inv = l[n][i] == 0.0f ? 0.0f : 1.0f / l[n][i];
                        const int row = n * 8 + quad * 2 + i;
                        if (r8 == 0 && row < info.rows) {
                            const float lse2 = l[n][i] == 0.0f ? -INFINITY : m[n][i] + log2f(l[n][i]);
                            if (info.slot >= 0) a.part_lse[info.slot * a.rows_cap + row] = lse2;
                            else if (a.lse) a.lse[static_cast<int64_t>(info.tok0 + token_of(row)) * a.n_heads + info.head * a.group + head_of(row)] = lse2 * kLn2;
                        }
#pragma unroll
                        for (int k = 0; k < D / 16; ++k)
#pragma unroll
                            for (int j = 0; j < 2; ++j)
                                slot0[row * L::PITCH + k * 16 + j * 8 + r8] = l[n][i] == 0.0f ? 0.0f : o[n][k][2 * j + i] * inv;
                    }
                __syncwarp();
                // whole rows, 32 / (D / 4) at a time
                constexpr int LANES = D / 4, STEP = 32 / LANES;
                const int c = lane % LANES * 4;
#pragma unroll 1
                for (int row = lane / LANES; row < info.rows; row += STEP) {
                    const float4 y = *reinterpret_cast<const float4*>(slot0 + row * L::PITCH + c);
                    if (info.slot >= 0) {
                        *reinterpret_cast<float4*>(a.part_o + (static_cast<int64_t>(info.slot) * a.rows_cap + row) * D + c) = y;
                    } else {
                        T* dst = static_cast<T*>(a.out) + static_cast<int64_t>(info.tok0 + token_of(row)) * a.ld_out +
                                 (info.head * a.group + head_of(row)) * D + c;
                        *reinterpret_cast<uint2*>(dst) = make_uint2(Half2Of<T>::pack(y.x, y.y), Half2Of<T>::pack(y.z, y.w));
                    }
                }
                __syncwarp();
                if (lane == 0) mbar_arrive(&free0);
            }
        }
    }
    __syncthreads();
}

// Joins the pieces of the units that the shares cut: out = sum_i 2^(lse_i - max) o_i / sum_i 2^(lse_i - max). Block x takes the unit
// that began in share x and was cut behind it, its rows divided over the y blocks. With a few rows and many pieces (one
// sequence over the whole grid) a block takes one row and its four warps every fourth piece; with many rows and two or
// three pieces each warp takes two rows. The launch overlaps the kernel before it (programmatic launch).
template <class T, int D, bool MANY_ROWS>
__global__ void __launch_bounds__(128) join_kernel(const __grid_constant__ AttnArgs a)
{
    __shared__ float acc[MANY_ROWS ? 1 : 4][D], acc_l[4];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    cudaTriggerProgrammaticLaunchCompletion();
    cudaGridDependencySynchronize();
    const Cut cut = reinterpret_cast<const Cut*>(a.cuts)[blockIdx.x];
    const int c0 = blockIdx.x, c1 = cut.last, rows = cut.n_tok * a.group;
    constexpr int N = D / 32;                    // consecutive values per lane
    constexpr int ROWS = MANY_ROWS ? 8 : 1;
    const int from = blockIdx.y * ROWS, to = min(rows, from + ROWS);
    for (int row = from + (MANY_ROWS ? warp : 0); row < to; row += MANY_ROWS ? 4 : 1) {
        auto slot = [&](int c) { return static_cast<int64_t>(2 * c + (c < c1 ? 1 : 0)) * a.rows_cap + row; };
        float top = -INFINITY;
        for (int c = c0 + lane; c <= c1; c += 32) top = fmaxf(top, a.part_lse[slot(c)]);
#pragma unroll
        for (int x = 16; x > 0; x >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, x));
        const float ref = top == -INFINITY ? 0.0f : top;
        float y[N], sum = 0.0f;
#pragma unroll
        for (int j = 0; j < N; ++j) y[j] = 0.0f;
#pragma unroll 4
        for (int c = c0 + (MANY_ROWS ? 0 : warp); c <= c1; c += MANY_ROWS ? 1 : 4) {
            const int64_t s = slot(c);
            const float f = ex2(a.part_lse[s] - ref);               // a piece that saw nothing holds zeros and -inf
            sum += f;
            const float* p = a.part_o + s * D + lane * N;
            if constexpr (N == 4) {
                const float4 z = *reinterpret_cast<const float4*>(p);
                y[0] += f * z.x; y[1] += f * z.y; y[2] += f * z.z; y[3] += f * z.w;
            } else {
                const float2 z = *reinterpret_cast<const float2*>(p);
                y[0] += f * z.x; y[1] += f * z.y;
            }
        }
        if constexpr (!MANY_ROWS) {
#pragma unroll
            for (int j = 0; j < N; ++j) acc[warp][lane * N + j] = y[j];
            if (lane == 0) acc_l[warp] = sum;
            __syncthreads();
            sum = (acc_l[0] + acc_l[1]) + (acc_l[2] + acc_l[3]);
#pragma unroll
            for (int j = 0; j < N; ++j) y[j] = (acc[0][lane * N + j] + acc[1][lane * N + j]) + (acc[2][lane * N + j] + acc[3][lane * N + j]);
            if (warp != 0) continue;
        }
        const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
        const int64_t tok = cut.tok0 + row / a.group, h = cut.head * a.group + row % a.group;
        T* dst = static_cast<T*>(a.out) + tok * a.ld_out + h * D + lane * N;
#pragma unroll
        for (int j = 0; j < N; j += 2) *reinterpret_cast<uint32_t*>(dst + j) = Half2Of<T>::pack(y[j] * inv, y[j + 1] * inv);
        if (lane == 0 && a.lse) a.lse[tok * a.n_heads + h] = sum == 0.0f ? -INFINITY : (top + log2f(sum)) * kLn2;
    }
}

template <class T, int D, int NT>
s3_status launch_split(const KvCacheState& c, const AttnArgs& a, cudaStream_t stream)
{
    using L = Layout<D, NT>;
    const s3_status allowed = allow_smem<split_kernel<T, D, NT>>(L::TOTAL);
    if (allowed != S3_OK) return allowed;
    Maps maps;
    memcpy(maps.k, c.wide_k, sizeof(maps.k));
    memcpy(maps.v, c.wide_v, sizeof(maps.v));
    return launch_overlapped(split_kernel<T, D, NT>, dim3(a.grid), THREADS, L::TOTAL, stream, maps, a);
}

template <class T, int D>
s3_status launch_rows(const KvCacheState& c, const AttnArgs& a, cudaStream_t stream)
{
    const int rows = (a.list_mode == LIST_PER_TOKEN ? 1 : a.b.max_q) * a.group;       // of the largest item
    // one group of 8 query rows or two (us, up to 8 rows): one token over 131072 keys 93 and 97, over 777 13.7 and 16.7; lists 328 and 466
    return rows <= 8 ? launch_split<T, D, 1>(c, a, stream) : launch_split<T, D, 2>(c, a, stream);
}

template <class T, int D>
s3_status launch_join_typed(const AttnArgs& a, bool tile, cudaStream_t stream)
{
    const int most = min(a.rows_cap, (a.list_mode == LIST_PER_TOKEN ? 1 : min(a.b.max_q, a.rows_cap)) * a.group);     // rows of an item
    const dim3 grid(static_cast<unsigned>(a.grid - 1), static_cast<unsigned>(tile ? (most + 7) / 8 : most));
    return tile ? launch_overlapped(join_kernel<T, D, true>, grid, 128, 0, stream, a) : launch_overlapped(join_kernel<T, D, false>, grid, 128, 0, stream, a);
}

}  // namespace

s3_status launch_attn_split(const KvCacheState& c, const AttnArgs& a, cudaStream_t stream)
{
    const bool wide = c.d.head_dim == 128;
    if (c.d.dtype == S3_BF16) return wide ? launch_rows<__nv_bfloat16, 128>(c, a, stream) : launch_rows<__nv_bfloat16, 64>(c, a, stream);
    return wide ? launch_rows<__half, 128>(c, a, stream) : launch_rows<__half, 64>(c, a, stream);
}

s3_status launch_attn_join(const KvCacheState& c, const AttnArgs& a, bool tile, cudaStream_t stream)
{
    const bool wide = c.d.head_dim == 128;
    if (c.d.dtype == S3_BF16) return wide ? launch_join_typed<__nv_bfloat16, 128>(a, tile, stream) : launch_join_typed<__nv_bfloat16, 64>(a, tile, stream);
    return wide ? launch_join_typed<__half, 128>(a, tile, stream) : launch_join_typed<__half, 64>(a, tile, stream);
}

}  // namespace s3
