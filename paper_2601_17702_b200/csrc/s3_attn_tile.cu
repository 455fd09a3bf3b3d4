// Attention of many query rows over a paged cache on the sm_100a tensor cores: chunks of a prompt, questions over listed blocks.
//
//   S = Q K^T (fp32, tensor memory);  P = 2^(scale log2e S - m);  O += P V;  out = O / sum P      one pass over the keys
//
// A thread block takes one (item, key head, split). The item's query rows (token, head of the group), packed, fill one or
// two tiles of 128; keys come in tiles of 128.
//   warp 0       TMA producer: Q once, then K and V tiles page by page into a ring of shared-memory slots (128-byte swizzle);
//   warp 1       MMA issuer: one thread issues tcgen05.mma for S = Q K^T (both operands in shared memory) and O += P V (P read
//                from tensor memory, V as the MN-major operand, so no transpose is ever made);
//   warp 2       zeroes the rows of a V tile that hold no position of the sequence (a page's tail may hold anything);
//   warps 4-7, 8-11   two softmax groups, a thread per row: S from tensor memory into registers, running maximum, exponentials,
//                P back over S in the cache's type.
// With two query tiles (PAIR) each group owns one and both use every key tile; with one query tile the groups take the even
// and the odd key tiles, with an accumulator each, and are joined at the end. Either way one group's exponentials run while
// the tensor core works for the other: the two sides need about the same time at head_dim 128.
// O stays in tensor memory. It is rescaled only when a row's maximum grows by more than 2^8 over the reference its
// exponentials use (P then stays below 2^8, well inside either type, and the sum in fp32); the MMA order makes S(j+1) complete
// only after O += P(j) V(j), so the group may touch O as soon as it sees the next S.
//
// Every mbarrier wait is bounded; one that runs out sets the status word and the block's abort flag, and the block waits for its
// copies and frees its tensor memory before it leaves.
#include <string.h>

#include "s3_kernels.cuh"
#include "s3_kv.cuh"

namespace s3 {
namespace {

using namespace kv;

constexpr int BM = 128, BN = 128;                  // query rows and keys per tile
constexpr int THREADS = 384;
constexpr int TMEM_COLS = 512;
constexpr float RESCALE_AT = 8.0f;

struct Maps {
    alignas(64) unsigned char q[128], k[128], v[128];
};

template <int D, bool PAIR>
struct Layout {
    static constexpr int TILE_BYTES = BN * D * 2;
    static constexpr int Q_TILES = PAIR ? 2 : 1;
    static constexpr int Q_BYTES = Q_TILES * BM * D * 2;
    static constexpr int SLOTS = D == 128 ? 5 : 8;
    static constexpr int RING = Q_BYTES;
    static constexpr int LIST = RING + SLOTS * TILE_BYTES;
    static constexpr int BARS = LIST + S3_MAX_BLOCK_LIST * 4;
    static constexpr int TOTAL = BARS + 256;
    static_assert(TOTAL <= 227 * 1024, "one thread block per SM");
};

__device__ __forceinline__ uint64_t desc_base(uint32_t saddr, uint32_t lbo, uint32_t sbo)
{
    uint64_t d = 0;
    d |= static_cast<uint64_t>((saddr >> 4) & 0x3FFFu);
    d |= static_cast<uint64_t>(lbo >> 4) << 16;
    d |= static_cast<uint64_t>(sbo >> 4) << 32;
    d |= static_cast<uint64_t>(1) << 46;                 // descriptor version of this architecture
    d |= static_cast<uint64_t>(2) << 61;                 // 128-byte swizzle
    return d;
}
__device__ __forceinline__ void mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool acc)
{
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
                 "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(acc ? 1u : 0u) : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, bool acc)
{
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
                 "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"(acc ? 1u : 0u) : "memory");
}
__device__ __forceinline__ void commit(uint64_t* bar)
{
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
}
__device__ __forceinline__ void wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tm_ld32(uint32_t taddr, float (&u)[32])
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=f"(u[0]), "=f"(u[1]), "=f"(u[2]), "=f"(u[3]), "=f"(u[4]), "=f"(u[5]), "=f"(u[6]), "=f"(u[7]), "=f"(u[8]),
          "=f"(u[9]), "=f"(u[10]), "=f"(u[11]), "=f"(u[12]), "=f"(u[13]), "=f"(u[14]), "=f"(u[15]), "=f"(u[16]),
          "=f"(u[17]), "=f"(u[18]), "=f"(u[19]), "=f"(u[20]), "=f"(u[21]), "=f"(u[22]), "=f"(u[23]), "=f"(u[24]),
          "=f"(u[25]), "=f"(u[26]), "=f"(u[27]), "=f"(u[28]), "=f"(u[29]), "=f"(u[30]), "=f"(u[31])
        : "r"(taddr) : "memory");
}
__device__ __forceinline__ void tm_st32(uint32_t taddr, const uint32_t (&u)[32])
{
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
        "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, "
        "%17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};" ::"r"(taddr),
        "r"(u[0]), "r"(u[1]), "r"(u[2]), "r"(u[3]), "r"(u[4]), "r"(u[5]), "r"(u[6]), "r"(u[7]), "r"(u[8]),
        "r"(u[9]), "r"(u[10]), "r"(u[11]), "r"(u[12]), "r"(u[13]), "r"(u[14]), "r"(u[15]), "r"(u[16]),
        "r"(u[17]), "r"(u[18]), "r"(u[19]), "r"(u[20]), "r"(u[21]), "r"(u[22]), "r"(u[23]), "r"(u[24]),
        "r"(u[25]), "r"(u[26]), "r"(u[27]), "r"(u[28]), "r"(u[29]), "r"(u[30]), "r"(u[31]) : "memory");
}

__device__ __forceinline__ void tm_st32(uint32_t taddr, const float (&f)[32])
{
    uint32_t u[32];
#pragma unroll
    for (int i = 0; i < 32; ++i) u[i] = __float_as_uint(f[i]);
    tm_st32(taddr, u);
}

template <class T, int D, bool PAIR>
__global__ void __launch_bounds__(THREADS, 1) tile_kernel(const __grid_constant__ Maps maps, const __grid_constant__ AttnArgs a)
{
    using L = Layout<D, PAIR>;
    constexpr int SLOTS = L::SLOTS, AHEAD = PAIR ? 1 : 2;       // key tiles whose S is issued before the first P V
    extern __shared__ __align__(1024) unsigned char smem[];            // swizzled tiles start on 1024-byte boundaries
    unsigned char* ring = smem + L::RING;
    int* list = reinterpret_cast<int*>(smem + L::LIST);
    uint64_t* full_bar = reinterpret_cast<uint64_t*>(smem + L::BARS);
    uint64_t* empty_bar = full_bar + SLOTS;
    uint64_t* s_full = empty_bar + SLOTS;
    uint64_t* p_full = s_full + 2;
    uint64_t& q_full = p_full[2];
    uint64_t& o_full = p_full[3];
    uint64_t& dirty_bar = p_full[4];
    uint64_t& clean_bar = p_full[5];
    uint64_t& meet_bar = p_full[6];
    uint32_t& tmem_slot = *reinterpret_cast<uint32_t*>(p_full + 7);
    volatile uint32_t* abort_flag = &tmem_slot + 1;

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int split = blockIdx.x % a.n_splits, head = (blockIdx.x / a.n_splits) % a.n_kv_heads;
    const int item = blockIdx.x / a.n_splits / a.n_kv_heads;
    AttnItem it;
    if (!attn_item(a, item, it)) return;
    const int tile_tok = min(BM / a.group, a.tok_per_item);            // tokens per 128-row tile
    const int pos_last = a.causal ? it.pos0 + it.n_tok - 1 : it.pos0;
    const int seen_lo = a.window > 0 ? max(it.pos0 - a.window + 1, 0) : 0;
    int v_lo = 0, v_hi = 0;
    if (a.list_mode == LIST_NONE) {
        v_lo = (seen_lo & ~(BN - 1)) + split * a.split_len;
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
    const int n_tiles = max(0, (v_hi - v_lo + BN - 1) / BN);

    if (threadIdx.x == 0) {
        mbar_init(&q_full, 1);
        for (int i = 0; i < SLOTS; ++i) { mbar_init(&full_bar[i], 1); mbar_init(&empty_bar[i], 1); }
        for (int i = 0; i < 2; ++i) { mbar_init(&s_full[i], 1); mbar_init(&p_full[i], 128); }
        mbar_init(&o_full, 1);
        mbar_init(&dirty_bar, 1);
        mbar_init(&clean_bar, 1);
        mbar_init(&meet_bar, 128);
        *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_slot)), "r"(TMEM_COLS) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_slot;
    auto tm_s = [&](int i) { return tmem + 128 * i; };                 // scores, then weights, of group i
    auto tm_o = [&](int i) { return tmem + 256 + 128 * i; };           // its accumulator

    // First position of virtual key v (a multiple of 16), or -1 where no block is listed.
    auto pos_of = [&](int v) -> int {
        if (a.list_mode == LIST_NONE) return v;
        const int e = v >> a.page_shift;
        if (e >= a.s || list[e] < 0) return -1;
        return (list[e] << a.page_shift) + (v & (a.page_size - 1));
    };
    // Whether a key tile has rows without a position of the sequence: their values have to be zeroed.
    auto unclean = [&](int j) -> bool {
        const int v0 = v_lo + j * BN;
        if (a.list_mode == LIST_NONE) return v0 + BN > it.kv;
        bool bad = false;
        for (int u = 0; u < BN; u += 16) {
            const int pos = pos_of(v0 + u);
            bad |= pos < 0 || pos + 16 > it.kv;
        }
        return bad;
    };

    // The launch gives every thread 168 registers; the four role warps hand theirs to the softmax rows (128 x 56 + 256 x 224 =
    // 384 x 168).
    int issued = 0;                                                    // ring loads started
    if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
    if (warp == 0) {
        // ---------------- producer ----------------
        if (lane == 0 && n_tiles > 0) {
            mbar_expect_tx(&q_full, L::Q_TILES * static_cast<uint32_t>(tile_tok * a.group) * D * 2);
            for (int i = 0; i < L::Q_TILES; ++i)
                for (int h = 0; h < D / 64; ++h)
                    tma_load_4d(smem + i * BM * D * 2 + h * BM * 128, maps.q, h * 64, 0, head, it.tok0 + i * tile_tok, &q_full);
            const int32_t* table = a.b.pages + it.seq * a.b.ld_pages;
            const int box = a.box_rows;
            auto load = [&](int j, bool value) -> bool {
                const int st = issued % SLOTS, round = issued / SLOTS;
                if (round > 0 && !mbar_wait(&empty_bar[st], (round - 1) & 1, abort_flag)) {
                    dev_set_error(a.status, DEV_TIMEOUT_SMEM_EMPTY);
                    *abort_flag = 1;
                    return false;
                }
                const void* map = value ? maps.v : maps.k;
                unsigned char* dst = ring + st * L::TILE_BYTES;
                // the count may run ahead of the copies: the barrier completes only with the arrival at the end
                for (int u = 0; u < BN; u += box) {
                    const int pos = pos_of(v_lo + j * BN + u);
                    if (pos < 0 || pos >= it.kv) continue;
                    int p = table[pos >> a.page_shift];
                    if (p < 0 || p >= a.n_pages) {
                        dev_set_error(a.status, DEV_BAD_PAGE);
                        p = a.n_pages;                                 // beyond the map: reads as zeros
                    }
                    asm volatile("mbarrier.expect_tx.relaxed.cta.shared::cta.b64 [%0], %1;" ::"r"(smem_u32(&full_bar[st])),
                                 "r"(static_cast<uint32_t>(box) * D * 2) : "memory");
#pragma unroll
                    for (int h = 0; h < D / 64; ++h)
                        tma_load_4d(dst + h * BN * 128 + u * 128, map, h * 64, pos & (a.page_size - 1), head, p, &full_bar[st]);
                }
                mbar_arrive(&full_bar[st]);
                ++issued;
                return true;
            };
            bool ok = true;
            for (int j = 0; j < min(AHEAD, n_tiles) && ok; ++j) ok = load(j, false);
            for (int j = 0; j < n_tiles && ok; ++j) {
                ok = load(j, true);
                if (ok && j + AHEAD < n_tiles) ok = load(j + AHEAD, false);
            }
        }
    } else if (warp == 1) {
        // ---------------- MMA issuer ----------------
        if (lane == 0 && n_tiles > 0) {
            constexpr uint32_t fmt = sizeof(T) == 2 && Half2Of<T>::is_bf16 ? 1u : 0u;
            constexpr uint32_t base = (1u << 4) | (fmt << 7) | (fmt << 10) | (static_cast<uint32_t>(BM >> 4) << 24);
            constexpr uint32_t idesc_s = base | (static_cast<uint32_t>(BN >> 3) << 17);
            constexpr uint32_t idesc_o = base | (1u << 16) | (static_cast<uint32_t>(D >> 3) << 17);     // V: MN-major
            const uint32_t q_addr = smem_u32(smem), r_addr = smem_u32(ring);
            uint32_t used = 0, cleaned = 0;
            bool ok = true;
            auto need = [&](uint64_t* bar, uint32_t parity, uint32_t code) {
                if (ok && !mbar_wait(bar, parity, abort_flag)) {
                    dev_set_error(a.status, code);
                    *abort_flag = 1;
                    ok = false;
                }
                return ok;
            };
            auto slot_ready = [&]() { return need(&full_bar[used % SLOTS], (used / SLOTS) & 1, DEV_TIMEOUT_TMA_FULL); };
            auto scores = [&](int i, int qt, uint32_t st) {
                tc_fence_after();
#pragma unroll
                for (int k = 0; k < D / 16; ++k) {
                    const uint32_t off = (k >> 2) * (BM * 128) + (k & 3) * 32;
                    mma_ss(tm_s(i), desc_base(q_addr + qt * BM * D * 2 + off, 16, 1024), desc_base(r_addr + st * L::TILE_BYTES + off, 16, 1024),
                           idesc_s, k > 0);
                }
                commit(&s_full[i]);
            };
            auto product = [&](int i, uint32_t st, bool acc) {
                tc_fence_after();
#pragma unroll
                for (int k = 0; k < BN / 16; ++k)
                    mma_ts(tm_o(i), tm_s(i) + k * 8, desc_base(r_addr + st * L::TILE_BYTES + k * 2048, BN * 128, 1024), idesc_o, acc || k > 0);
            };
            need(&q_full, 0, DEV_TIMEOUT_TMA_FULL);
            for (int j = 0; j < min(AHEAD, n_tiles) && ok; ++j) {
                if (!slot_ready()) break;
                const uint32_t st = used % SLOTS;
                if (PAIR) { scores(0, 0, st); scores(1, 1, st); }
                else scores(j & 1, 0, st);
                commit(&empty_bar[st]);
                ++used;
            }
            for (int j = 0; j < n_tiles && ok; ++j) {
                if (!slot_ready()) break;
                const uint32_t sv = used % SLOTS;
                ++used;
                if (unclean(j)) {
                    mbar_arrive(&dirty_bar);
                    if (!need(&clean_bar, cleaned++ & 1, DEV_TIMEOUT_ACC_EMPTY)) break;
                }
                const bool more = j + AHEAD < n_tiles;
                const uint32_t sk = used % SLOTS;
                if (PAIR) {
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        if (!need(&p_full[i], j & 1, DEV_TIMEOUT_ACC_EMPTY)) break;
                        product(i, sv, j > 0);
                        if (i == 1) commit(&empty_bar[sv]);
                        if (more) {
                            if (i == 0 && !slot_ready()) break;
                            scores(i, i, sk);
                        }
                    }
                    if (more && ok) { commit(&empty_bar[sk]); ++used; }
                } else {
                    const int i = j & 1;
                    if (!need(&p_full[i], (j >> 1) & 1, DEV_TIMEOUT_ACC_EMPTY)) break;
                    product(i, sv, j > 1);
                    commit(&empty_bar[sv]);
                    if (more) {
                        if (!slot_ready()) break;
                        scores(i, 0, sk);
                        commit(&empty_bar[sk]);
                        ++used;
                    }
                }
            }
            if (ok) commit(&o_full);
        }
    } else if (warp == 2) {
        // ---------------- values past the sequence ----------------
        // The MMA thread hands the tile over once it has landed. V tile j is ring load number 2j + AHEAD while key tiles still
        // come (K_{j+AHEAD} follows V_j).
        uint32_t at = min(AHEAD, n_tiles), handed = 0;
        bool ok = true;
        for (int j = 0; j < n_tiles && ok; ++j) {
            if (unclean(j)) {
                const uint32_t st = at % SLOTS;
                ok = __all_sync(0xffffffffu, mbar_wait(&dirty_bar, handed++ & 1, abort_flag));
                if (!ok) break;                                        // the MMA thread has reported why
                for (int u = 0; u < BN; u += 16) {
                    const int pos = pos_of(v_lo + j * BN + u);
                    const int live = pos < 0 ? 0 : min(max(it.kv - pos, 0), 16);
                    for (int x = lane; x < (16 - live) * (D / 8); x += 32) {
                        const int row = u + live + x / (D / 8), c = x % (D / 8);
                        *reinterpret_cast<uint4*>(ring + st * L::TILE_BYTES + (c >> 3) * BN * 128 + row * 128 + (c & 7) * 16) = make_uint4(0, 0, 0, 0);
                    }
                }
                fence_async_smem();
                __syncwarp();
                if (lane == 0) mbar_arrive(&clean_bar);
            }
            at += j + AHEAD < n_tiles ? 2 : 1;
        }
    }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 224;");
        // ---------------- softmax ----------------
        const int i = (warp - 4) >> 2;                                 // group
        const int row = (warp & 3) * 32 + lane;                        // row of the tile = lane of tensor memory
        const uint32_t lane_base = static_cast<uint32_t>((warp & 3) * 32) << 16;
        const uint32_t my_s = tm_s(i) + lane_base, my_o = tm_o(i) + lane_base;
        const int first_tok = PAIR ? i * tile_tok : 0;                 // first token of the tile, relative to the item
        const int tok = first_tok + row / a.group, g = row % a.group;
        const bool live = row < tile_tok * a.group && tok < it.n_tok;
        const int qpos = a.causal ? it.pos0 + tok : it.pos0;
        const int qlo = a.causal ? it.pos0 + first_tok : it.pos0;      // smallest and largest position of the tile's rows
        const int qhi = a.causal ? min(qlo + tile_tok - 1, pos_last) : qlo;
        float m = -INFINITY, l = 0.0f;                                 // reference of the exponentials (scaled, base 2), sum
        bool ok = true;
        int turns = 0;
        for (int j = PAIR ? 0 : i; j < n_tiles; j += PAIR ? 1 : 2, ++turns) {
            ok = __all_sync(0xffffffffu, mbar_wait(&s_full[i], turns & 1, abort_flag));
            if (!ok) {
                if (lane == 0) { dev_set_error(a.status, DEV_TIMEOUT_ACC_FULL); *abort_flag = 1; }
                break;
            }
            tc_fence_after();
            float s[4][32];
#pragma unroll
            for (int c = 0; c < 4; ++c) tm_ld32(my_s + 32 * c, s[c]);
            wait_ld();
            const int v0 = v_lo + j * BN;
            bool edge;
            if (a.list_mode == LIST_NONE) edge = v0 + BN - 1 > qlo || (a.window > 0 && v0 <= qhi - a.window);
            else {
                edge = false;
                for (int u = 0; u < BN; u += 16) {
                    const int pos = pos_of(v0 + u);
                    edge |= pos < 0 || pos + 15 > qlo || (a.window > 0 && pos <= qhi - a.window);
                }
            }
            if (edge) {
#pragma unroll
                for (int u = 0; u < BN; u += 16) {
                    const int pos = pos_of(v0 + u);
                    const int hi = pos < 0 ? -1 : qpos - pos, lo = a.window > 0 ? hi - a.window : -1;      // visible: lo < c <= hi
#pragma unroll
                    for (int c = 0; c < 16; ++c)
                        if (c > hi || c <= lo) s[u / 32][u % 32 + c] = -INFINITY;
                }
            }
            float mx[4] = {s[0][0], s[1][0], s[2][0], s[3][0]};
#pragma unroll
            for (int c = 1; c < 32; ++c)
#pragma unroll
                for (int x = 0; x < 4; ++x) mx[x] = fmaxf(mx[x], s[x][c]);
            const float top = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) * a.scale_log2;
            const bool grow = live && top > m + RESCALE_AT;
            if (__any_sync(0xffffffffu, grow)) {
                const float now = live ? fmaxf(m, top) : m;
                const float f = m == -INFINITY ? 0.0f : ex2(m - now);
                m = now;
                l *= f;
                if (turns > 0) {
#pragma unroll
                    for (int c = 0; c < D; c += 32) {
                        float o[32];
                        tm_ld32(my_o + c, o);
                        wait_ld();
#pragma unroll
                        for (int x = 0; x < 32; ++x) o[x] *= f;
                        tm_st32(my_o + c, o);
                    }
                }
            }
            const float ref = m == -INFINITY ? 0.0f : m;
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                uint32_t p[32];
#pragma unroll
                for (int c = 0; c < 32; ++c) {
                    float &x = s[2 * half + c / 16][(2 * c) % 32], &y = s[2 * half + c / 16][(2 * c) % 32 + 1];
                    x = ex2(fmaf(x, a.scale_log2, -ref));
                    y = ex2(fmaf(y, a.scale_log2, -ref));
                    p[c] = Half2Of<T>::pack(x, y);
                }
                tm_st32(my_s + 32 * half, p);
            }
            wait_st();
            tc_fence_before();
            mbar_arrive(&p_full[i]);
            float sum[4] = {0, 0, 0, 0};
#pragma unroll
            for (int c = 0; c < 32; ++c)
#pragma unroll
                for (int x = 0; x < 4; ++x) sum[x] += s[x][c];
            l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
        }
        // ---------------- results ----------------
        if (ok && n_tiles > 0) {
            ok = __all_sync(0xffffffffu, mbar_wait(&o_full, 0, abort_flag));
            if (!ok && lane == 0) { dev_set_error(a.status, DEV_TIMEOUT_ACC_FULL); *abort_flag = 1; }
        }
        tc_fence_after();
        float f_own = 1.0f;
        float* meet = reinterpret_cast<float*>(ring);                  // [2][128] then [128][D + 4]: the odd tiles' share
        constexpr int PITCH = D + 4;
        if (!PAIR && ok) {
            // every copy has landed and every MMA has read its operands: the ring is free
            if (i == 1) {
                meet[row] = m;
                meet[128 + row] = l;
                if (turns > 0) {
#pragma unroll
                    for (int c = 0; c < D; c += 32) {
                        float o[32];
                        tm_ld32(my_o + c, o);
                        wait_ld();
#pragma unroll
                        for (int x = 0; x < 32; x += 4)
                            *reinterpret_cast<float4*>(meet + 256 + row * PITCH + c + x) = make_float4(o[x], o[x + 1], o[x + 2], o[x + 3]);
                    }
                }
            }
            if (i == 1) mbar_arrive(&meet_bar);
            else {
                ok = __all_sync(0xffffffffu, mbar_wait(&meet_bar, 0, abort_flag));
                if (!ok && lane == 0) { dev_set_error(a.status, DEV_TIMEOUT_ACC_FULL); *abort_flag = 1; }
            }
        }
        if (ok && (PAIR || i == 0)) {
            float f_other = 0.0f;
            if (!PAIR) {
                const float m1 = meet[row], l1 = meet[128 + row], both = fmaxf(m, m1), ref = both == -INFINITY ? 0.0f : both;
                f_own = ex2(m - ref);
                f_other = ex2(m1 - ref);
                l = l * f_own + l1 * f_other;
                m = both;
            }
            const float inv = l == 0.0f ? 0.0f : 1.0f / l;
            const int t = it.tok0 + tok, h = head * a.group + g;
            const int64_t out_row = static_cast<int64_t>(t) * a.n_heads + h;
            const int64_t part = static_cast<int64_t>(split) * a.b.T * a.n_heads + out_row;
            const float lse2 = l == 0.0f ? -INFINITY : m + log2f(l);
            if (live) {
                if (a.n_splits > 1) a.part_lse[part] = lse2;
                else if (a.lse) a.lse[out_row] = lse2 / kLog2e;
            }
#pragma unroll
            for (int c = 0; c < D; c += 32) {
                float o[32];
                if (turns > 0) {
                    tm_ld32(my_o + c, o);
                    wait_ld();
                }
                const bool other = !PAIR && n_tiles > 1;
#pragma unroll
                for (int x = 0; x < 32; x += 4) {
                    float4 z = make_float4(0, 0, 0, 0);
                    if (other) z = *reinterpret_cast<const float4*>(meet + 256 + row * PITCH + c + x);
                    o[x] = turns == 0 || l == 0.0f ? 0.0f : (o[x] * f_own + z.x * f_other) * inv;
                    o[x + 1] = turns == 0 || l == 0.0f ? 0.0f : (o[x + 1] * f_own + z.y * f_other) * inv;
                    o[x + 2] = turns == 0 || l == 0.0f ? 0.0f : (o[x + 2] * f_own + z.z * f_other) * inv;
                    o[x + 3] = turns == 0 || l == 0.0f ? 0.0f : (o[x + 3] * f_own + z.w * f_other) * inv;
                }
                if (!live) continue;
                if (a.n_splits > 1) {
                    if (l != 0.0f)
#pragma unroll
                        for (int x = 0; x < 32; x += 4)
                            *reinterpret_cast<float4*>(a.part_o + part * D + c + x) = make_float4(o[x], o[x + 1], o[x + 2], o[x + 3]);
                } else {
                    T* dst = static_cast<T*>(a.out) + static_cast<int64_t>(t) * a.ld_out + h * D + c;
#pragma unroll
                    for (int x = 0; x < 32; x += 8)
                        *reinterpret_cast<uint4*>(dst + x) = make_uint4(Half2Of<T>::pack(o[x], o[x + 1]), Half2Of<T>::pack(o[x + 2], o[x + 3]),
                                                                        Half2Of<T>::pack(o[x + 4], o[x + 5]), Half2Of<T>::pack(o[x + 6], o[x + 7]));
                }
            }
        }
        tc_fence_before();
    }
    __syncthreads();
    if (*abort_flag && threadIdx.x == 0) {                             // no copy may be in flight when the block leaves
        if (n_tiles > 0) mbar_wait(&q_full, 0, nullptr);
        for (int x = max(0, issued - SLOTS); x < issued; ++x) mbar_wait(&full_bar[x % SLOTS], (x / SLOTS) & 1, nullptr);
    }
    __syncthreads();
    if (warp == 1) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(TMEM_COLS) : "memory");
    }
}

template <class T, int D, bool PAIR>
s3_status launch_tile(const KvCacheState& c, const AttnArgs& a, cudaStream_t stream)
{
    using L = Layout<D, PAIR>;
    static bool raised[64] = {};                 // the attribute is kept per device; setting it twice does no harm
    int dev = 0;
    S3_CUDA_TRY(cudaGetDevice(&dev));
    if (dev >= 64 || !raised[dev]) {
        S3_CUDA_TRY(cudaFuncSetAttribute(tile_kernel<T, D, PAIR>, cudaFuncAttributeMaxDynamicSharedMemorySize, L::TOTAL));
        if (dev < 64) raised[dev] = true;
    }
    Maps maps;
    memcpy(maps.k, c.map_k, sizeof(maps.k));
    memcpy(maps.v, c.map_v, sizeof(maps.v));
    const int tile_tok = BM / a.group < a.tok_per_item ? BM / a.group : a.tok_per_item;
    s3_status st = make_kv_query_map(maps.q, c, a.q, a.ldq, a.b.T, a.group, tile_tok);
    if (st != S3_OK) return st;
    const int64_t blocks = static_cast<int64_t>(a.n_items) * a.n_kv_heads * a.n_splits;
    S3_REQUIRE(blocks < (int64_t(1) << 31), S3_ERR_UNSUPPORTED, "the batch needs too many thread blocks");
    tile_kernel<T, D, PAIR><<<static_cast<unsigned>(blocks), THREADS, L::TOTAL, stream>>>(maps, a);
    S3_CUDA_TRY(cudaGetLastError());
    return S3_OK;
}

template <class T, int D>
s3_status launch_dim(const KvCacheState& c, const AttnArgs& a, cudaStream_t stream)
{
    return a.tok_per_item > BM / a.group ? launch_tile<T, D, true>(c, a, stream) : launch_tile<T, D, false>(c, a, stream);
}

}  // namespace

s3_status launch_attn_tile(const KvCacheState& c, const AttnArgs& a, cudaStream_t stream)
{
    const bool wide = c.d.head_dim == 128;
    if (c.d.dtype == S3_BF16) return wide ? launch_dim<__nv_bfloat16, 128>(c, a, stream) : launch_dim<__nv_bfloat16, 64>(c, a, stream);
    return wide ? launch_dim<__half, 128>(c, a, stream) : launch_dim<__half, 64>(c, a, stream);
}

}  // namespace s3
