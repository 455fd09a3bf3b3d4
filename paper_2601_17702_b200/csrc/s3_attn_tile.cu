// Attention of many query rows over a paged cache on the sm_100a tensor cores: chunks of a prompt, questions over listed blocks.
//
//   S = Q K^T (fp32, tensor memory);  P = 2^(scale log2e S - m);  O += P V;  out = O / sum P      one pass over the keys
//
// A persistent thread block per SM walks its segments (a unit of one item and one key head, or a piece of it). The item's query
// rows (token, head of the group), packed, fill one or two tiles of 128; keys come in tiles of 128.
//   warp 0       TMA producer: finds the segments, copies Q, then K and V tiles page by page into a ring of shared-memory slots
//                (128-byte swizzle), running ahead into the next segment;
//   warp 1       MMA issuer: one elected lane issues tcgen05.mma for S = Q K^T (both operands in shared memory) and O += P V (P read
//                from tensor memory, V as the MN-major operand, so no transpose is ever made), after the warp has zeroed the rows of V
//                that hold no position of the sequence;
//   warps 4-7, 8-11   two softmax groups, a thread per row: S from tensor memory into registers, running maximum, exponentials,
//                P back over S in the cache's type.
// With two query tiles (PAIR) each group owns one and both use every key tile; with one query tile the groups take the even
// and the odd key tiles, with an accumulator each, and are joined at the end. Either way one group's exponentials run while
// the tensor core works for the other: the two sides need about the same time at head_dim 128.
// O stays in tensor memory. It is rescaled only when a row's maximum has grown far over the reference its exponentials use (P
// stays inside the type, see WeightRange, and the sum in fp32); the MMA order makes S(j+1) complete
// only after O += P(j) V(j), so the group may touch O as soon as it sees the next S.
//
// Measured: 2048 tokens of 4 x 8 heads at the end of 32768 keys in 840 us from rest (1.27 PFLOP/s; 1.63 is what a large library product
// reaches here) and 940 to 985 us back to back, when the power limit holds the clock down (1.08 to 1.13; the product 1.38 then), with
// the tensor pipe busy 62 % and that of the exponentials 65 % of the time; 7 ragged chunks of up to 733 tokens at head_dim 64
// 72 us, where the units' starts and ends show.
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

struct Maps {
    alignas(64) unsigned char q[128], k[128], v[128];
};

// What the producer tells the other roles about a segment.
struct SegInfo {
    AttnItem it;
    int head, t_lo, n_tiles, v_base, slot;         // n_tiles 0: no more segments
};

// First position of each 16 keys of a tile, -1 where no block is listed; whether some of its rows hold no position of the sequence.
// Written with the copy of the tile's keys into entry (tile mod 8): by the time an entry is written again, the tile eight before
// has been consumed, since fewer than eight tiles fit the ring.
struct TileWhere {
    int pos[BN / 16];
    int unclean, unused[7];
};

template <int D, bool PAIR>
struct Layout {
    static constexpr int TILE_BYTES = BN * D * 2;
    static constexpr int Q_TILES = PAIR ? 2 : 1;
    static constexpr int Q_BYTES = Q_TILES * BM * D * 2;
    static constexpr int SLOTS = (D == 128 ? 7 : 10) - Q_TILES;
    static constexpr int RING = Q_BYTES;
    static constexpr int MEET = RING + SLOTS * TILE_BYTES;             // [2][128] floats: reference and sum of the odd tiles' group
    static constexpr int WHERE = MEET + 1024;                          // positions of the key tiles in flight, for lists
    static constexpr int BARS = WHERE + 8 * static_cast<int>(sizeof(TileWhere));
    static constexpr int TOTAL = BARS + 512;
    static_assert(TOTAL <= 227 * 1024, "one thread block per SM");
};

// Shared-memory matrix descriptor, 128-byte swizzle: the low word holds the address and the leading offset, the high word the
// stride between 8-row groups, the architecture's descriptor version and the swizzle.
constexpr uint32_t kDescHi = (1024u >> 4) | (1u << 14) | (2u << 29);
__device__ __forceinline__ uint32_t desc_lo(uint32_t saddr, uint32_t lbo) { return ((saddr >> 4) & 0x3FFFu) | ((lbo >> 4) << 16); }

// The MMA warp issues as a whole, one elected lane doing the work: its addresses then are warp-uniform values, and an
// instruction costs a few cycles to issue. (Behind `if (lane == 0)` each cost about 90, more than the 64 that a 128 x 128 x 16
// product takes, and the two products of a tile needed 3900 cycles where 2048 will do.)
__device__ __forceinline__ uint32_t elect_one()
{
    uint32_t p;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(p));
    return p;
}
__device__ __forceinline__ void mma_ss(uint32_t one, uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, bool acc)
{
    asm volatile("{\n\t.reg .pred p, e;\n\t.reg .b64 da, db;\n\tsetp.ne.b32 p, %4, 0;\n\tsetp.ne.b32 e, %6, 0;\n\t"
                 "mov.b64 da, {%1, %5};\n\tmov.b64 db, {%2, %5};\n\t"
                 "@e tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %3, p;\n\t}" ::"r"(d), "r"(a), "r"(b), "r"(idesc), "r"(acc ? 1u : 0u),
                 "r"(kDescHi), "r"(one) : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t one, uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, bool acc)
{
    asm volatile("{\n\t.reg .pred p, e;\n\t.reg .b64 db;\n\tsetp.ne.b32 p, %4, 0;\n\tsetp.ne.b32 e, %6, 0;\n\t"
                 "mov.b64 db, {%2, %5};\n\t"
                 "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], db, %3, p;\n\t}" ::"r"(d), "r"(a), "r"(b), "r"(idesc), "r"(acc ? 1u : 0u),
                 "r"(kDescHi), "r"(one) : "memory");
}
__device__ __forceinline__ void commit(uint32_t one, uint64_t* bar)
{
    asm volatile("{\n\t.reg .pred e;\n\tsetp.ne.b32 e, %1, 0;\n\t"
                 "@e tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}" ::"r"(smem_u32(bar)), "r"(one) : "memory");
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

__device__ __forceinline__ void tm_ld16(uint32_t taddr, float (&u)[16])
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
                 : "=f"(u[0]), "=f"(u[1]), "=f"(u[2]), "=f"(u[3]), "=f"(u[4]), "=f"(u[5]), "=f"(u[6]), "=f"(u[7]),
                   "=f"(u[8]), "=f"(u[9]), "=f"(u[10]), "=f"(u[11]), "=f"(u[12]), "=f"(u[13]), "=f"(u[14]), "=f"(u[15])
                 : "r"(taddr) : "memory");
}
__device__ __forceinline__ void tm_st16(uint32_t taddr, const float (&u)[16])
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(taddr),
                 "f"(u[0]), "f"(u[1]), "f"(u[2]), "f"(u[3]), "f"(u[4]), "f"(u[5]), "f"(u[6]), "f"(u[7]),
                 "f"(u[8]), "f"(u[9]), "f"(u[10]), "f"(u[11]), "f"(u[12]), "f"(u[13]), "f"(u[14]), "f"(u[15]) : "memory");
}

// ---- weights -------------------------------------------------------------------------------------
typedef unsigned long long f32x2;

__device__ __forceinline__ f32x2 pair_of(float a, float b)
{
    f32x2 r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ void split_pair(f32x2 v, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ f32x2 fma2(f32x2 a, f32x2 b, f32x2 c)
{
    f32x2 r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ f32x2 add2(f32x2 a, f32x2 b)
{
    f32x2 r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ float max3(float a, float b, float c)       // NaN if one is NaN
{
    float r;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
__device__ __forceinline__ float max_of(const float (&s)[32])
{
    float m[4];
#pragma unroll
    for (int x = 0; x < 4; ++x) {
        m[x] = max3(s[8 * x], s[8 * x + 1], s[8 * x + 2]);
        m[x] = max3(m[x], s[8 * x + 3], s[8 * x + 4]);
        m[x] = max3(m[x], s[8 * x + 5], s[8 * x + 6]);
        m[x] = max3(m[x], s[8 * x + 7], s[8 * x + 7]);
    }
    return max3(max3(m[0], m[1], m[2]), m[3], m[3]);
}
// Weights 2^(s scale + ref) of 32 scores, packed to the type; their sum is added to `sum`. ex2 runs at 16 per clock and SM: 128 x 128
// of them take the 1024 clocks that the tile's two products take. (Some of them by a polynomial on the multiply-add pipes
// was tried: with the reduction, clamping and exponent steps it costs 12 clocks a pair and warp against 16, and gains nothing.)
template <class T>
__device__ __forceinline__ void weights(const float (&s)[32], f32x2 scale, f32x2 ref, uint32_t* p, f32x2 (&sum)[2])
{
#pragma unroll
    for (int c = 0; c < 16; ++c) {
        float x, y;
        split_pair(fma2(pair_of(s[2 * c], s[2 * c + 1]), scale, ref), x, y);
        x = ex2(x);
        y = ex2(y);
        sum[c & 1] = add2(sum[c & 1], pair_of(x, y));
        p[c] = Half2Of<T>::pack(x, y);
    }
}
__device__ __forceinline__ float total(const f32x2 (&sum)[2])
{
    float a, b;
    split_pair(add2(sum[0], sum[1]), a, b);
    return a + b;
}

// Eight lanes with eight 16-byte pieces each (lane r: pieces of row r) -> lane c has piece c of the eight rows, so that a store
// instruction writes whole 128-byte lines of four rows instead of a piece of 32 (11 000 clocks per tile of fp32 results, 3000 so).
__device__ __forceinline__ void transpose_pieces(uint32_t (&v)[8][4], int lane)
{
#pragma unroll
    for (int bit = 1; bit < 8; bit <<= 1) {
        const bool up = lane & bit;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            if (k & bit) continue;
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const uint32_t got = __shfl_xor_sync(0xffffffffu, up ? v[k][w] : v[k | bit][w], bit);
                if (up) v[k][w] = got;
                else v[k | bit][w] = got;
            }
        }
    }
}

template <class T, int D, bool PAIR, bool MASKED>
__global__ void __launch_bounds__(THREADS, 1) tile_kernel(const __grid_constant__ Maps maps, const __grid_constant__ AttnArgs a)
{
    using L = Layout<D, PAIR>;
    using Range = WeightRange<T>;
    constexpr int SLOTS = L::SLOTS, AHEAD = PAIR ? 1 : 2;       // key tiles whose S is issued before the first P V
    extern __shared__ __align__(1024) unsigned char smem[];            // swizzled tiles start on 1024-byte boundaries
    unsigned char* ring = smem + L::RING;
    float* meet = reinterpret_cast<float*>(smem + L::MEET);
    uint64_t* full_bar = reinterpret_cast<uint64_t*>(smem + L::BARS);
    uint64_t* empty_bar = full_bar + SLOTS;
    uint64_t* s_full = empty_bar + SLOTS;
    uint64_t* p_full = s_full + 2;
    uint64_t* p_half = p_full + 2;
    uint64_t* seg_full = p_half + 2;
    uint64_t* seg_empty = seg_full + 2;
    uint64_t& q_full = seg_empty[2];
    uint64_t& q_empty = seg_empty[3];
    uint64_t& o_full = seg_empty[4];
    uint64_t& meet_bar = seg_empty[5];
    uint64_t& met_bar = seg_empty[6];
    TileWhere* where = reinterpret_cast<TileWhere*>(smem + L::WHERE);
    SegInfo* infos = reinterpret_cast<SegInfo*>(seg_empty + 7);
    uint32_t& tmem_slot = *reinterpret_cast<uint32_t*>(infos + 2);
    volatile uint32_t* abort_flag = &tmem_slot + 1;
    static_assert((2 * SLOTS + 17) * 8 + 2 * sizeof(SegInfo) + 8 <= 512, "barriers and descriptions fit");

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    cudaTriggerProgrammaticLaunchCompletion();       // the join's blocks may take their places; they wait for this grid's end
    if (threadIdx.x == 0) {
        for (int i = 0; i < SLOTS; ++i) { mbar_init(&full_bar[i], 1); mbar_init(&empty_bar[i], 1); }
        for (int i = 0; i < 2; ++i) {
            mbar_init(&s_full[i], 1);
            mbar_init(&p_half[i], 4);                                  // the group's warps
            mbar_init(&p_full[i], 4);
            mbar_init(&seg_full[i], 1);
            mbar_init(&seg_empty[i], 9);                               // MMA warp and eight softmax warps
        }
        mbar_init(&q_full, 1);
        mbar_init(&q_empty, 1);
        mbar_init(&o_full, 1);
        mbar_init(&meet_bar, 4);
        mbar_init(&met_bar, 4);
        *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_slot)), "r"(TMEM_COLS) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    cudaGridDependencySynchronize();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = __reduce_max_sync(0xffffffffu, tmem_slot);   // the same in every lane, and known to be
    auto tm_s = [&](int i) { return tmem + 128 * i; };                 // scores, then weights, of group i
    auto tm_o = [&](int i) { return tmem + 256 + 128 * i; };           // its accumulator
    const int tile_tok = min(BM / a.group, a.tok_per_item);            // tokens per 128-row tile

    const bool placed = a.list_mode != LIST_NONE || MASKED;           // the producer says where a tile's keys are
    // First position of virtual key v (a multiple of 16), or -1 where no block is listed.
    auto pos_of = [&](const AttnItem& it, int head, int v) -> int {
        if (MASKED) {
            const uint32_t* seen = a.unions + (static_cast<int64_t>(item_number(a, it)) * a.list_heads + (a.list_heads == 1 ? 0 : head)) * a.mask_words;
            return seen[v >> a.page_shift >> 5] >> (v >> a.page_shift & 31) & 1u ? v : -1;
        }
        if (a.list_mode == LIST_NONE) return v;
        const int e = v >> a.page_shift;
        if (e >= a.s || it.pos_last < 0) return -1;
        const int id = a.lists[(static_cast<int64_t>(it.list) * a.list_heads + (a.list_heads == 1 ? 0 : head)) * a.s + e];
        // a block all of whose positions are out of sight counts as not listed
        if (id < 0 || id > (it.pos_last >> a.page_shift) || ((id + 1) << a.page_shift) <= first_seen(a, it)) return -1;
        return (id << a.page_shift) + (v & (a.page_size - 1));
    };
    // Whether key tile `tile` of the block (at v0 of its segment) has rows without a position: their values have to be zeroed.
    auto unclean = [&](const AttnItem& it, int v0, uint32_t tile) -> bool {
        return !placed ? v0 + BN > it.kv : where[tile % 8].unclean != 0;
    };
    // First position of the u-th 16 keys of that tile.
    auto pos_at = [&](int v0, uint32_t tile, int u) -> int { return !placed ? v0 + 16 * u : where[tile % 8].pos[u]; };
    auto give_up = [&](uint32_t code) {
        dev_set_error(a.status, code);
        *abort_flag = 1;
    };

    // The launch gives every thread 168 registers; the four role warps hand some of theirs to the softmax rows (128 x 104 + 256 x 200 =
    // 384 x 168).
    uint32_t issued = 0;                                               // ring loads started
    if (warp < 4) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 104;");
        if (warp == 0) {
            // ---------------- producer ----------------
            // A lane per box: the lanes read the table entries of the next 32 boxes together, a group of tiles ahead of the
            // copies (one lane reading an entry before each copy bound the kernel at 2.5 us per key tile).
            prefetch_tables(a);
            if (lane == 0) {
                prefetch_map(maps.k);
                prefetch_map(maps.v);
                prefetch_map(maps.q);
            }
            Walk<BN> walk;
            Segment g, g_next;
            walk.start(a);
            bool some = walk.next(a, g), some_next = false;
            const int box = a.box_rows, per_tile = BN / box, group_tiles = 32 / per_tile;
            int segs = 0;
            uint32_t first_tile = 0;                                   // of the segment, among the block's
            bool ok = true;
            auto wait = [&](uint64_t* bar, uint32_t parity) {
                ok = __all_sync(0xffffffffu, mbar_wait(bar, parity, abort_flag));
                if (!ok && lane == 0) give_up(DEV_TIMEOUT_SMEM_EMPTY);
                return ok;
            };
            for (;;) {
                if (segs >= 2 && !wait(&seg_empty[segs & 1], ((segs >> 1) - 1) & 1)) break;
                if (lane == 0) {
                    infos[segs & 1] = SegInfo{g.it, g.head, g.t_lo, some ? g.t_hi - g.t_lo : 0, g.v_base, g.slot};
                    mbar_arrive(&seg_full[segs & 1]);
                }
                if (!some) break;
                const int n_tiles = g.t_hi - g.t_lo, v_lo = g.v_base + g.t_lo * BN;
                const int32_t* table = a.b.pages + g.it.seq * a.b.ld_pages;
                const int gone = first_seen(a, g.it) - box;            // boxes from here and before end before every row's window
                auto entry = [&](int t, int& page, int& pos) {         // this lane's box of the group of tiles from t
                    page = -1;
                    pos = t + lane / per_tile < n_tiles ? pos_of(g.it, g.head, v_lo + t * BN + lane * box) : -1;
                    if (pos < 0 || pos >= g.it.kv) return;
                    page = a.n_pages;                                  // beyond the map: reads as zeros
                    if (pos <= gone) return;
                    const int p = table[pos >> a.page_shift];
                    if (p < 0 || p >= a.n_pages) dev_set_error(a.status, DEV_BAD_PAGE);
                    else page = p;
                };
                int t0 = 0, page0, pos0, page1, pos1;                  // groups from t0 and from t0 + group_tiles
                entry(0, page0, pos0);
                entry(group_tiles, page1, pos1);
                if (segs > 0 && !wait(&q_empty, (segs - 1) & 1)) break;
                ++segs;
                if (lane == 0) {
                    mbar_expect_tx(&q_full, L::Q_TILES * static_cast<uint32_t>(tile_tok * a.group) * D * 2);
                    for (int i = 0; i < L::Q_TILES; ++i)
                        for (int h = 0; h < D / 64; ++h)
                            tma_load_4d(smem + i * BM * D * 2 + h * BM * 128, maps.q, h * 64, 0, g.head, g.it.tok0 + i * tile_tok, &q_full);
                }
                auto load = [&](int j, bool value) -> bool {
                    const uint32_t st = issued % SLOTS, round = issued / SLOTS;
                    const int x = j - t0, from = (x % group_tiles) * per_tile + lane % per_tile;
                    const int pa = __shfl_sync(0xffffffffu, page0, from), pb = __shfl_sync(0xffffffffu, page1, from);
                    const int qa = __shfl_sync(0xffffffffu, pos0, from), qb = __shfl_sync(0xffffffffu, pos1, from);
                    const int page = x < group_tiles ? pa : pb, pos = x < group_tiles ? qa : qb;
                    if (round > 0 && !wait(&empty_bar[st], (round - 1) & 1)) return false;
                    const bool mine = lane < per_tile && page >= 0;
                    const uint32_t boxes = __popc(__ballot_sync(0xffffffffu, mine));
                    if (!value && placed) {
                        TileWhere& w = where[(first_tile + j) % 8];
                        const int units = box / 16;
                        const bool part = lane < per_tile && (page < 0 || pos + box > g.it.kv);
                        const uint32_t parts = __ballot_sync(0xffffffffu, part);
                        if (lane < per_tile)
                            for (int u = 0; u < units; ++u) w.pos[lane * units + u] = page < 0 || pos + 16 * u >= g.it.kv ? -1 : pos + 16 * u;
                        if (lane == 0) w.unclean = parts != 0;
                        __syncwarp();
                    }
                    if (lane == 0) {
                        if (boxes) mbar_expect_tx(&full_bar[st], boxes * static_cast<uint32_t>(box) * D * 2);
                        else mbar_arrive(&full_bar[st]);
                    }
                    ++issued;
                    __syncwarp();
                    if (mine) {
                        unsigned char* dst = ring + st * L::TILE_BYTES + lane * box * 128;
#pragma unroll
                        for (int h = 0; h < D / 64; ++h)
                            tma_load_4d(dst + h * BN * 128, value ? maps.v : maps.k, h * 64, pos & (a.page_size - 1), g.head, page, &full_bar[st]);
                    }
                    return true;
                };
                for (int j = 0; j < min(AHEAD, n_tiles) && ok; ++j) load(j, false);
                for (int j = 0; j < n_tiles && ok; ++j) {
                    if (!load(j, true)) break;
                    if (j + AHEAD < n_tiles) load(j + AHEAD, false);
                    // the next segment is looked up while the ring is full
                    if (j == min(2, n_tiles - 1)) some_next = walk.next(a, g_next);
                    if (j + 1 - t0 == group_tiles) {
                        t0 += group_tiles;
                        page0 = page1;
                        pos0 = pos1;
                        entry(t0 + group_tiles, page1, pos1);
                    }
                }
                if (!ok) break;
                first_tile += n_tiles;
                g = g_next;
                some = some_next;
            }
            if (lane == 0) walk.leave_cut(a);
            if (lane == 0 && *abort_flag) {                            // no copy may be in flight when the block leaves
                if (segs > 0) mbar_wait(&q_full, (segs - 1) & 1, nullptr);
                for (uint32_t x = issued > SLOTS ? issued - SLOTS : 0; x < issued; ++x) mbar_wait(&full_bar[x % SLOTS], (x / SLOTS) & 1, nullptr);
            }
        } else if (warp == 1) {
            // ---------------- MMA issuer ----------------
            {
                const uint32_t one = elect_one();
                constexpr uint32_t fmt = Half2Of<T>::is_bf16 ? 1u : 0u;
                constexpr uint32_t base = (1u << 4) | (fmt << 7) | (fmt << 10) | (static_cast<uint32_t>(BM >> 4) << 24);
                constexpr uint32_t idesc_s = base | (static_cast<uint32_t>(BN >> 3) << 17);
                constexpr uint32_t idesc_o = base | (1u << 16) | (static_cast<uint32_t>(D >> 3) << 17);     // V: MN-major
                // 227 KB of shared memory: an address in 16-byte units never carries out of its 14 bits
                const uint32_t q_desc = desc_lo(smem_u32(smem), 16), k_desc = desc_lo(smem_u32(ring), 16), v_desc = desc_lo(smem_u32(ring), BN * 128);
                uint32_t used = 0, turns0 = 0, turns1 = 0;             // ring loads, weights taken from each group
                uint32_t tile = 0;                                     // key tiles of the block so far
                bool ok = true;
                auto need = [&](uint64_t* bar, uint32_t parity, uint32_t code) {
                    ok = ok && __all_sync(0xffffffffu, mbar_wait(bar, parity, abort_flag));
                    if (!ok && lane == 0) give_up(code);
                    return ok;
                };
                auto slot_ready = [&]() { return need(&full_bar[used % SLOTS], (used / SLOTS) & 1, DEV_TIMEOUT_TMA_FULL); };
                auto scores = [&](int i, int qt, uint32_t st) {
                    tc_fence_after();
#pragma unroll
                    for (int k = 0; k < D / 16; ++k) {
                        const uint32_t off = ((k >> 2) * (BM * 128) + (k & 3) * 32) >> 4;
                        mma_ss(one, tm_s(i), q_desc + qt * (BM * D * 2 >> 4) + off, k_desc + st * (L::TILE_BYTES >> 4) + off, idesc_s, k > 0);
                    }
                    commit(one, &s_full[i]);
                };
                auto product = [&](int i, uint32_t st, bool acc, uint32_t parity) {
#pragma unroll
                    for (int k = 0; k < BN / 16; ++k) {
                        if (k == 0 && !need(&p_half[i], parity, DEV_TIMEOUT_ACC_EMPTY)) return false;
                        if (k == BN / 32 && !need(&p_full[i], parity, DEV_TIMEOUT_ACC_EMPTY)) return false;
                        if (k % (BN / 32) == 0) tc_fence_after();
                        mma_ts(one, tm_o(i), tm_s(i) + k * 8, v_desc + st * (L::TILE_BYTES >> 4) + k * (2048 >> 4), idesc_o, acc || k > 0);
                    }
                    return true;
                };
                for (int seg = 0; ok; ++seg) {
                    if (!need(&seg_full[seg & 1], (seg >> 1) & 1, DEV_TIMEOUT_TMA_FULL)) break;
                    const SegInfo& info = infos[seg & 1];              // stays there until this segment is done
                    const int n_tiles = __reduce_max_sync(0xffffffffu, info.n_tiles), v_lo = __reduce_max_sync(0xffffffffu, info.v_base + info.t_lo * BN);
                    if (n_tiles == 0) break;
                    need(&q_full, seg & 1, DEV_TIMEOUT_TMA_FULL);
                    for (int j = 0; j < min(AHEAD, n_tiles) && ok; ++j) {
                        if (!slot_ready()) break;
                        const uint32_t st = used % SLOTS;
                        if (PAIR) { scores(0, 0, st); scores(1, 1, st); }
                        else scores(j & 1, 0, st);
                        commit(one, &empty_bar[st]);
                        ++used;
                    }
                    if (ok && n_tiles <= AHEAD) commit(one, &q_empty);
                    for (int j = 0; j < n_tiles && ok; ++j, ++tile) {
                        if (!slot_ready()) break;
                        const uint32_t sv = used % SLOTS;
                        ++used;
                        if (unclean(info.it, v_lo + j * BN, tile)) {
                            // rows of V that hold no position may hold anything (a page's tail, an older tile): zero them
                            unsigned char* tile_v = ring + sv * L::TILE_BYTES;
                            for (int u = 0; u < BN / 16; ++u) {
                                const int pos = pos_at(v_lo + j * BN, tile, u), there = pos < 0 ? 0 : min(max(info.it.kv - pos, 0), 16);
                                for (int x = lane; x < (16 - there) * (D / 8); x += 32) {
                                    const int row = 16 * u + there + x / (D / 8), c = x % (D / 8);
                                    *reinterpret_cast<uint4*>(tile_v + (c >> 3) * BN * 128 + row * 128 + (c & 7) * 16) = make_uint4(0, 0, 0, 0);
                                }
                            }
                            fence_async_smem();
                            __syncwarp();
                        }
                        const bool more = j + AHEAD < n_tiles;
                        const uint32_t sk = used % SLOTS;
                        if (PAIR) {
#pragma unroll
                            for (int i = 0; i < 2; ++i) {
                                if (!product(i, sv, j > 0, turns0 & 1)) break;
                                if (i == 1) commit(one, &empty_bar[sv]);
                                if (more) {
                                    if (i == 0 && !slot_ready()) break;
                                    scores(i, i, sk);
                                }
                            }
                            ++turns0;
                            if (more && ok) { commit(one, &empty_bar[sk]); ++used; }
                        } else {
                            const int i = j & 1;
                            if (!product(i, sv, j > 1, (i ? turns1 : turns0) & 1)) break;
                            if (i) ++turns1;
                            else ++turns0;
                            commit(one, &empty_bar[sv]);
                            if (more) {
                                if (!slot_ready()) break;
                                scores(i, 0, sk);
                                commit(one, &empty_bar[sk]);
                                ++used;
                            }
                        }
                        if (ok && more && j + AHEAD + 1 == n_tiles) commit(one, &q_empty);      // the segment's last S has been issued
                    }
                    if (ok) commit(one, &o_full);
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&seg_empty[seg & 1]);
                }
            }
        }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 200;");
        // ---------------- softmax ----------------
        const int i = (warp - 4) >> 2;                                 // group
        const int row = (warp & 3) * 32 + lane;                        // row of the tile = lane of tensor memory
        const uint32_t lane_base = static_cast<uint32_t>((warp & 3) * 32) << 16;
        const uint32_t my_s = tm_s(i) + lane_base, my_o = tm_o(i) + lane_base;
        const int first_tok = PAIR ? i * tile_tok : 0;                 // first token of the tile, relative to the item
        const int tok = first_tok + row / a.group, g = row % a.group;
        const f32x2 scale2 = pair_of(a.scale_log2, a.scale_log2);
        constexpr float most = static_cast<float>(1 << static_cast<int>(Range::most));
        uint32_t turn = 0, tile0 = 0;                                  // key tiles this group has taken; the block's before this segment
        bool ok = true;
        for (int seg = 0;; ++seg) {
            ok = __all_sync(0xffffffffu, mbar_wait(&seg_full[seg & 1], (seg >> 1) & 1, abort_flag));
            if (!ok) break;
            const SegInfo& info = infos[seg & 1];                      // stays there until this segment is done
            if (info.n_tiles == 0) break;
            const bool live = row < tile_tok * a.group && tok < info.it.n_tok;
            const int qpos = a.causal ? info.it.pos0 + tok : info.it.pos0;
            const int qlo = a.causal ? info.it.pos0 + first_tok : info.it.pos0;      // smallest and largest position of the tile's rows
            const int qhi = a.causal ? min(qlo + tile_tok - 1, info.it.pos_last) : qlo;
            float m = -INFINITY, l = 0.0f;                             // reference of the exponentials (scaled, base 2), sum
            int turns = 0;
            // the row's blocks, where lists came as masks: those of a key tile are in one word (a tile holds 1, 2, 4 or 8)
            const uint32_t* mask_row = MASKED && live ? a.masks + (static_cast<int64_t>(info.it.tok0 + tok) * a.list_heads +
                                                                    (a.list_heads == 1 ? 0 : info.head)) * a.mask_words : nullptr;
            const uint32_t all_bits = (1u << (BN >> a.page_shift)) - 1;
            uint32_t bits = all_bits;
            auto bits_of = [&](int v) { return mask_row[v >> a.page_shift >> 5] >> (v >> a.page_shift & 31) & all_bits; };
            for (int j = PAIR ? 0 : i; j < info.n_tiles; j += PAIR ? 1 : 2, ++turns, ++turn) {
                ok = __all_sync(0xffffffffu, mbar_wait(&s_full[i], turn & 1, abort_flag));
                if (!ok) break;
                tc_fence_after();
                const int v0 = info.v_base + (info.t_lo + j) * BN;
                const uint32_t tile = tile0 + j;
                float s[4][32];
                tm_ld32(my_s, s[0]);
                if (MASKED) bits = mask_row ? bits_of(v0) : 0u;
                bool look;                                             // some row may not see some key, or there is no reference yet
                if (!placed) look = v0 + BN - 1 > qlo || (a.window > 0 && v0 <= qhi - a.window);
                else {
                    look = false;
#pragma unroll
                    for (int u = 0; u < BN / 16; ++u) {
                        const int pos = where[tile % 8].pos[u];
                        look |= pos < 0 || pos + 15 > qlo || (a.window > 0 && pos <= qhi - a.window);
                    }
                }
                const bool edge = look, part = MASKED && __any_sync(0xffffffffu, live && bits != all_bits);
                look |= part || turns == 0;
                wait_ld();
#pragma unroll
                for (int c = 1; c < 4; ++c) tm_ld32(my_s + 32 * c, s[c]);

                // Where keys are masked, and on the first tile, the tile's maximum is looked at first. Otherwise the weights are made
                // with the reference as it stands; before the first half of them is handed over, its sum and the largest score of
                // the second half, which the multiply-add pipes find meanwhile, tell whether a weight may be too large (or a score
                // is not a number), and then it is done over with the maximum looked at.
                uint32_t p_lo[32], p_hi[32];
                f32x2 sum[2], ref2;
                for (;;) {
                    if (look) {
                        wait_ld();
                        if (edge) {
#pragma unroll
                            for (int u = 0; u < BN / 16; ++u) {
                                int pos = pos_at(v0, tile, u);
                                if (MASKED && !(bits >> (16 * u >> a.page_shift) & 1u)) pos = -1;
                                const int hi = pos < 0 ? -1 : qpos - pos, lo = a.window > 0 ? hi - a.window : -1;      // visible: lo < c <= hi
#pragma unroll
                                for (int c = 0; c < 16; ++c)
                                    if (c > hi || c <= lo) s[u / 2][u % 2 * 16 + c] = -INFINITY;
                            }
                        } else if (part) {
#pragma unroll
                            for (int u = 0; u < BN / 16; ++u) {
                                const bool off = !(bits >> (16 * u >> a.page_shift) & 1u);
#pragma unroll
                                for (int c = 0; c < 16; ++c)
                                    if (off) s[u / 2][u % 2 * 16 + c] = -INFINITY;
                            }
                        }
                        const float a_lo = max_of(s[0]), b_lo = max_of(s[1]), a_hi = max_of(s[2]), b_hi = max_of(s[3]);
                        const float top = fmaxf(fmaxf(a_lo, b_lo), fmaxf(a_hi, b_hi)) * a.scale_log2;
                        const bool grow = live && top > m + Range::grow;
                        if (__any_sync(0xffffffffu, grow)) {
                            const float now = grow ? top - Range::lift : m;
                            const float f = m == -INFINITY ? 0.0f : ex2(m - now);
                            m = now;
                            l *= f;
                            if (turns > 0) {
#pragma unroll
                                for (int c = 0; c < D; c += 16) {      // narrow steps: the scores stay in registers meanwhile
                                    float o[16];
                                    tm_ld16(my_o + c, o);
                                    wait_ld();
#pragma unroll
                                    for (int x = 0; x < 16; ++x) o[x] *= f;
                                    tm_st16(my_o + c, o);
                                }
                            }
                        }
                    }
                    const float ref = m == -INFINITY ? 0.0f : -m;
                    ref2 = pair_of(ref, ref);
                    sum[0] = sum[1] = 0;                               // pairs of +0
                    weights<T>(s[0], scale2, ref2, p_lo, sum);
                    wait_ld();
                    weights<T>(s[1], scale2, ref2, p_lo + 16, sum);
                    if (look) break;
                    const float a_hi = max_of(s[2]), b_hi = max_of(s[3]), top = max3(a_hi, b_hi, b_hi) * a.scale_log2;
                    look = __any_sync(0xffffffffu, live && !(total(sum) <= most && top <= m + Range::most));
                    if (!look) break;
                }
                tm_st32(my_s, p_lo);
                weights<T>(s[2], scale2, ref2, p_hi, sum);
                wait_st();
                // the first product of a segment overwrites the odd group's accumulator, which the even group may still be reading
                if (!PAIR && i == 1 && turns == 0 && seg > 0) {
                    ok = __all_sync(0xffffffffu, mbar_wait(&met_bar, (seg - 1) & 1, abort_flag));
                    if (!ok) break;
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&p_half[i]);                // one arrival per warp: 128 on one barrier take turns
                weights<T>(s[3], scale2, ref2, p_hi + 16, sum);
                tm_st32(my_s + 32, p_hi);
                wait_st();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&p_full[i]);
                l += total(sum);
            }
            tile0 += info.n_tiles;
            // ---------------- results ----------------
            if (ok) ok = __all_sync(0xffffffffu, mbar_wait(&o_full, seg & 1, abort_flag));
            if (ok && !PAIR) {
                // the even tiles' group reads the odd one's accumulator itself (same lanes of tensor memory)
                if (i == 1) {
                    if (turns == 0 && seg > 0) ok = __all_sync(0xffffffffu, mbar_wait(&met_bar, (seg - 1) & 1, abort_flag));
                    meet[row] = m;
                    meet[128 + row] = l;
                    __syncwarp();
                    if (ok && lane == 0) mbar_arrive(&meet_bar);
                } else ok = __all_sync(0xffffffffu, mbar_wait(&meet_bar, seg & 1, abort_flag));
            }
            if (!ok) break;
            tc_fence_after();
            if (PAIR || i == 0) {
                float f_own = 1.0f, f_other = 0.0f;
                if (!PAIR) {
                    const float m1 = meet[row], l1 = meet[128 + row], both = fmaxf(m, m1), both_ref = both == -INFINITY ? 0.0f : both;
                    f_own = ex2(m - both_ref);
                    f_other = ex2(m1 - both_ref);
                    l = l * f_own + l1 * f_other;
                    m = both;
                }
                const bool other = !PAIR && info.n_tiles > 1, empty = l == 0.0f;
                const float inv = empty ? 0.0f : 1.0f / l;
                f_own *= inv;
                f_other *= inv;
                const int t = info.it.tok0 + tok, h = info.head * a.group + g;
                const int64_t out_row = static_cast<int64_t>(t) * a.n_heads + h;
                const int64_t part = static_cast<int64_t>(info.slot) * a.rows_cap + first_tok * a.group + row;
                const float lse2 = empty ? -INFINITY : m + log2f(l);
                if (live) {
                    if (info.slot >= 0) a.part_lse[part] = lse2;
                    else if (a.lse) a.lse[out_row] = lse2 * kLn2;
                }
                // a store's lane writes piece lane % 8 of the lines of rows x + 8 (lane / 8)
                auto scaled = [&](int c, float (&o)[32]) {             // 32 results of this lane's row
                    tm_ld32(my_o + c, o);
                    wait_ld();
#pragma unroll
                    for (int x = 0; x < 32; ++x) o[x] = empty ? 0.0f : o[x] * f_own;
                    if (other) {
                        float z[32];
                        tm_ld32(tm_o(1) + lane_base + c, z);
                        wait_ld();
#pragma unroll
                        for (int x = 0; x < 32; ++x) o[x] = empty ? 0.0f : fmaf(z[x], f_other, o[x]);
                    }
                };
                const uint32_t alive = __ballot_sync(0xffffffffu, live);
                const int my_piece = lane & 7, my_row = lane & 24;
                if (info.slot >= 0) {
                    float* base = a.part_o + (part - lane) * D;        // the warp's first row
#pragma unroll 1
                    for (int c = 0; c < D; c += 32) {
                        float o[32];
                        scaled(c, o);
                        uint32_t v[8][4];
#pragma unroll
                        for (int x = 0; x < 32; ++x) v[x / 4][x % 4] = __float_as_uint(o[x]);
                        transpose_pieces(v, lane);
#pragma unroll
                        for (int x = 0; x < 8; ++x)
                            if (alive >> (my_row + x) & 1)
                                *reinterpret_cast<uint4*>(base + (my_row + x) * D + c + my_piece * 4) = make_uint4(v[x][0], v[x][1], v[x][2], v[x][3]);
                    }
                } else {
                    T* dst = static_cast<T*>(a.out) + static_cast<int64_t>(t) * a.ld_out + static_cast<int64_t>(h) * D;
                    const uint64_t mine = reinterpret_cast<uint64_t>(dst);
#pragma unroll 1
                    for (int c = 0; c < D; c += 64) {
                        uint32_t v[8][4];
#pragma unroll
                        for (int y = 0; y < 2; ++y) {
                            float o[32];
                            scaled(c + 32 * y, o);
#pragma unroll
                            for (int x = 0; x < 32; x += 2) v[4 * y + x / 8][x / 2 % 4] = Half2Of<T>::pack(o[x], o[x + 1]);
                        }
                        transpose_pieces(v, lane);
#pragma unroll
                        for (int x = 0; x < 8; ++x) {
                            T* to = reinterpret_cast<T*>(__shfl_sync(0xffffffffu, mine, my_row + x));
                            if (alive >> (my_row + x) & 1)
                                *reinterpret_cast<uint4*>(to + c + my_piece * 8) = make_uint4(v[x][0], v[x][1], v[x][2], v[x][3]);
                        }
                    }
                }
                tc_fence_before();
                __syncwarp();
                if (!PAIR && lane == 0) mbar_arrive(&met_bar);
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(&seg_empty[seg & 1]);
        }
        if (!ok && lane == 0) give_up(DEV_TIMEOUT_ACC_FULL);
        tc_fence_before();
    }
    __syncthreads();
    if (warp == 1) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(TMEM_COLS) : "memory");
    }
}

// Lists per token -> masks, and their union over the tokens of an item: a block per item and list head, a warp per token. Entries
// past the masks' width are past every sequence's end.
constexpr int MASK_WARPS = 32;
__global__ void __launch_bounds__(32 * MASK_WARPS) mask_kernel(const AttnArgs a)
{
    __shared__ uint32_t row[MASK_WARPS][kMaxMaskWords], all[kMaxMaskWords];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, words = a.mask_words;
    for (int w = threadIdx.x; w < words; w += blockDim.x) all[w] = 0u;
    cudaTriggerProgrammaticLaunchCompletion();
    cudaGridDependencySynchronize();
    __syncthreads();
    AttnItem it;
    if (!attn_item(a, blockIdx.x, it)) return;                         // the same for every warp
    for (int tok = warp; tok < it.n_tok; tok += MASK_WARPS) {
        const int64_t list = static_cast<int64_t>(it.tok0 + tok) * a.list_heads + blockIdx.y;
        for (int w = lane; w < words; w += 32) row[warp][w] = 0u;
        __syncwarp();
        for (int e = lane; e < a.s; e += 32) {
            const int id = a.lists[list * a.s + e];
            if (id >= 0 && id < words * 32) atomicOr(&row[warp][id >> 5], 1u << (id & 31));
        }
        __syncwarp();
        for (int w = lane; w < words; w += 32) {
            a.masks[list * words + w] = row[warp][w];
            if (row[warp][w]) atomicOr(&all[w], row[warp][w]);
        }
        __syncwarp();
    }
    __syncthreads();
    uint32_t* out = a.unions + (static_cast<int64_t>(item_number(a, it)) * a.list_heads + blockIdx.y) * words;
    for (int w = threadIdx.x; w < words; w += blockDim.x) out[w] = all[w];
}

template <class T, int D, bool PAIR, bool MASKED>
s3_status launch_tile(const KvCacheState& c, const AttnArgs& a, cudaStream_t stream)
{
    using L = Layout<D, PAIR>;
    const s3_status allowed = allow_smem<tile_kernel<T, D, PAIR, MASKED>>(L::TOTAL);
    if (allowed != S3_OK) return allowed;
    Maps maps;
    memcpy(maps.k, c.map_k, sizeof(maps.k));
    memcpy(maps.v, c.map_v, sizeof(maps.v));
    const int tile_tok = BM / a.group < a.tok_per_item ? BM / a.group : a.tok_per_item;
    s3_status st = make_kv_query_map(maps.q, c, a.q, a.ldq, a.b.T, a.group, tile_tok);
    if (st != S3_OK) return st;
    return launch_overlapped(tile_kernel<T, D, PAIR, MASKED>, dim3(a.grid), THREADS, L::TOTAL, stream, maps, a);
}

template <class T, int D>
s3_status launch_dim(const KvCacheState& c, const AttnArgs& a, cudaStream_t stream)
{
    // masks as a variant of their own: in one kernel with the others they cost those 4 % (registers), lists or not
    if (a.tok_per_item > BM / a.group) return a.masks ? launch_tile<T, D, true, true>(c, a, stream) : launch_tile<T, D, true, false>(c, a, stream);
    return a.masks ? launch_tile<T, D, false, true>(c, a, stream) : launch_tile<T, D, false, false>(c, a, stream);
}

}  // namespace

s3_status launch_attn_masks(const AttnArgs& a, cudaStream_t stream)
{
    return launch_overlapped(mask_kernel, dim3(a.n_items, a.list_heads), 32 * MASK_WARPS, 0, stream, a);
}

s3_status launch_attn_tile(const KvCacheState& c, const AttnArgs& a, cudaStream_t stream)
{
    const bool wide = c.d.head_dim == 128;
    if (c.d.dtype == S3_BF16) return wide ? launch_dim<__nv_bfloat16, 128>(c, a, stream) : launch_dim<__nv_bfloat16, 64>(c, a, stream);
    return wide ? launch_dim<__half, 128>(c, a, stream) : launch_dim<__half, 64>(c, a, stream);
}

}  // namespace s3
