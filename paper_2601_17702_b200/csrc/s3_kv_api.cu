// C ABI of the paged key / value cache: argument checks, the cache handle with its copy descriptors, and the choice of kernel
// and splits for attention.
#include <math.h>
#include <string.h>

#include <new>

#include "s3_kernels.cuh"
#include "s3_kv.cuh"

namespace s3 {
namespace {

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                  const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                  CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

s3_status encode_fn(EncodeTiledFn* out)
{
    static EncodeTiledFn fn = nullptr;
    if (!fn) {
        void* sym = nullptr;
        cudaDriverEntryPointQueryResult qres;
        S3_CUDA_TRY(cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &sym, cudaEnableDefault, &qres));
        S3_REQUIRE(sym != nullptr && qres == cudaDriverEntryPointSuccess, S3_ERR_CUDA, "the driver does not provide cuTensorMapEncodeTiled");
        fn = reinterpret_cast<EncodeTiledFn>(sym);
    }
    *out = fn;
    return S3_OK;
}

// Map of values of N dimensions, 64 columns first (bytes: the whole row of 64 or 128); strides in elements; rows of the box swizzled.
template <int N>
s3_status make_map(unsigned char (&map)[128], CUtensorMapDataType type, const void* base, const uint64_t (&dims)[N], const uint64_t (&strides)[N - 1],
                   const uint32_t (&box)[N])
{
    static_assert(sizeof(CUtensorMap) == 128, "a copy descriptor has 128 bytes");
    EncodeTiledFn fn;
    const s3_status st = encode_fn(&fn);
    if (st != S3_OK) return st;
    cuuint64_t d[N], s[N - 1];
    cuuint32_t b[N], unit[N];
    const int size = type == CU_TENSOR_MAP_DATA_TYPE_UINT8 ? 1 : 2;
    for (int i = 0; i < N; ++i) {
        d[i] = dims[i];
        b[i] = box[i];
        unit[i] = 1;
        if (i + 1 < N) s[i] = strides[i] * size;
    }
    const CUresult r = fn(reinterpret_cast<CUtensorMap*>(map), type, N, const_cast<void*>(base), d, s, b, unit, CU_TENSOR_MAP_INTERLEAVE_NONE,
                          box[0] * size == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B,
                          CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    S3_REQUIRE(r == CUDA_SUCCESS, S3_ERR_CUDA, "cuTensorMapEncodeTiled failed with code %d", static_cast<int>(r));
    return S3_OK;
}

CUtensorMapDataType map_type(s3_dtype dtype) { return dtype == S3_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16; }

// Rows per item up to which the split kernel serves (its registers hold 16). Split and tile kernel there, keys times 8 heads of 128: one
// row over 131072 keys times 4 heads 92 and 105 us, 32 sequences of 16 rows over 8192 176 and 191, over 2000 62 and 86, 64 over 700
// 52 and 92, one over 777 20.1 and 19.5; lists per token, 64 tokens of 8 heads 30 and 71, of 16 heads 42 and 71.
constexpr int kSplitRows = 16;
constexpr int kTileRows = 128;

// Modelled time of a pair tile under masks, and of the masks themselves and the start (us).
constexpr double kMaskedTile = 2.7, kMaskedFixed = 12.0;

// Keys and values of a sequence from which whole rounds go before shares (bytes), see choose_shares.
constexpr int64_t kRoundsBytes = 76000000;

// What a plan depends on beside the batch's bounds.
struct PlanShape {
    int sms, group, n_kv_heads, page_shift;
    int held_bytes;                        // of a key and its value
    bool i8;
};

// Bytes of a key and its value as pages hold them.
int held_bytes(int head_dim, bool i8) { return i8 ? 2 * (head_dim + 4) : 4 * head_dim; }

// How an attention call is cut. None of it depends on the device-side lengths.
struct AttnPlan {
    bool tile;                             // tile kernel, else split kernel
    bool masked;                           // lists per token as masks over all blocks
    int tok_per_item, n_items, one_item_per_seq;
    int grid, share_min, whole_rounds, rows_cap;
};

// Chooses whole units or shares for a plan whose items are set, and returns the modelled time in key tiles. tile_cost: time of one of
// this plan's key tiles; extra: what shares cost beside their tiles (second launch, partial results, segments cut short): 12 tiles of
// the split kernel, 6 of the tile kernel. Whole and shares measured (us, 4 x 8 heads of 128):
//   split, lists of 16 blocks of 64, of 8 sequences 16.8 and 15.0, of 16 19.6 and 23.9, 24 24.7 and 28.9, 36 31.9 and 33.4, 48 (two rounds)
//   43.7 and 46.3; one row over 500 keys 10.4 and 11.7, 777 13.1 and 13.5, 1500 18.5 and 12.4, 6000 57 and 16;
//   tile, one query tile, 64 tokens over 500 keys 15.9 and 20.4, 1000 20.3 and 20.7, 2000 29.9 and 23.3; 256 over 4000 49 and 42; 512 over
//   4000 51 and 58; two query tiles, 4 x 128 over 1000 27.5 and 33.6, 4 x 128 over 3000 57 and 55, 8 x 128 over 3000 108 and 80.
double choose_shares(AttnPlan& p, const s3_kv_batch& b, const PlanShape& c, int list_mode, int64_t keys, double tile_cost, double extra)
{
    const int64_t places = (p.tile ? 1 : 2) * static_cast<int64_t>(c.sms);     // thread blocks that run at a time
    const int64_t units = static_cast<int64_t>(p.n_items) * c.n_kv_heads, tiles = (keys + (p.tile ? 127 : 63)) / (p.tile ? 128 : 64);
    // Lists and the items of one sequence are alike: whole units take whole rounds. Sequences of a batch may have any length up to
    // max_kv, which the host does not see: on average taken as 0.6 of it, and whole units end with the longest. Whole and shares, one
    // row each: 24 sequences of up to 4000 keys 48.6 and 43.5, 16 43.5 and 34.6, 80 (three rounds) 141 and 117. Where they are all of
    // the bound's length the guess loses: 24 of 2000 35.6 and 42.2 (taken), 16 chunks of 64 tokens over 4000 78 and 101 (taken).
    const bool alike = list_mode != LIST_NONE || b.n_seqs == 1;
    const int64_t rounds = (units + places - 1) / places;
    const double whole = alike || rounds <= 1 ? static_cast<double>(rounds * tiles) * tile_cost : 1e30;
    const double share = (alike ? 1.0 : 0.6) * static_cast<double>(units) * tiles / places * tile_cost + extra;
    p.whole_rounds = 0;
    if (whole <= share) {
        p.grid = static_cast<int>(units < places ? units : places);
        p.share_min = 0;
        return whole;
    }
    p.grid = static_cast<int>(places);
    // A share has at least this many tiles, or the join has more pieces than it saves. Least shares of 1, 2, 4, 8 tiles: split, one row
    // over 777 keys 11.1, 13.1, 13.3, 16.2, over 3000 14.5, 14.5, 14.8, 17.2; of 1, 2, 4: tile, 64 tokens over 1000 23.4, 23.5, 25.8.
    p.share_min = p.tile || c.i8 ? 2 : 4;                              // 8-bit pages: the split kernel's tiles hold twice the keys
    // A chunk late in a prompt: units of nearly equal length. Whole rounds of them may go first, all blocks sweeping the keys in step, and
    // only the rest be shared: the blocks of a key head then read the same tiles at the same time, which counts once the keys and
    // values of the sequence no longer stay in the L2 cache. Shares only and with rounds, from rest, 2048 tokens of 4 x 8 heads of 128:
    // over 9000 keys (37 MB) 251 and 262 us, 16384 (67 MB) 432 and 438, 20000 (82 MB) 535 and 530, 24000 (98 MB) 653 and 626, 32768
    // (134 MB) 929 and 846; 2700 tokens of 7 x 4 heads over 11000 (23 MB) 336 and 367, over 65536 (134 MB) 2116 and 1961.
    if (p.tile && list_mode == LIST_NONE && b.n_seqs == 1 && b.max_kv >= 4 * static_cast<int64_t>(b.max_q) &&
        static_cast<int64_t>(b.max_kv) * c.n_kv_heads * c.held_bytes >= kRoundsBytes)
        p.whole_rounds = static_cast<int>(units / places);
    return share;
}

// Items of several tokens of a sequence; keys: the most virtual keys an item can have; time: modelled, in key tiles.
AttnPlan plan_tokens(const s3_kv_batch& b, const PlanShape& c, int list_mode, int64_t keys, double& time)
{
    AttnPlan p;
    p.masked = false;
    p.tile = static_cast<int64_t>(b.max_q) * c.group > kSplitRows;
    const int one = (p.tile ? kTileRows : kSplitRows) / c.group;
    auto items = [&](AttnPlan& q, int tokens) {
        q.tok_per_item = tokens;
        q.one_item_per_seq = b.max_q <= tokens;
        q.n_items = q.one_item_per_seq ? b.n_seqs : b.n_seqs == 1 ? (b.T + tokens - 1) / tokens : b.T / tokens + b.n_seqs;
    };
    items(p, one);
    // With one query tile per item the two softmax groups share the keys: a key tile takes a little more than half the time that it
    // takes with two, there are twice as many units, and every key is copied twice as often. One and two, 4 x 8 heads of 128: 512
    // tokens over 1000 keys 20.7 and 26.5, 1 x 64 over 2000 23.3 and 25.9; 4 x 128 over 1000 34 and 27.5, 16 x 64 over 1000 55 and 33, 8 x 128
    // over 3000 94 and 80.
    time = choose_shares(p, b, c, list_mode, keys, p.tile ? 0.6 : 1.0, p.tile ? 6.0 : 12.0);
    if (p.tile && b.max_q > one) {
        AttnPlan q = p;
        items(q, 2 * one);
        const double pair = choose_shares(q, b, c, list_mode, keys, 1.0, 6.0);
        if (pair <= time) {
            p = q;
            time = pair;
        }
    }
    return p;
}

int shift_of(int page_size) { return page_size == 16 ? 4 : page_size == 32 ? 5 : page_size == 64 ? 6 : 7; }

int mask_words(const s3_kv_batch& b, int page_shift) { return b.max_kv > 0 ? ((b.max_kv - 1) >> page_shift) / 32 + 1 : 1; }

// Masks of the tokens, and the unions of items of tok_per_item tokens or more.
size_t mask_bytes(const s3_kv_batch& b, int page_shift, int list_heads, int tok_per_item)
{
    const size_t words = mask_words(b, page_shift) < kMaxMaskWords ? mask_words(b, page_shift) : kMaxMaskWords;
    return round_up(static_cast<size_t>(b.T) * list_heads * words * 4, 256) +
           round_up((static_cast<size_t>(b.T) / tok_per_item + b.n_seqs) * list_heads * words * 4, 256);
}

// keys: the most virtual keys an item can have.
AttnPlan plan_attention(const s3_kv_batch& b, const PlanShape& c, int list_mode, int64_t keys)
{
    AttnPlan p;
    p.masked = false;
    if (list_mode == LIST_PER_TOKEN) {
        p.tile = c.group > kSplitRows;
        p.tok_per_item = 1;
        p.n_items = b.T;
        p.one_item_per_seq = 0;
        const double listed = choose_shares(p, b, c, list_mode, keys, 1.0, p.tile ? 6.0 : 12.0) * (p.tile ? 2.0 : 0.7);     // us
        // As masks over the blocks that an item lists: a key tile's copies and products serve up to 256 rows, in vain where a row
        // does not list the block, so it pays where the lists are a good part of the context. Measured as lists and as masks, 1024
        // tokens of 4 x 8 heads, 16 random blocks of 64 of each: over 2K keys 325 and 57 us, 8K 325 and 175, 16K 326 and 331, 32K 326
        // and 845; 32 tokens over 2K keys 16.5 and 24.8. The two constants are fitted to these and know neither head_dim nor page size:
        // with 8 blocks of 128 over 8K keys 322 and 177, 24 blocks of 16 184 and 247, 16 of 64 at head_dim 64 299 and 157, 600 tokens of 7 x 4
        // heads over 4K 107 and 73, 300 of 4 x 4 heads of 64 with 24 blocks of 16 over 4K 32.9 and 40.2, each the faster one taken.
        if (static_cast<int64_t>(b.max_q) * c.group > kSplitRows && mask_words(b, c.page_shift) <= kMaxMaskWords) {
            double over_all;
            AttnPlan q = plan_tokens(b, c, LIST_NONE, b.max_kv, over_all);
            if (over_all * kMaskedTile + kMaskedFixed < listed) {
                p = q;
                p.masked = true;
            }
        }
    } else {
        double time;
        p = plan_tokens(b, c, list_mode, keys, time);
    }
    p.rows_cap = p.tile ? p.tok_per_item * c.group : kSplitRows;
    return p;
}

// Partial results: two slots per thread block.
size_t partial_bytes(const AttnPlan& p, int head_dim)
{
    if (p.share_min == 0) return 0;
    const size_t rows = 2 * static_cast<size_t>(p.grid) * p.rows_cap;
    return round_up(rows * head_dim * 4, 256) + round_up(rows * 4, 256) + round_up(static_cast<size_t>(p.grid) * sizeof(Cut), 256);
}

}  // namespace

s3_status make_kv_query_map(unsigned char (&map)[128], const KvCacheState& c, const void* d_q, int64_t ldq, int T, int group, int box_tokens)
{
    const uint64_t D = c.d.head_dim;
    const uint64_t dims[4] = {D, static_cast<uint64_t>(group), static_cast<uint64_t>(c.d.n_kv_heads), static_cast<uint64_t>(T)};
    const uint64_t strides[3] = {D, D * group, static_cast<uint64_t>(ldq)};
    const uint32_t box[4] = {64, static_cast<uint32_t>(group), 1, static_cast<uint32_t>(box_tokens)};
    return make_map<4>(map, map_type(c.d.dtype), d_q, dims, strides, box);
}

}  // namespace s3

using namespace s3;

struct s3_kv_cache {
    KvCacheState st;
};

namespace {

s3_status check_batch(const s3_kv_cache* cache, const s3_kv_batch* b)
{
    S3_REQUIRE(cache != nullptr && b != nullptr, S3_ERR_INVALID_ARG, "cache or batch is null");
    S3_REQUIRE(b->n_seqs >= 0 && b->T >= 0 && b->max_q >= 0 && b->max_kv >= 0 && b->ld_pages >= 0, S3_ERR_INVALID_ARG,
               "n_seqs = %d, T = %d, max_q = %d, max_kv = %d, ld_pages = %lld out of range", b->n_seqs, b->T, b->max_q, b->max_kv,
               (long long)b->ld_pages);
    if (b->T == 0 || b->n_seqs == 0) return S3_OK;
    S3_REQUIRE(b->d_cu_q && b->d_kv_len && b->d_pages, S3_ERR_INVALID_ARG, "null pointer in the batch");
    S3_REQUIRE(aligned4(b->d_cu_q) && aligned4(b->d_kv_len) && aligned4(b->d_pages), S3_ERR_INVALID_ARG, "misaligned pointer in the batch");
    S3_REQUIRE(static_cast<int64_t>(b->max_kv) <= b->ld_pages * cache->st.d.page_size, S3_ERR_INVALID_ARG,
               "max_kv = %d does not fit %lld table entries of %d positions", b->max_kv, (long long)b->ld_pages, cache->st.d.page_size);
    S3_REQUIRE(b->max_q >= 1 && b->max_q <= b->T, S3_ERR_INVALID_ARG, "max_q = %d out of [1, T = %d]", b->max_q, b->T);
    S3_REQUIRE(b->max_kv <= (1 << 30) && b->T <= (1 << 30), S3_ERR_UNSUPPORTED, "more than 2^30 positions or rows");
    return S3_OK;
}

s3_status check_heads(int n_heads, int k)
{
    S3_REQUIRE(n_heads >= 1 && n_heads % k == 0, S3_ERR_INVALID_ARG, "n_heads = %d is not a multiple of %d key heads", n_heads, k);
    S3_REQUIRE(n_heads / k <= S3_MAX_HEAD_GROUP, S3_ERR_UNSUPPORTED, "%d query heads per key head exceed %d", n_heads / k, S3_MAX_HEAD_GROUP);
    return S3_OK;
}

s3_status check_rows(const char* what, const void* p, int64_t ld, int heads, int dim)
{
    S3_REQUIRE(p != nullptr && aligned16(p), S3_ERR_INVALID_ARG, "%s is null or misaligned", what);
    S3_REQUIRE(ld % 8 == 0 && ld >= static_cast<int64_t>(heads) * dim, S3_ERR_INVALID_ARG,
               "%s: row pitch %lld must be a multiple of 8 and at least %d", what, (long long)ld, heads * dim);
    S3_REQUIRE(ld < (int64_t(1) << 38), S3_ERR_UNSUPPORTED, "%s: row pitch %lld is too large", what, (long long)ld);
    return S3_OK;
}

s3_status check_workspace(const void* d_ws, size_t ws_bytes)
{
    S3_REQUIRE(d_ws != nullptr && ws_bytes >= S3_WS_HEADER_BYTES, S3_ERR_CAPACITY, "workspace missing or smaller than %d bytes", S3_WS_HEADER_BYTES);
    S3_REQUIRE(aligned16(d_ws), S3_ERR_INVALID_ARG, "d_ws must be 16-byte aligned");
    return S3_OK;
}

#define S3_TRY(expr)                      \
    do {                                  \
        const s3_status st__ = (expr);    \
        if (st__ != S3_OK) return st__;   \
    } while (0)

KvBatchDev device_batch(const s3_kv_batch& b)
{
    return KvBatchDev{b.d_cu_q, b.d_kv_len, b.d_pages, b.ld_pages, b.n_seqs, b.T, b.max_q, b.max_kv};
}

s3_status attention(const s3_kv_cache* cache, const s3_kv_batch* batch, const void* d_q, int64_t ldq, int n_heads,
                    const int32_t* d_blocks, int s, int list_heads, int list_mode, const s3_attn_params* params, const s3_score_form* form,
                    void* d_out, int64_t ld_out, float* d_lse, void* d_ws, size_t ws_bytes, void* stream)
{
    S3_TRY(check_batch(cache, batch));
    S3_TRY(check_heads(n_heads, cache->st.d.n_kv_heads));
    S3_REQUIRE(params != nullptr, S3_ERR_INVALID_ARG, "params is null");
    S3_REQUIRE(isfinite(params->scale) && params->scale > 0.0f, S3_ERR_INVALID_ARG, "scale must be positive and finite");
    S3_REQUIRE(params->window >= 0, S3_ERR_INVALID_ARG, "window = %d is negative", params->window);
    const s3_score_form f = form ? *form : s3_score_form{};
    S3_REQUIRE(isfinite(f.cap) && f.cap >= 0.0f, S3_ERR_INVALID_ARG, "cap must be finite and not negative");
    // the cap enters as scale / cap and as cap log2(e), which have to be numbers other than 0 and infinity
    S3_REQUIRE(f.cap == 0.0f || (f.cap >= 1e-6f && f.cap <= 1e30f && params->scale / f.cap >= 1e-30f && params->scale / f.cap <= 1e30f), S3_ERR_UNSUPPORTED,
               "cap = %g out of range for scale = %g", f.cap, params->scale);
    S3_REQUIRE(aligned4(f.d_slopes) && aligned4(f.d_prefix), S3_ERR_INVALID_ARG, "d_slopes or d_prefix is misaligned");
    const KvCacheState& c = cache->st;
    const s3_kv_batch& b = *batch;
    if (b.T == 0 || b.n_seqs == 0) return S3_OK;
    S3_TRY(check_rows("d_q", d_q, ldq, n_heads, c.d.head_dim));
    S3_TRY(check_rows("d_out", d_out, ld_out, n_heads, c.d.head_dim));
    S3_REQUIRE(aligned4(d_blocks) && aligned4(d_lse), S3_ERR_INVALID_ARG, "d_blocks or d_lse is misaligned");
    S3_TRY(check_workspace(d_ws, ws_bytes));
    const int group = n_heads / c.d.n_kv_heads;
    const AttnPlan p = plan_attention(b, PlanShape{device_sm_count(), group, c.d.n_kv_heads, c.page_shift, held_bytes(c.d.head_dim, c.k_scale != nullptr), c.k_scale != nullptr}, list_mode,
                                      list_mode == LIST_NONE ? b.max_kv : static_cast<int64_t>(s) << c.page_shift);

    AttnArgs a;
    memset(&a, 0, sizeof(a));
    a.b = device_batch(b);
    a.n_heads = n_heads;
    a.n_kv_heads = c.d.n_kv_heads;
    a.group = group;
    a.page_size = c.d.page_size;
    a.page_shift = c.page_shift;
    a.box_rows = c.box_rows;
    a.n_pages = c.d.n_pages;
    a.head_dim = c.d.head_dim;
    a.scale_log2 = params->scale * kLog2e;
    a.causal = params->causal != 0;
    a.window = params->window < b.max_kv ? params->window : 0;         // a window that holds every position hides none
    a.cap2 = f.cap * kLog2e;
    a.score_in = f.cap > 0.0f ? params->scale / f.cap : a.scale_log2;
    a.slopes = f.d_slopes;
    a.prefix = a.causal ? f.d_prefix : nullptr;                        // every row sees everything otherwise
    a.k_scale = c.k_scale;
    a.v_scale = c.v_scale;
    a.lists = d_blocks;
    a.s = s;
    a.list_heads = list_heads;
    a.list_mode = list_mode;
    a.q = d_q;
    a.ldq = ldq;
    a.out = d_out;
    a.ld_out = ld_out;
    a.lse = d_lse;
    a.tok_per_item = p.tok_per_item;
    a.n_items = p.n_items;
    a.one_item_per_seq = p.one_item_per_seq;
    a.status = static_cast<uint32_t*>(d_ws);
    // a byte per block of the tile kernel, between the status block and the pieces
    a.redo = ws_bytes >= 256 && p.grid <= 256 - S3_WS_HEADER_BYTES ? static_cast<uint8_t*>(d_ws) + S3_WS_HEADER_BYTES : nullptr;

    a.grid = p.grid;
    a.share_min = p.share_min;
    a.whole_rounds = p.whole_rounds;
    a.rows_cap = p.rows_cap;
    const size_t partial = partial_bytes(p, c.d.head_dim), need = 256 + partial + (p.masked ? mask_bytes(b, c.page_shift, list_heads, p.tok_per_item) : 0);
    S3_REQUIRE((p.share_min == 0 && !p.masked) || ws_bytes >= need, S3_ERR_CAPACITY, "workspace holds %zu bytes, %zu needed", ws_bytes, need);
    if (p.share_min > 0) {
        const size_t rows = 2 * static_cast<size_t>(p.grid) * p.rows_cap;
        a.part_o = reinterpret_cast<float*>(static_cast<unsigned char*>(d_ws) + 256);
        a.part_lse = reinterpret_cast<float*>(static_cast<unsigned char*>(d_ws) + 256 + round_up(rows * c.d.head_dim * 4, 256));
        a.cuts = reinterpret_cast<int32_t*>(reinterpret_cast<unsigned char*>(a.part_lse) + round_up(rows * 4, 256));
    }
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (p.masked) {
        unsigned char* at = static_cast<unsigned char*>(d_ws) + 256 + partial;
        a.mask_words = mask_words(b, c.page_shift);
        a.masks = reinterpret_cast<uint32_t*>(at);
        a.unions = reinterpret_cast<uint32_t*>(at + round_up(static_cast<size_t>(b.T) * list_heads * a.mask_words * 4, 256));
        a.list_mode = LIST_NONE;
        S3_TRY(launch_attn_masks(a, st));
    }
    S3_TRY(p.tile ? launch_attn_tile(c, a, st) : launch_attn_split(c, a, st));
    return p.share_min > 0 && p.grid > 1 ? launch_attn_join(c, a, p.tile, st) : S3_OK;
}

s3_status create_cache(s3_kv_cache** out, const s3_kv_cache_desc* desc, bool i8, float* d_k_scale, float* d_v_scale)
{
    S3_REQUIRE(out != nullptr, S3_ERR_INVALID_ARG, "out is null");
    *out = nullptr;
    S3_REQUIRE(desc != nullptr, S3_ERR_INVALID_ARG, "desc is null");
    const s3_kv_cache_desc& d = *desc;
    S3_REQUIRE(d.d_k && d.d_v && aligned16(d.d_k) && aligned16(d.d_v), S3_ERR_INVALID_ARG, "key or value pages are null or misaligned");
    S3_REQUIRE((d.d_code != nullptr) == (d.d_scale != nullptr), S3_ERR_INVALID_ARG, "summaries need codes and scales");
    S3_REQUIRE(aligned16(d.d_code) && aligned16(d.d_scale), S3_ERR_INVALID_ARG, "summary arrays must be 16-byte aligned");
    S3_REQUIRE(!i8 || (d_k_scale && d_v_scale && aligned16(d_k_scale) && aligned16(d_v_scale)), S3_ERR_INVALID_ARG, "scales are null or misaligned");
    S3_REQUIRE(d.dtype == S3_BF16 || d.dtype == S3_F16, S3_ERR_UNSUPPORTED, "a cache's rows are bf16 or f16 (got dtype %d)", (int)d.dtype);
    S3_REQUIRE(d.n_pages >= 1 && d.n_kv_heads >= 1 && d.n_kv_heads <= 65535, S3_ERR_INVALID_ARG, "n_pages = %d, n_kv_heads = %d out of range",
               d.n_pages, d.n_kv_heads);
    S3_REQUIRE(d.head_dim == 64 || d.head_dim == 128, S3_ERR_UNSUPPORTED, "head_dim = %d (64 or 128)", d.head_dim);
    S3_REQUIRE(d.page_size == 16 || d.page_size == 32 || d.page_size == 64 || d.page_size == 128, S3_ERR_UNSUPPORTED,
               "page_size = %d (16, 32, 64 or 128)", d.page_size);
    const int64_t page = static_cast<int64_t>(d.n_kv_heads) * d.page_size * d.head_dim;
    const int unit = i8 ? 16 : 8;                                      // elements in 16 bytes
    S3_REQUIRE(d.k_page_stride >= page && d.v_page_stride >= page && d.k_page_stride % unit == 0 && d.v_page_stride % unit == 0, S3_ERR_INVALID_ARG,
               "page strides %lld, %lld must be multiples of %d and at least %lld", (long long)d.k_page_stride, (long long)d.v_page_stride, unit,
               (long long)page);
    S3_REQUIRE(d.k_page_stride < (int64_t(1) << 38) && d.v_page_stride < (int64_t(1) << 38), S3_ERR_UNSUPPORTED, "page stride too large");
    int n_dev = 0;
    S3_CUDA_TRY(cudaGetDeviceCount(&n_dev));
    S3_REQUIRE(device_cc_major() == 10, S3_ERR_UNSUPPORTED, "this library runs on sm_100 devices only (found compute capability %d.x)",
               device_cc_major());
    s3_kv_cache* c = new (std::nothrow) s3_kv_cache;
    S3_REQUIRE(c != nullptr, S3_ERR_NOMEM, "out of host memory");
    c->st.d = d;
    c->st.page_shift = shift_of(d.page_size);
    c->st.box_rows = d.page_size < 64 ? d.page_size : 64;
    const uint64_t D = d.head_dim, P = d.page_size;
    const uint64_t K = d.n_kv_heads, N = d.n_pages, ks = d.k_page_stride, vs = d.v_page_stride, half = 64;
    const uint32_t rows = c->st.box_rows;
    const uint64_t dims[4] = {D, P, K, N}, ks4[3] = {D, D * P, ks}, vs4[3] = {D, D * P, vs};
    const uint32_t box[4] = {i8 ? static_cast<uint32_t>(d.head_dim) : 64, rows, 1, 1};
    const uint64_t wide[5] = {64, P, D / 64, K, N}, ks5[4] = {D, half, D * P, ks}, vs5[4] = {D, half, D * P, vs};
    const uint32_t wide_box[5] = {64, rows, static_cast<uint32_t>(d.head_dim / 64), 1, 1};
    c->st.k_scale = d_k_scale;
    c->st.v_scale = d_v_scale;
    const CUtensorMapDataType type = i8 ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : map_type(d.dtype);
    s3_status st = make_map<4>(c->st.map_k, type, d.d_k, dims, ks4, box);
    if (st == S3_OK) st = make_map<4>(c->st.map_v, type, d.d_v, dims, vs4, box);
    if (st == S3_OK && !i8) st = make_map<5>(c->st.wide_k, type, d.d_k, wide, ks5, wide_box);
    if (st == S3_OK && !i8) st = make_map<5>(c->st.wide_v, type, d.d_v, wide, vs5, wide_box);
    if (st != S3_OK) {
        delete c;
        return st;
    }
    *out = c;
    return S3_OK;
}

// An append's arguments; also those of its form with norms.
s3_status append(const s3_kv_cache* cache, const s3_kv_batch* batch, const s3_head_norm* norm, const s3_rope* rope, const int32_t* d_positions,
                 const void* d_q, int64_t ldq, int n_heads, void* d_q_out, int64_t ld_qo, const void* d_k, int64_t ldk,
                 const void* d_v, int64_t ldv, void* d_ws, size_t ws_bytes, void* stream)
{
    S3_TRY(check_batch(cache, batch));
    const KvCacheState& c = cache->st;
    if (rope) {
        S3_REQUIRE(rope->rot_dim >= 0 && rope->rot_dim <= c.d.head_dim, S3_ERR_INVALID_ARG, "rot_dim = %d out of [0, %d]", rope->rot_dim, c.d.head_dim);
        S3_REQUIRE(rope->rot_dim % 16 == 0, S3_ERR_UNSUPPORTED, "rot_dim = %d must be a multiple of 16", rope->rot_dim);
        if (rope->rot_dim > 0) {
            S3_REQUIRE(rope->d_cos && rope->d_sin && aligned16(rope->d_cos) && aligned16(rope->d_sin), S3_ERR_INVALID_ARG,
                       "rotation tables are null or misaligned");
            S3_REQUIRE(rope->n_pos >= 1, S3_ERR_INVALID_ARG, "the rotation tables are empty");
        }
    }
    if (norm) {
        S3_REQUIRE(isfinite(norm->eps) && norm->eps > 0.0f, S3_ERR_INVALID_ARG, "eps must be positive and finite");
        S3_REQUIRE(aligned16(norm->d_q_weight) && aligned16(norm->d_k_weight), S3_ERR_INVALID_ARG, "the norm's weights must be 16-byte aligned");
    }
    if (d_q) S3_TRY(check_heads(n_heads, cache->st.d.n_kv_heads));
    if (batch->T == 0 || batch->n_seqs == 0) return S3_OK;
    if (d_q) {
        S3_TRY(check_rows("d_q", d_q, ldq, n_heads, c.d.head_dim));
        S3_TRY(check_rows("d_q_out", d_q_out, ld_qo, n_heads, c.d.head_dim));
    }
    S3_TRY(check_rows("d_k", d_k, ldk, c.d.n_kv_heads, c.d.head_dim));
    S3_TRY(check_rows("d_v", d_v, ldv, c.d.n_kv_heads, c.d.head_dim));
    S3_REQUIRE(aligned4(d_positions), S3_ERR_INVALID_ARG, "d_positions is misaligned");
    S3_TRY(check_workspace(d_ws, ws_bytes));
    // the plain append has a kernel of its own: its bits are those of the rotation alone, and it needs fewer registers
    if (c.k_scale || (norm && ((d_q && norm->d_q_weight) || norm->d_k_weight)))
        return launch_kv_append_norm(c, device_batch(*batch), norm, rope, d_positions, d_q, ldq, n_heads, d_q_out, ld_qo, d_k, ldk, d_v, ldv,
                                     static_cast<uint32_t*>(d_ws), static_cast<cudaStream_t>(stream));
    return launch_kv_append(c, device_batch(*batch), rope, d_positions, d_q, ldq, n_heads, d_q_out, ld_qo, d_k, ldk, d_v, ldv,
                            static_cast<uint32_t*>(d_ws), static_cast<cudaStream_t>(stream));
}

}  // namespace

extern "C" {

s3_status s3_kv_cache_create(s3_kv_cache** out, const s3_kv_cache_desc* desc) { return create_cache(out, desc, false, nullptr, nullptr); }

s3_status s3_kv_cache_create_i8(s3_kv_cache** out, const s3_kv_cache_desc* desc, float* d_k_scale, float* d_v_scale)
{
    return create_cache(out, desc, true, d_k_scale, d_v_scale);
}

s3_status s3_kv_cache_destroy(s3_kv_cache* cache)
{
    delete cache;
    return S3_OK;
}

size_t s3_kv_workspace_bytes(const s3_kv_cache* cache, const s3_kv_batch* batch, int n_heads)
{
    if (check_batch(cache, batch) != S3_OK || check_heads(n_heads, cache->st.d.n_kv_heads) != S3_OK) return 0;
    size_t most = 0;
    if (batch->T > 0 && batch->n_seqs > 0)
        // every call uses at most one of these: the tile kernel's pieces of two query tiles or one, the split kernel's
        for (int tile = 0; tile < 2; ++tile) {
            AttnPlan p;
            p.grid = (tile ? 1 : 2) * device_sm_count();
            p.share_min = 1;
            const int group = n_heads / cache->st.d.n_kv_heads, one = kTileRows / group;
            if (tile && static_cast<int64_t>(batch->max_q) * group <= kSplitRows && group <= kSplitRows) continue;
            p.rows_cap = tile ? (batch->max_q > one ? 2 * one : one) * group : kSplitRows;
            const size_t bytes = partial_bytes(p, cache->st.d.head_dim);
            if (bytes > most) most = bytes;
        }
    return 256 + most + (batch->T > 0 && batch->n_seqs > 0 ? mask_bytes(*batch, cache->st.page_shift, cache->st.d.n_kv_heads, kTileRows * cache->st.d.n_kv_heads / n_heads) : 0);
}

s3_status s3_attn_plan_describe(const s3_kv_batch* batch, int n_heads, int n_kv_heads, int head_dim, int page_size, int s, int per_token,
                                int n_sms, s3_attn_plan* out)
{
    S3_REQUIRE(batch != nullptr && out != nullptr, S3_ERR_INVALID_ARG, "batch or out is null");
    S3_REQUIRE(n_kv_heads >= 1 && n_sms >= 1 && s >= 0, S3_ERR_INVALID_ARG, "n_kv_heads = %d, n_sms = %d, s = %d out of range", n_kv_heads, n_sms, s);
    S3_TRY(check_heads(n_heads, n_kv_heads));
    S3_REQUIRE(s <= S3_MAX_BLOCK_LIST, S3_ERR_UNSUPPORTED, "s = %d exceeds %d", s, S3_MAX_BLOCK_LIST);
    S3_REQUIRE(head_dim == 64 || head_dim == 128, S3_ERR_UNSUPPORTED, "head_dim = %d (64 or 128)", head_dim);
    S3_REQUIRE(page_size == 16 || page_size == 32 || page_size == 64 || page_size == 128, S3_ERR_UNSUPPORTED, "page_size = %d (16, 32, 64 or 128)", page_size);
    S3_REQUIRE(batch->n_seqs >= 1 && batch->max_q >= 1 && batch->max_q <= batch->T && batch->max_kv >= 0, S3_ERR_INVALID_ARG,
               "n_seqs = %d, T = %d, max_q = %d, max_kv = %d out of range", batch->n_seqs, batch->T, batch->max_q, batch->max_kv);
    const int shift = shift_of(page_size), mode = s == 0 ? LIST_NONE : per_token ? LIST_PER_TOKEN : LIST_PER_SEQ;
    const AttnPlan p = plan_attention(*batch, PlanShape{n_sms, n_heads / n_kv_heads, n_kv_heads, shift, held_bytes(head_dim, false), false}, mode,
                                      s == 0 ? batch->max_kv : static_cast<int64_t>(s) << shift);
    *out = s3_attn_plan{p.tile, p.masked, p.tok_per_item, p.n_items, p.grid, p.share_min > 0, p.whole_rounds, 0};
    return S3_OK;
}

s3_status s3_kv_append(const s3_kv_cache* cache, const s3_kv_batch* batch, const s3_rope* rope, const int32_t* d_positions,
                       const void* d_q, int64_t ldq, int n_heads, void* d_q_out, int64_t ld_qo, const void* d_k, int64_t ldk,
                       const void* d_v, int64_t ldv, void* d_ws, size_t ws_bytes, void* stream)
{
    return append(cache, batch, nullptr, rope, d_positions, d_q, ldq, n_heads, d_q_out, ld_qo, d_k, ldk, d_v, ldv, d_ws, ws_bytes, stream);
}

s3_status s3_kv_append_norm(const s3_kv_cache* cache, const s3_kv_batch* batch, const s3_head_norm* norm, const s3_rope* rope,
                            const int32_t* d_positions, const void* d_q, int64_t ldq, int n_heads, void* d_q_out, int64_t ld_qo,
                            const void* d_k, int64_t ldk, const void* d_v, int64_t ldv, void* d_ws, size_t ws_bytes, void* stream)
{
    return append(cache, batch, norm, rope, d_positions, d_q, ldq, n_heads, d_q_out, ld_qo, d_k, ldk, d_v, ldv, d_ws, ws_bytes, stream);
}

s3_status s3_kv_read(const s3_kv_cache* cache, const s3_kv_batch* batch, void* d_k, int64_t ldk, void* d_v, int64_t ldv, void* d_ws, size_t ws_bytes,
                     void* stream)
{
    S3_TRY(check_batch(cache, batch));
    const KvCacheState& c = cache->st;
    S3_REQUIRE(d_k != nullptr || d_v != nullptr || batch->T == 0 || batch->n_seqs == 0, S3_ERR_INVALID_ARG, "d_k and d_v are null");
    if (batch->T == 0 || batch->n_seqs == 0) return S3_OK;
    if (d_k) S3_TRY(check_rows("d_k", d_k, ldk, c.d.n_kv_heads, c.d.head_dim));
    if (d_v) S3_TRY(check_rows("d_v", d_v, ldv, c.d.n_kv_heads, c.d.head_dim));
    S3_TRY(check_workspace(d_ws, ws_bytes));
    return launch_kv_read(c, device_batch(*batch), d_k, ldk, d_v, ldv, static_cast<uint32_t*>(d_ws), static_cast<cudaStream_t>(stream));
}

s3_status s3_block_select(const s3_kv_cache* cache, const s3_kv_batch* batch, const void* d_q, int64_t ldq, int n_heads, int s,
                          int n_first, int n_last, int32_t* d_blocks, void* d_ws, size_t ws_bytes, void* stream)
{
    S3_TRY(check_batch(cache, batch));
    S3_TRY(check_heads(n_heads, cache->st.d.n_kv_heads));
    const KvCacheState& c = cache->st;
    S3_REQUIRE(c.d.d_code != nullptr, S3_ERR_STATE, "the cache was created without summaries");
    S3_REQUIRE(s >= 1 && n_first >= 0 && n_last >= 0, S3_ERR_INVALID_ARG, "s = %d, n_first = %d, n_last = %d out of range", s, n_first, n_last);
    S3_REQUIRE(s <= S3_MAX_SELECT, S3_ERR_UNSUPPORTED, "s = %d exceeds %d", s, S3_MAX_SELECT);
    S3_REQUIRE(n_first <= s && n_last <= s && n_first + n_last <= s, S3_ERR_INVALID_ARG, "n_first + n_last exceeds s = %d", s);
    S3_REQUIRE(batch->max_kv <= static_cast<int64_t>(S3_MAX_SELECT_BLOCKS) * c.d.page_size, S3_ERR_UNSUPPORTED, "max_kv = %d exceeds %d blocks",
               batch->max_kv, S3_MAX_SELECT_BLOCKS);
    if (batch->T == 0 || batch->n_seqs == 0) return S3_OK;
    S3_TRY(check_rows("d_q", d_q, ldq, n_heads, c.d.head_dim));
    S3_REQUIRE(d_blocks != nullptr && aligned4(d_blocks), S3_ERR_INVALID_ARG, "d_blocks is null or misaligned");
    S3_TRY(check_workspace(d_ws, ws_bytes));
    return launch_block_select(c, device_batch(*batch), d_q, ldq, n_heads, s, n_first, n_last, d_blocks, static_cast<uint32_t*>(d_ws),
                               static_cast<cudaStream_t>(stream));
}

s3_status s3_paged_attention(const s3_kv_cache* cache, const s3_kv_batch* batch, const void* d_q, int64_t ldq, int n_heads,
                             const s3_attn_params* params, void* d_out, int64_t ld_out, float* d_lse, void* d_ws, size_t ws_bytes, void* stream)
{
    return attention(cache, batch, d_q, ldq, n_heads, nullptr, 0, 1, LIST_NONE, params, nullptr, d_out, ld_out, d_lse, d_ws, ws_bytes, stream);
}

s3_status s3_paged_attention_scored(const s3_kv_cache* cache, const s3_kv_batch* batch, const void* d_q, int64_t ldq, int n_heads,
                                    const s3_attn_params* params, const s3_score_form* form, void* d_out, int64_t ld_out, float* d_lse,
                                    void* d_ws, size_t ws_bytes, void* stream)
{
    S3_REQUIRE(form != nullptr, S3_ERR_INVALID_ARG, "form is null");
    return attention(cache, batch, d_q, ldq, n_heads, nullptr, 0, 1, LIST_NONE, params, form, d_out, ld_out, d_lse, d_ws, ws_bytes, stream);
}

s3_status s3_block_attention(const s3_kv_cache* cache, const s3_kv_batch* batch, const void* d_q, int64_t ldq, int n_heads,
                             const int32_t* d_blocks, int s, int list_heads, int per_token, const s3_attn_params* params, void* d_out,
                             int64_t ld_out, float* d_lse, void* d_ws, size_t ws_bytes, void* stream)
{
    S3_REQUIRE(cache != nullptr, S3_ERR_INVALID_ARG, "cache is null");
    S3_REQUIRE(s >= 1, S3_ERR_INVALID_ARG, "s = %d out of range", s);
    S3_REQUIRE(s <= S3_MAX_BLOCK_LIST, S3_ERR_UNSUPPORTED, "s = %d exceeds %d", s, S3_MAX_BLOCK_LIST);
    S3_REQUIRE(list_heads == 1 || list_heads == cache->st.d.n_kv_heads, S3_ERR_INVALID_ARG, "list_heads = %d (1 or %d)", list_heads,
               cache->st.d.n_kv_heads);
    S3_REQUIRE(d_blocks != nullptr || (batch && (batch->T == 0 || batch->n_seqs == 0)), S3_ERR_INVALID_ARG, "d_blocks is null");
    return attention(cache, batch, d_q, ldq, n_heads, d_blocks, s, list_heads, per_token ? LIST_PER_TOKEN : LIST_PER_SEQ, params, nullptr, d_out, ld_out,
                     d_lse, d_ws, ws_bytes, stream);
}

}  // extern "C"
