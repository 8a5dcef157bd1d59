// dd_cached_attention: queries over a paged cache of e4m3 keys and values.
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <cmath>
#include <mutex>
#include <type_traits>

#include "dd_common.cuh"
#include "dd_ptx.cuh"

namespace {

using namespace ddptx;

constexpr int kTileKeys = 128, kTileRows = 128;     // keys of a chunk, the wide kernel's query rows

struct CachedParams {
    const __nv_bfloat16 *q;
    __nv_bfloat16 *out;
    dd_strides qs, os;
    const int32_t *table, *kv_len;
    const float *scale[2];                  // of the keys', of the values' pages
    float *ws;
    unsigned int *status, *mirror;
    int B, Hkv, G, Nq, rows, row_tiles;     // G query heads read a key head; rows = G * Nq
    int num_pages, max_pages, page, page_log2;
    float scale_log2;
    int ctas;                               // at most
    int tile_rows, part_rows;               // query rows of an item, of a part in the workspace
};

__device__ __forceinline__ void report(const CachedParams &p, unsigned code)
{
    if (atomicCAS(p.status, 0u, code) == 0u && p.mirror) {
        *reinterpret_cast<volatile unsigned int *>(p.mirror) = code;
        __threadfence_system();
    }
}

__device__ __forceinline__ int keys_of(const CachedParams &p, int b)
{
    return max(0, min(p.kv_len[b], p.max_pages << p.page_log2));
}
__device__ __forceinline__ int tiles_of(int keys) { return (int)(((unsigned)keys + kTileKeys - 1) / kTileKeys); }
__device__ __forceinline__ int chunks_of(const CachedParams &p, int b) { return tiles_of(keys_of(p, b)); }

// A part of an item in the workspace: its rows in fp32 (from cached_attention_wide_kernel four columns of every row together, which is how
// its threads have them), then (reference, sum) of each row.  A CTA has two places: for the part of the item that
// its share begins in the middle of, and for that of an item whose beginning it has.
template <int D>
__host__ __device__ constexpr size_t part_floats(int rows) { return (size_t)rows * D + 2 * rows; }
template <int D>
__device__ __forceinline__ float *part_of(const CachedParams &p, unsigned cta, bool from_start)
{
    return p.ws + (2 * (size_t)cta + from_start) * part_floats<D>(p.part_rows);
}

// Four e4m3 numbers to two pairs of f16 (exact).
__device__ __forceinline__ void e4m3_to_f16(uint32_t v, uint32_t &lo, uint32_t &hi)
{
    asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, l;\n\tcvt.rn.f16x2.e4m3x2 %1, h;\n\t}"
        : "=r"(lo), "=r"(hi) : "r"(v));
}
// The nearest e4m3 numbers to four values (the first in the lowest byte); the values become what is left of them.
__device__ __forceinline__ uint32_t split_e4m3(float (&v)[4])
{
    uint32_t w, lo, hi;
    asm("{\n\t.reg .b16 l, h;\n\tcvt.rn.satfinite.e4m3x2.f32 l, %2, %1;\n\tcvt.rn.satfinite.e4m3x2.f32 h, %4, %3;\n\tmov.b32 %0, {l, h};\n\t}"
        : "=r"(w) : "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]));
    e4m3_to_f16(w, lo, hi);
    const float2 a = __half22float2(*reinterpret_cast<__half2 *>(&lo)), b = __half22float2(*reinterpret_cast<__half2 *>(&hi));
    v[0] -= a.x; v[1] -= a.y; v[2] -= b.x; v[3] -= b.y;
    return w;
}
// A row's 16-byte piece c in a slot (the copies' swizzle: 128 bytes for D = 128, 64 bytes for D = 64).
template <int D>
__device__ __forceinline__ int piece(int row, int c)
{
    return D == 128 ? row * 128 + ((c ^ (row & 7)) << 4) : row * 64 + ((c ^ ((row >> 1) & 3)) << 4);
}
__device__ __forceinline__ float power_of_two(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }
__device__ __forceinline__ uint32_t half2_bits(float a, float b)
{
    __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<uint32_t *>(&h);
}

// How the chunks of all items (in order, an item's in the keys' order) are shared out, found by each warp for itself, no barrier.
// Shares of equal cost, across items, where an item costs its chunks and kEnds more at its front for its start and end.
// 16 x 32 heads, 32 queries over up to 1024 keys (CTAs with one to four items) 45 us without that cost, 36 with it; of 1, 2 and 3 the best was 2.
// Where tiles are no more than CTAs, that cost leaves some CTAs without a tile and others with two (51 of 256 each for 32 items of 8 tiles).
// (Items cut into parts of equal length, a CTA each, where that makes none longer: 0.2 us less for one shape, 0.3 to 4 more for fourteen others.)
struct Split {
    static constexpr unsigned kEnds = 2;
    unsigned n, each, more;                 // CTAs at work; the first `more` shares are of `each` + 1, the others of `each`

    __device__ __forceinline__ Split(const CachedParams &p, int lane)
    {
        const unsigned heads = (unsigned)p.Hkv * p.row_tiles;
        unsigned chunks = 0, items = 0;
        for (int i = lane; i < p.B; i += 32) {
            const unsigned c = chunks_of(p, i);
            chunks += c;
            items += c > 0;
        }
        chunks = __reduce_add_sync(0xFFFFFFFFu, chunks) * heads;
        items = __reduce_add_sync(0xFFFFFFFFu, items) * heads;
        n = min(chunks, (unsigned)p.ctas);
        if (n == 0) { each = more = 0; return; }
        const unsigned cost = chunks + items * kEnds;
        each = cost / n;
        more = cost - each * n;
    }

    // of an item of a sequence of this many chunks
    __device__ __forceinline__ unsigned weight(unsigned chunks) const { return chunks ? chunks + kEnds : 0; }
    __device__ __forceinline__ unsigned first(unsigned cta) const { return cta * each + min(cta, more); }
    __device__ __forceinline__ unsigned cta_of(unsigned u) const
    {
        const unsigned head = more * (each + 1);
        return u < head ? u / (each + 1) : more + (u - head) / each;
    }
};

// Where a warp is in its CTA's share: chunk c of item (b, h, row tile), whose part here ends at `end`.
struct Cursor {
    int b, h, rt, c, c0, end, n, keys;      // c0: where the part begins; n, keys: chunks and keys of sequence b
    unsigned left;                          // what the share has behind this item, if that gives it any chunk
    // (cost) the part of the item that begins `at` into it and takes what is left of the share
    __device__ __forceinline__ void enter(unsigned at, unsigned share)
    {
        const unsigned take = min(share, n + Split::kEnds - at), to = at + take;
        c = c0 = at > Split::kEnds ? at - Split::kEnds : 0;
        end = to > Split::kEnds ? to - Split::kEnds : 0;
        left = share - take > Split::kEnds ? share - take : 0;
    }
    __device__ __forceinline__ void next(const CachedParams &p)        // (only where something is left)
    {
        if (++rt == p.row_tiles) {
            rt = 0;
            if (++h == p.Hkv) {
                h = 0;
                do ++b; while (b < p.B && (keys = keys_of(p, b)) == 0);
                n = tiles_of(keys);
            }
        }
        enter(0, left);
    }
};

// What the join has to know of a CTA: how many parts the item has whose first part it left behind (0: none).
struct Record {
    int parts, b, h, rt;
};
template <int D>
__device__ __forceinline__ Record *record_of(const CachedParams &p, unsigned cta)
{
    return reinterpret_cast<Record *>(p.ws + 2 * (size_t)p.ctas * part_floats<D>(p.part_rows)) + cta;
}

// This CTA's share: `now` is its first part.  False: there is nothing for it to do.
__device__ __forceinline__ bool find_share(const CachedParams &p, int lane, const Split &split, Cursor &now)
{
    if (blockIdx.x >= split.n) return false;
    const unsigned heads = (unsigned)p.Hkv * p.row_tiles, u0 = split.first(blockIdx.x), u1 = split.first(blockIdx.x + 1);
    unsigned before = 0;                    // weights of the sequences before, times heads
    for (int b0 = 0; b0 < p.B; b0 += 32) {
        const int keys = b0 + lane < p.B ? keys_of(p, b0 + lane) : 0;
        const unsigned n = tiles_of(keys), weight = split.weight(n);
        unsigned sum = weight;
#pragma unroll
        for (int o = 1; o < 32; o *= 2) {
            const unsigned v = __shfl_up_sync(0xFFFFFFFFu, sum, o);
            if (lane >= o) sum += v;
        }
        const unsigned past = __ballot_sync(0xFFFFFFFFu, u0 < before + sum * heads);
        if (past) {
            const int at = __ffs(past) - 1;
            now.b = b0 + at;
            now.n = __shfl_sync(0xFFFFFFFFu, n, at);
            now.keys = __shfl_sync(0xFFFFFFFFu, keys, at);
            const unsigned w = __shfl_sync(0xFFFFFFFFu, weight, at);
            const unsigned in = u0 - (before + (__shfl_sync(0xFFFFFFFFu, sum, at) - w) * heads), item = in / w, rest = in - item * w;
            now.h = p.row_tiles == 1 ? item : item / p.row_tiles;
            now.rt = item - now.h * p.row_tiles;
            now.enter(rest, u1 - u0);
            return now.c < now.end;         // (a share may lie in an item's start alone)
        }
        before += __shfl_sync(0xFFFFFFFFu, sum, 31) * heads;
    }
    return false;
}

// By one lane, of the CTA's last item.
template <int D>
__device__ __forceinline__ void write_record(const CachedParams &p, const Split &split, const Cursor &last, bool work)
{
    int parts = 0;
    if (work && last.c0 == 0 && last.end < last.n)
        parts = split.cta_of(split.first(blockIdx.x + 1) - 1 + (last.n - last.end)) - blockIdx.x + 1;
    *reinterpret_cast<int4 *>(record_of<D>(p, blockIdx.x)) = make_int4(parts, last.b, last.h, last.rt);
}

// Sequences without a key: zeros, by all threads of CTAs b, b + CTAs, ...
template <int D>
__device__ __forceinline__ void clear_empty(const CachedParams &p)
{
    for (int b = blockIdx.x; b < p.B; b += gridDim.x) {
        if (keys_of(p, b) > 0) continue;
        const long pieces = (long)p.Nq * p.G * p.Hkv * (D / 8);
        for (long i = threadIdx.x; i < pieces; i += blockDim.x) {
            const long row = i / (D / 8), iq = row / (p.G * p.Hkv), h = row - iq * (p.G * p.Hkv);
            reinterpret_cast<uint4 *>(p.out + (b * p.os.batch + iq * p.os.token + h * p.os.head))[i % (D / 8)] = make_uint4(0u, 0u, 0u, 0u);
        }
    }
}

// Items whose chunks lie in several CTAs: their parts are weighted and added, in the keys' order, 16 rows a CTA; CTA x of the grid's first
// dimension joins the item whose first part CTA x of the kernel before left behind.  (A CTA for every item, which found out for itself
// whether and where the item was cut, took 4 to 9 us of a call.)
// What it costs is the latency of reads that wait for one another, so the reference points and rows of eight parts are on their way together
// (part after part, 128 rows of ten parts each took some 12 us).
template <int D>
__global__ void __launch_bounds__(16 * D / 8) cached_attention_join_kernel(const CachedParams p)
{
    constexpr int kBatch = 8;
    grid_trigger();
    grid_wait();
    const int4 record = *reinterpret_cast<const int4 *>(record_of<D>(p, blockIdx.x));
    const bool by_row = p.tile_rows < 128;  // how the part's kernel left it
    const int tid = threadIdx.x, r = by_row ? tid / (D / 8) : tid % 16, c8 = by_row ? tid % (D / 8) : tid / 16, row = blockIdx.y * 16 + r;
    const int parts = record.x, b = record.y, h = record.z, rt = record.w;
    if (parts == 0 || row >= min(p.tile_rows, p.rows - rt * p.tile_rows)) return;
    const unsigned i0 = blockIdx.x;
    const size_t from = by_row ? row * (D / 4) + 2 * c8 : (size_t)2 * c8 * p.part_rows + row, behind = by_row ? 1 : p.part_rows;
    float top = -INFINITY, sum = 0.f, v[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = 0.f;
    for (int k0 = 0; k0 < parts; k0 += kBatch) {
        float2 ml[kBatch];
        float4 x[kBatch][2];
#pragma unroll
        for (int k = 0; k < kBatch; ++k) {
            ml[k] = make_float2(-INFINITY, 0.f);
            x[k][0] = x[k][1] = make_float4(0.f, 0.f, 0.f, 0.f);
            if (k0 + k < parts) {
                const float *part = part_of<D>(p, i0 + k0 + k, k0 + k == 0);
                ml[k] = *reinterpret_cast<const float2 *>(part + p.part_rows * D + 2 * row);
                x[k][0] = reinterpret_cast<const float4 *>(part)[from];
                x[k][1] = reinterpret_cast<const float4 *>(part)[from + behind];
            }
        }
        float now = top;
#pragma unroll
        for (int k = 0; k < kBatch; ++k) now = fmaxf(now, ml[k].x);
        const float old = top == -INFINITY ? 0.f : ex2(top - now);
        top = now;
        sum *= old;
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] *= old;
#pragma unroll
        for (int k = 0; k < kBatch; ++k) {
            // a part without a key is zeros; a NaN among its weights (its sum is one, whatever its reference point) stays one
            const float w = ml[k].x == -INFINITY ? 1.f : ex2(ml[k].x - top);
            sum += ml[k].y * w;
            v[0] += x[k][0].x * w; v[1] += x[k][0].y * w; v[2] += x[k][0].z * w; v[3] += x[k][0].w * w;
            v[4] += x[k][1].x * w; v[5] += x[k][1].y * w; v[6] += x[k][1].z * w; v[7] += x[k][1].w * w;
        }
    }
    // no key at all: 0
    const float inv = top == -INFINITY && sum == 0.f ? 0.f : 1.f / sum;
    const int rw = rt * p.tile_rows + row, i = rw / p.G, hq = h * p.G + rw - i * p.G;
    __nv_bfloat162 o[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) o[j] = __floats2bfloat162_rn(v[2 * j] * inv, v[2 * j + 1] * inv);
    *reinterpret_cast<uint4 *>(p.out + (b * p.os.batch + i * p.os.token + hq * p.os.head) + 8 * c8) = *reinterpret_cast<uint4 *>(o);
}

#include "dd_cached_attention_tiles.cuh"
#include "dd_cached_attention_wide.cuh"
#include "dd_cached_attention_narrow.cuh"

// ---------------------------------------------------------------------------- host side

typedef CUresult (*EncodeTiledFn)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                                  const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                                  CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// A pool as rows of D bytes; a copy takes `rows` of them (of one page).
int make_pool_map(CUtensorMap *m, void *base, const dd_cache *c, int rows)
{
    static std::mutex mu;
    static EncodeTiledFn fn = nullptr;
    {
        std::lock_guard<std::mutex> lock(mu);
        if (!fn) {
            void *sym = nullptr;
            cudaDriverEntryPointQueryResult q;
            DD_CUDA_TRY(cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &sym, cudaEnableDefault, &q));
            if (q != cudaDriverEntryPointSuccess) return dd::cuda_fail(cudaErrorSymbolNotFound, "cuTensorMapEncodeTiled entry point");
            fn = reinterpret_cast<EncodeTiledFn>(sym);
        }
    }
    const cuuint64_t dims[2] = {(cuuint64_t)c->D, (cuuint64_t)c->num_pages * c->heads * c->page_size};
    const cuuint64_t strides[1] = {(cuuint64_t)c->D};
    const cuuint32_t box[2] = {(cuuint32_t)c->D, (cuuint32_t)rows}, estr[2] = {1, 1};
    if (fn(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, base, dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
           c->D == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
           CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
        return dd::cuda_fail(cudaErrorInvalidValue, "cuTensorMapEncodeTiled");
    return DD_OK;
}

template <int D>
int launch_cached(const dd_cache *c, const CachedParams &p, cudaStream_t s)
{
    static bool done[3][64] = {};
    CUtensorMap tk, tv;
    int rc;
    const int rows = c->page_size < kTileKeys ? c->page_size : kTileKeys;
    if ((rc = make_pool_map(&tk, c->k, c, rows)) != DD_OK || (rc = make_pool_map(&tv, c->v, c, rows)) != DD_OK) return rc;
    auto run = [&](auto kernel, int threads, int smem, bool (&allowed)[64]) -> int {
        int rc = dd::allow_smem((const void *)kernel, smem, allowed);
        if (rc != DD_OK) return rc;
        DD_CUDA_TRY(dd::launch(kernel, (unsigned)p.ctas, threads, smem, s, 1, tk, tv, p));
        return DD_OK;
    };
    if (p.tile_rows == 16) rc = run(cached_attention_narrow_kernel<D, 16>, NarrowShape<D, 16>::kThreads, NarrowShape<D, 16>::kTotal, done[0]);
    else if (p.tile_rows == 32) rc = run(cached_attention_narrow_kernel<D, 32>, NarrowShape<D, 32>::kThreads, NarrowShape<D, 32>::kTotal, done[1]);
    else rc = run(cached_attention_wide_kernel<D>, kWideThreads, WideShape<D>::kTotal, done[2]);
    if (rc != DD_OK) return rc;
    dd::count_launch();
    DD_CUDA_TRY(dd::launch_2d(cached_attention_join_kernel<D>, (unsigned)p.ctas, (unsigned)(p.part_rows / 16), 16 * D / 8, 0, s, p));
    dd::count_launch();
    return DD_OK;
}

// What a call's sizes decide: the kernel (by tile_rows), the rows' tiles and the workspace.  DD_OK, or why not.
int make_plan(int B, int H, int Nq, const dd_cache *cache, CachedParams &p, size_t &workspace)
{
    int sms = 0, rc;
    const long rows = (long)(H / cache->heads) * Nq;
    if (rows >= (1L << 31) - 128) return DD_ERR_UNSUPPORTED;
    // The narrow kernel's softmax warps go by sixteens of rows.  Up to 16 rows on its form for 32: one token of 16 sequences of 16384 keys, 32 heads on 8,
    // 103 us for 86; 8 x 32 heads, 16 queries over 2048 keys 41 for 32.  17 to 32 rows on the wide kernel: 16 x 32 heads, 20 queries over up
    // to 1024 keys 52 us for 35, 4 x 32 heads 23.7 for 18.8, those with D = 64 18.7 for 17.9.
    p.tile_rows = rows <= 16 ? 16 : rows <= 32 ? 32 : 128;
    p.part_rows = rows < 128 ? (int)(rows + 15) / 16 * 16 : 128;
    const long tiles = (rows + p.tile_rows - 1) / p.tile_rows;
    // items, and key tiles of all items, are counted in 32 bits
    const long keys = (long)cache->max_pages * cache->page_size, items = tiles * cache->heads;
    if (items >= (1L << 28) || items * B >= (1L << 28) || items * B * ((keys + kTileKeys - 1) / kTileKeys) >= (1L << 31)) return DD_ERR_UNSUPPORTED;
    if ((rc = dd::sm_count(&sms)) != DD_OK) return rc;
    p.ctas = 2 * sms;                       // two on each SM
    p.B = B;
    p.Hkv = cache->heads;
    p.G = H / cache->heads;
    p.Nq = Nq;
    p.rows = (int)rows;
    p.row_tiles = (int)tiles;
    workspace = 2 * (size_t)p.ctas * (cache->D == 64 ? part_floats<64>(p.part_rows) : part_floats<128>(p.part_rows)) * 4 + p.ctas * sizeof(Record);
    return DD_OK;
}

}  // namespace

extern "C" size_t dd_cached_attention_workspace_bytes(int B, int H, int Nq, const dd_cache *cache)
{
    CachedParams p = {};
    size_t bytes = 0;
    if (B <= 0 || H <= 0 || Nq <= 0 || dd::check_cache(cache) != DD_OK || H % cache->heads != 0) return 0;
    return make_plan(B, H, Nq, cache, p, bytes) == DD_OK ? bytes : 0;
}

extern "C" int dd_cached_attention(const void *q, const dd_strides *q_strides, const dd_cache *cache, const int32_t *kv_len,
                                   void *out, const dd_strides *out_strides, int B, int H, int Nq, float scale,
                                   void *workspace, size_t workspace_bytes, void *stream)
{
    if (!q || !out || !kv_len || !workspace || B <= 0 || H <= 0 || Nq <= 0) return DD_ERR_INVALID_ARG;
    int rc;
    if ((rc = dd::check_cache(cache)) != DD_OK) return rc;
    if (H % cache->heads != 0 || !std::isfinite(scale)) return DD_ERR_INVALID_ARG;
    if ((rc = dd::check_strides(q, q_strides)) != DD_OK || (rc = dd::check_strides(out, out_strides)) != DD_OK) return rc;
    if (scale < 0.f || ((uintptr_t)workspace & 15) != 0) return DD_ERR_UNSUPPORTED;
    CachedParams p = {};
    size_t need = 0;
    if ((rc = make_plan(B, H, Nq, cache, p, need)) != DD_OK) return rc;
    if (workspace_bytes < need) return DD_ERR_UNSUPPORTED;
    dd::DeviceCtx *ctx = dd::current_ctx();
    if (!ctx) return DD_ERR_CUDA;
    if ((rc = dd::ensure_mirror(ctx)) != DD_OK || (rc = dd::check_mirror(ctx, 0)) != DD_OK || (rc = dd::ensure_attn_status(ctx)) != DD_OK) return rc;
    p.q = (const __nv_bfloat16 *)q;
    p.out = (__nv_bfloat16 *)out;
    p.qs = *q_strides;
    p.os = *out_strides;
    p.table = cache->page_table;
    p.kv_len = kv_len;
    p.scale[0] = cache->k_scale;
    p.scale[1] = cache->v_scale;
    p.ws = (float *)workspace;
    p.status = ctx->attn_status;
    p.mirror = ctx->mirror_dev;
    p.num_pages = cache->num_pages;
    p.max_pages = cache->max_pages;
    p.page = cache->page_size;
    p.page_log2 = cache->page_size == 16 ? 4 : cache->page_size == 32 ? 5 : cache->page_size == 64 ? 6 : 7;
    p.scale_log2 = scale * 1.4426950408889634f;
    return cache->D == 64 ? launch_cached<64>(cache, p, (cudaStream_t)stream) : launch_cached<128>(cache, p, (cudaStream_t)stream);
}
