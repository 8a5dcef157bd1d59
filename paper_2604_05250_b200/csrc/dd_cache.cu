// dd_qk_norm_rope and dd_cache_append: what a layer does with its projections before the attention of the drafter's step.
#include <cuda_bf16.h>
#include <cuda_fp8.h>
#include <cuda_runtime.h>

#include <cmath>

#include "dd_common.cuh"
#include "dd_ptx.cuh"
#include "dd_rope.cuh"

namespace {

using namespace ddrope;

// ----------------------------------------------------------------------------- norms of queries and keys, rotation

struct RopeParams {
    const __nv_bfloat16 *x[2];          // queries, keys
    __nv_bfloat16 *out[2];
    const __nv_bfloat16 *weight[2];
    dd_strides in[2];
    int heads[2];
    const int32_t *start;
    Rotation rot;
    float eps;
    int B, N, head_major;
};

// A group of D / 16 lanes takes kHeads heads of one token, whose angles it loads once.  Bound by bytes: 64 heads of 8192 tokens 47.6 us, 5.7
// TB/s (before packed products 49.8; two heads a group 54, eight 57, CTAs of 256 threads 52); where one round of single heads fits the chip, by latency: one
// token's 40 heads 2.0 us (four heads a group 3.1).
constexpr int kRopeThreads = 128;
template <int D, int kHeads>
__global__ void __launch_bounds__(kRopeThreads) qk_norm_rope_kernel(const RopeParams p, const unsigned items, const unsigned blocks)
{
    constexpr int kLanes = Lane<D>::kLanes;
    ddptx::grid_wait();
    const int lane = threadIdx.x % kLanes;
    const Lane<D> l(lane, p.rot);
    const unsigned item = blockIdx.x * (kRopeThreads / kLanes) + threadIdx.x / kLanes;
    const bool live = item < items;
    const unsigned token = live ? item / blocks : 0;                  // b * N + i
    const int h0 = live ? (int)(item - token * blocks) * kHeads : 0;
    const int b = (int)(token / (unsigned)p.N), i = (int)(token - (unsigned)b * p.N);
    const int all = p.heads[0] + p.heads[1];
    uint4 raw[kHeads][2];
#pragma unroll
    for (int j = 0; j < kHeads; ++j) {
        const int h = h0 + j, which = h >= p.heads[0];
        raw[j][0] = raw[j][1] = make_uint4(0u, 0u, 0u, 0u);
        if (live && h < all) {
            const dd_strides &s = p.in[which];
            const uint4 *row = reinterpret_cast<const uint4 *>(p.x[which] + (b * s.batch + i * s.token + (h - which * p.heads[0]) * s.head));
            raw[j][0] = row[l.a];
            raw[j][1] = row[l.b];
        }
    }
    Angles t;
    load_angles(t, p.rot, (p.start ? (long)p.start[b] : 0L) + i, lane, l.rotates);
    ddptx::grid_trigger();
#pragma unroll
    for (int j = 0; j < kHeads; ++j) {
        const int h = h0 + j, which = h >= p.heads[0];
        float x[16];
        unpack(x, raw[j][0]);
        unpack(x + 8, raw[j][1]);
        norm_rows<D>(x, p.weight[which], p.weight[0] || p.weight[1], p.eps, l);
        rotate_row<D>(x, t, l.rotates, p.rot.interleaved);
        if (live && h < all) {
            const int head = h - which * p.heads[0], heads = p.heads[which];
            const size_t row = p.head_major ? ((size_t)b * heads + head) * p.N + i : (size_t)token * heads + head;
            uint4 *to = reinterpret_cast<uint4 *>(p.out[which] + row * D);
            to[l.a] = pack(x);
            to[l.b] = pack(x + 8);
        }
    }
}

template <int D, int kHeads>
int launch_rope(const RopeParams &p, cudaStream_t s)
{
    const long blocks = (p.heads[0] + p.heads[1] + kHeads - 1) / kHeads, items = (long)p.B * p.N * blocks;
    const long grid = (items + kRopeThreads / Lane<D>::kLanes - 1) / (kRopeThreads / Lane<D>::kLanes);
    if (items >= (1L << 31)) return DD_ERR_UNSUPPORTED;
    DD_CUDA_TRY(dd::launch(qk_norm_rope_kernel<D, kHeads>, (unsigned)grid, kRopeThreads, 0, s, 1, p, (unsigned)items, (unsigned)blocks));
    dd::count_launch();
    return DD_OK;
}

// ----------------------------------------------------------------------------- keys and values into the cache

struct AppendParams {
    const __nv_bfloat16 *x[2];          // keys, values
    dd_strides in[2];
    uint8_t *pool[2];
    float *scale[2];
    const __nv_bfloat16 *weight;        // of the keys' norm
    const int32_t *table, *start, *count, *held;
    Rotation rot;
    float eps;
    int B, N, H, num_pages, max_pages, page_log2, touched;
};

constexpr int kScaleLow = -60, kScaleHigh = 60, kHeldHigh = 100;       // of the scales made here, and of those that a cache may hold

// Smallest e with x <= 448 * 2^e = 1.75 * 2^(e + 8), for finite x >= 0; within the range of scales.
__device__ __forceinline__ int scale_exponent(float x)
{
    const uint32_t u = __float_as_uint(x);
    const int e = (int)(u >> 23) - 127 - 8 + ((u & 0x7FFFFFu) > 0x600000u);
    return max(kScaleLow, min(kScaleHigh, e));
}
// Smallest power of two that is no smaller than a scale in the cache (which is one, if it was written here).
__device__ __forceinline__ int held_exponent(float x)
{
    const uint32_t u = __float_as_uint(x);
    if (!(x > 0.f)) return kScaleLow;
    const int e = (int)(u >> 23) - 127 + ((u & 0x7FFFFFu) != 0);
    return max(kScaleLow, min(kHeldHigh, e));
}
__device__ __forceinline__ float power_of_two(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }

// Four e4m3 numbers, each the nearest (ties to even), beyond 448 the largest; the first in the lowest byte.
__device__ __forceinline__ uint32_t to_e4m3x4(float a, float b, float c, float d)
{
    uint32_t w;
    asm("{\n\t.reg .b16 l, h;\n\tcvt.rn.satfinite.e4m3x2.f32 l, %2, %1;\n\tcvt.rn.satfinite.e4m3x2.f32 h, %4, %3;\n\tmov.b32 %0, {l, h};\n\t}"
        : "=r"(w) : "f"(a), "f"(b), "f"(c), "f"(d));
    return w;
}
// Both halves of a bf16 pair times a bf16 number, exact conversion and one rounding: no instruction to unpack them.
__device__ __forceinline__ float2 scaled(uint32_t pair, __nv_bfloat16 by)
{
    float2 v;
    asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %2;\n\tfma.rn.f32.bf16 %0, l, %3, 0f00000000;\n\tfma.rn.f32.bf16 %1, h, %3, 0f00000000;\n\t}"
        : "=f"(v.x), "=f"(v.y) : "r"(pair), "h"(*reinterpret_cast<const unsigned short *>(&by)));
    return v;
}
__device__ __forceinline__ uint2 to_e4m3x8(const uint4 &v, __nv_bfloat16 by)
{
    const float2 a = scaled(v.x, by), b = scaled(v.y, by), c = scaled(v.z, by), d = scaled(v.w, by);
    return make_uint2(to_e4m3x4(a.x, a.y, b.x, b.y), to_e4m3x4(c.x, c.y, d.x, d.y));
}
// The larger magnitudes of two pairs of bf16 numbers; NaN only where both are.
__device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b)
{
    const __nv_bfloat162 m = __hmax2(*reinterpret_cast<const __nv_bfloat162 *>(&a), __habs2(*reinterpret_cast<const __nv_bfloat162 *>(&b)));
    return *reinterpret_cast<const uint32_t *>(&m);
}
__device__ __forceinline__ float2 from_e4m3x2(uint32_t pair)
{
    const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)pair, __NV_E4M3);
    return __half22float2(*reinterpret_cast<const __half2 *>(&h));
}

// Four e4m3 numbers, each times the ratio.
__device__ __forceinline__ uint32_t times(uint32_t v, float ratio)
{
    const float2 a = from_e4m3x2(v & 0xFFFF), b = from_e4m3x2(v >> 16);
    return to_e4m3x4(a.x * ratio, a.y * ratio, b.x * ratio, b.y * ratio);
}

// A group of threads takes one page of some heads, of the keys or of the values, one head after the other.  A head's new rows are read
// once, stay in registers until their largest magnitude is known to the whole group, and are written under the scale that this gives.
// What bounds it: for prompts bytes, 3 a value, and where keys are normed or rotated as much the instructions (4.5 to 5.9 TB/s, IPC 2.4, ALU pipe
// 55 %); a few dependent reads (start, page number, rows) for single tokens, 2.5 us.  The next heads' rows
// are copied to shared memory meanwhile, each lane's pieces to a place of its own (no barrier), and a lane's angles stay in registers: with
// a group for each head, which waits for its rows and reads the angles anew, 4 prompts of up to 8192 tokens took 269 us where this takes 115
// (angles read anew for each head of 256 threads with four rows each: 142; before packed products and mixed multiply-adds 123).  Values, and keys without norm and rotation, are
// scaled straight from bf16 (see scaled()): 4 x 8192 tokens 199 -> 130 us, 6.2 TB/s.
// kMost: new rows that a group has room for in a page.  By the call's tokens, not by the page's size: a single token is one warp's work
// (by the page's size, 64: 8.1 us for 2.5).
template <int D, int kMost>
struct AppendShape {
    static constexpr int kLanes = Lane<D>::kLanes;                                         // of a row
    static constexpr int kRows = kMost * kLanes <= 32 ? 1 : 2;                             // of a thread
    static constexpr int kGroup = kMost * kLanes / kRows;                                  // threads: 32 to 512
    static constexpr int kThreads = kGroup < 128 ? 128 : kGroup;
    static constexpr int kGroups = kThreads / kGroup, kStages = 3;
    static constexpr int kSmem = kStages * kRows * 2 * 16 * kThreads;
    static constexpr int kCtas = 512 / kThreads;                                           // an SM, at the least: 128 registers a thread
};

__device__ __forceinline__ void copy16(uint32_t to, const void *from) { asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory"); }
__device__ __forceinline__ void copies_end() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

template <int D, int kMost>
__global__ void __launch_bounds__(AppendShape<D, kMost>::kThreads, AppendShape<D, kMost>::kCtas)
cache_append_kernel(const AppendParams p, const unsigned items, const int heads_each)
{
    using S = AppendShape<D, kMost>;
    constexpr int kLanes = S::kLanes, kStep = S::kGroup / kLanes, kRows = S::kRows;
    extern __shared__ uint4 staged[];
    __shared__ float most[2][S::kThreads / 32];
    ddptx::grid_wait();
    const int group = threadIdx.x / S::kGroup, in_group = threadIdx.x % S::kGroup, lane = threadIdx.x % kLanes;
    const unsigned item = blockIdx.x * S::kGroups + group, blocks = (p.H + heads_each - 1) / heads_each;
    // item = ((b * touched + j) * 2 + which) * blocks + block of heads
    const unsigned block = item % blocks, rest = item / blocks, which = rest & 1, slot = rest >> 1;
    const int b = (int)(slot / p.touched), j = (int)(slot - (unsigned)b * p.touched);
    bool live = item < items;
    long start = 0, base = 0, end = 0, held = 0;
    int id = -1;
    if (live) {
        start = p.start[b];
        const int n = p.count ? max(0, min(p.count[b], p.N)) : p.N;
        end = start + n;
        held = p.held ? (long)p.held[b] : start;
        const long page_index = (start > 0 ? start >> p.page_log2 : 0) + j;                // (no token has a place before the first page)
        base = page_index << p.page_log2;
        live = page_index < p.max_pages && base < end && n > 0;
        if (live) {
            id = p.table[(size_t)b * p.max_pages + page_index];
            live = id >= 0 && id < p.num_pages;
        }
    }
    const int h0 = block * heads_each, h1 = live ? min(h0 + heads_each, p.H) : h0;
    // rows that are stored as they are: no norm, no rotation
    const bool plain = which == 1 || (!p.weight && p.rot.dims == 0);
    Lane<D> l(lane, p.rot);
    if (plain) { l.a = lane; l.b = lane + kLanes; }
    // tokens of the page that stay: held, and not among the new ones
    const long page_end = base + (1L << p.page_log2), last = min(held, page_end), from = max(start, base), to = min(end, page_end);
    const bool stay = last > base && (from > base || last > to);
    // this thread's new rows: `first` rows behind `from`, and every kStep-th
    const int first = in_group / kLanes;
    bool fresh[kRows];
#pragma unroll
    for (int r = 0; r < kRows; ++r) fresh[r] = live && from + first + r * kStep < to;
    const dd_strides &in = p.in[which];
    const __nv_bfloat16 *source = p.x[which] + (b * in.batch + (from - start + first) * in.token);
    const uint32_t stage0 = ddptx::smem_u32(staged) + threadIdx.x * 16;
    float was_next = 1.f;
    auto request = [&](int h) {
        if (h < h1) {
#pragma unroll
            for (int r = 0; r < kRows; ++r)
                if (fresh[r]) {
                    const uint4 *x = reinterpret_cast<const uint4 *>(source + (r * kStep * in.token + h * in.head));
                    const uint32_t at = stage0 + ((h - h0) % S::kStages * kRows + r) * (2 * 16 * S::kThreads);
                    copy16(at, x + l.a);
                    copy16(at + 16 * S::kThreads, x + l.b);
                }
        }
        copies_end();
    };
    request(h0);
    request(h0 + 1);
    Angles angles[kRows];
#pragma unroll
    for (int r = 0; r < kRows; ++r)
        if (which == 0 && fresh[r]) load_angles(angles[r], p.rot, from + first + r * kStep, lane, l.rotates);
    if (live && stay) was_next = p.scale[which][(size_t)id * p.H + h0];
    // (the same number of turns for every group of the CTA)
    for (int h = h0; h < h0 + heads_each; ++h) {
        request(h + S::kStages - 1);
        const float was = was_next;
        if (stay && h + 1 < h1) was_next = p.scale[which][(size_t)id * p.H + h + 1];
        if (h + 3 >= h0 + heads_each) ddptx::grid_trigger();
        copies_wait<S::kStages - 1>();
        uint4 raw[kRows][2];
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            raw[r][0] = raw[r][1] = make_uint4(0u, 0u, 0u, 0u);
            if (fresh[r] && h < h1) {
                const uint4 *at = staged + threadIdx.x + ((h - h0) % S::kStages * kRows + r) * (2 * S::kThreads);
                raw[r][0] = at[0];
                raw[r][1] = at[S::kThreads];
            }
        }
        float x[kRows][16], mx;
        if (plain) {
            uint32_t top = 0u;
#pragma unroll
            for (int r = 0; r < kRows; ++r)
#pragma unroll
                for (int c = 0; c < 2; ++c) top = larger(larger(larger(larger(top, raw[r][c].x), raw[r][c].y), raw[r][c].z), raw[r][c].w);
            mx = fmaxf(0.f, fmaxf(__uint_as_float(top << 16), __uint_as_float(top & 0xFFFF0000u)));
        } else {
            mx = 0.f;
#pragma unroll
            for (int r = 0; r < kRows; ++r) {
                unpack<true>(x[r], raw[r][0]);
                unpack<true>(x[r] + 8, raw[r][1]);
                norm_rows<D, true>(x[r], p.weight, p.weight != nullptr, p.eps, l);
                if (fresh[r]) rotate_row<D>(x[r], angles[r], l.rotates, p.rot.interleaved);
#pragma unroll
                for (int i = 0; i < 16; i += 2) mx = ddptx::max3(mx, fabsf(x[r][i]), fabsf(x[r][i + 1]));
            }
        }
        // ---- the page's scale (magnitudes as integers: they order alike)
        mx = __uint_as_float(__reduce_max_sync(0xFFFFFFFFu, __float_as_uint(mx)));
        if (S::kGroup > 32) {
            if (threadIdx.x % 32 == 0) most[h & 1][threadIdx.x / 32] = mx;
            ddptx::named_bar_sync(1 + group, S::kGroup);
            mx = most[h & 1][group * (S::kGroup / 32) + threadIdx.x % (S::kGroup / 32)];
            mx = __uint_as_float(__reduce_max_sync(0xFFFFFFFFu, __float_as_uint(mx)));
        } else __syncwarp();        // (the old scale has been read by everybody)
        if (h >= h1) continue;
        int e = scale_exponent(fminf(mx, 3.4e38f));
        if (stay) e = max(e, held_exponent(was));
        const float scale = power_of_two(e), inverse = power_of_two(-e);
        const size_t head_page = (size_t)id * p.H + h;
        uint8_t *page = p.pool[which] + ((head_page << p.page_log2) + (from - base + first)) * D;
#pragma unroll
        for (int r = 0; r < kRows; ++r)
            if (fresh[r]) {
                uint2 *at = reinterpret_cast<uint2 *>(page + r * kStep * D);
                if (plain) {
                    at[l.a] = to_e4m3x8(raw[r][0], __float2bfloat16_rn(inverse));
                    at[l.b] = to_e4m3x8(raw[r][1], __float2bfloat16_rn(inverse));
                    continue;
                }
#pragma unroll
                for (int i = 0; i < 16; i += 2) {
                    const float2 y = __fmul2_rn(make_float2(x[r][i], x[r][i + 1]), make_float2(inverse, inverse));
                    x[r][i] = y.x;
                    x[r][i + 1] = y.y;
                }
                at[l.a] = make_uint2(to_e4m3x4(x[r][0], x[r][1], x[r][2], x[r][3]), to_e4m3x4(x[r][4], x[r][5], x[r][6], x[r][7]));
                at[l.b] = make_uint2(to_e4m3x4(x[r][8], x[r][9], x[r][10], x[r][11]), to_e4m3x4(x[r][12], x[r][13], x[r][14], x[r][15]));
            }
        if (stay && scale != was) {
            // the tokens that stay, 16 bytes a thread: exact but for results below 2^-6, by a power of two less
            const float ratio = was * inverse;
            uint4 *all = reinterpret_cast<uint4 *>(p.pool[which] + (head_page << p.page_log2) * D);
            for (int i = in_group; i < (int)(last - base) * (D / 16); i += S::kGroup) {
                const long at = base + i / (D / 16);
                if (at >= from && at < to) continue;
                const uint4 v = all[i];
                all[i] = make_uint4(times(v.x, ratio), times(v.y, ratio), times(v.z, ratio), times(v.w, ratio));
            }
        }
        if (in_group == 0) p.scale[which][head_page] = scale;
    }
}

template <int D, int kMost>
int launch_append(const AppendParams &p, cudaStream_t s)
{
    using S = AppendShape<D, kMost>;
    static bool allowed[64] = {};
    int sms = 0, rc;
    if ((rc = dd::sm_count(&sms)) != DD_OK || (rc = dd::allow_smem((const void *)cache_append_kernel<D, kMost>, S::kSmem, allowed)) != DD_OK) return rc;
    // as many heads to a group as leave every SM its 512 threads: what follows in a second round is then the next heads, on their way already
    // (prompts: at most 8 heads 125 us, 16 115, 32 118)
    const long pages = (long)p.B * p.touched * 2;
    int each = 1;
    while (each < 16 && each < p.H && pages * ((p.H + 2 * each - 1) / (2 * each)) * S::kGroup >= 512L * sms) each *= 2;
    const long items = pages * ((p.H + each - 1) / each);
    DD_CUDA_TRY(dd::launch(cache_append_kernel<D, kMost>, (unsigned)((items + S::kGroups - 1) / S::kGroups), S::kThreads, S::kSmem, s, 1, p, (unsigned)items, each));
    dd::count_launch();
    return DD_OK;
}

}  // namespace

extern "C" int dd_qk_norm_rope(const void *q, const dd_strides *q_strides, int H, const void *k, const dd_strides *k_strides, int Hkv,
                               const void *q_weight, const void *k_weight, float eps, const dd_rotation *rotation, const int32_t *start,
                               void *out_q, void *out_k, int B, int N, int D, int layout, void *stream)
{
    if (!q || !out_q || B <= 0 || N <= 0 || H <= 0 || D <= 0 || Hkv < 0) return DD_ERR_INVALID_ARG;
    if (Hkv > 0 && (!k || !out_k)) return DD_ERR_INVALID_ARG;
    if (layout != DD_LAYOUT_BHND && layout != DD_LAYOUT_BNHD) return DD_ERR_INVALID_ARG;
    if (!std::isfinite(eps) || eps < 0.f) return DD_ERR_INVALID_ARG;
    if (D != 64 && D != 128) return DD_ERR_UNSUPPORTED;
    RopeParams p = {};
    int rc;
    if ((rc = check_rotation(rotation, D, p.rot)) != DD_OK || (rc = dd::check_strides(q, q_strides)) != DD_OK) return rc;
    if (Hkv > 0 && (rc = dd::check_strides(k, k_strides)) != DD_OK) return rc;
    if ((((uintptr_t)q_weight | (uintptr_t)k_weight | (uintptr_t)out_q | (uintptr_t)out_k) & 15) != 0) return DD_ERR_UNSUPPORTED;
    p.x[0] = (const __nv_bfloat16 *)q;
    p.x[1] = (const __nv_bfloat16 *)k;
    p.out[0] = (__nv_bfloat16 *)out_q;
    p.out[1] = (__nv_bfloat16 *)out_k;
    p.weight[0] = (const __nv_bfloat16 *)q_weight;
    p.weight[1] = Hkv > 0 ? (const __nv_bfloat16 *)k_weight : nullptr;
    p.in[0] = *q_strides;
    if (Hkv > 0) p.in[1] = *k_strides;
    p.heads[0] = H;
    p.heads[1] = Hkv;
    p.start = start;
    p.eps = eps;
    p.B = B;
    p.N = N;
    p.head_major = layout == DD_LAYOUT_BHND;
    if ((long)B * N >= (1L << 31) || (long)H + Hkv >= (1L << 20)) return DD_ERR_UNSUPPORTED;
    cudaStream_t s = (cudaStream_t)stream;
    int sms = 0;
    if ((rc = dd::sm_count(&sms)) != DD_OK) return rc;
    if ((long)B * N * (H + Hkv) * (D / 16) <= 512L * sms) return D == 64 ? launch_rope<64, 1>(p, s) : launch_rope<128, 1>(p, s);
    return D == 64 ? launch_rope<64, 4>(p, s) : launch_rope<128, 4>(p, s);
}

extern "C" int dd_cache_append(const void *k, const dd_strides *k_strides, const void *v, const dd_strides *v_strides, const dd_cache *cache,
                               const int32_t *start, const int32_t *count, const int32_t *kv_len, const void *k_weight, float eps,
                               const dd_rotation *rotation, int B, int N, void *stream)
{
    if (!k || !v || !cache || !start || B <= 0 || N <= 0) return DD_ERR_INVALID_ARG;
    int rc;
    if ((rc = dd::check_cache(cache)) != DD_OK) return rc;
    if (!std::isfinite(eps) || eps < 0.f) return DD_ERR_INVALID_ARG;
    AppendParams p = {};
    if ((rc = check_rotation(rotation, cache->D, p.rot)) != DD_OK || (rc = dd::check_strides(k, k_strides)) != DD_OK ||
        (rc = dd::check_strides(v, v_strides)) != DD_OK)
        return rc;
    if (((uintptr_t)k_weight & 15) != 0) return DD_ERR_UNSUPPORTED;
    p.x[0] = (const __nv_bfloat16 *)k;
    p.x[1] = (const __nv_bfloat16 *)v;
    p.in[0] = *k_strides;
    p.in[1] = *v_strides;
    p.pool[0] = (uint8_t *)cache->k;
    p.pool[1] = (uint8_t *)cache->v;
    p.scale[0] = cache->k_scale;
    p.scale[1] = cache->v_scale;
    p.weight = (const __nv_bfloat16 *)k_weight;
    p.table = cache->page_table;
    p.start = start;
    p.count = count;
    p.held = kv_len;
    p.eps = eps;
    p.B = B;
    p.N = N;
    p.H = cache->heads;
    p.num_pages = cache->num_pages;
    p.max_pages = cache->max_pages;
    const int page = cache->page_size;
    p.touched = (int)(((long)N + page - 2) / page + 1);
    if (p.touched > cache->max_pages) p.touched = cache->max_pages;      // (a start beyond the first page touches fewer of the table's)
    if ((long)B * p.touched * 2 * p.H >= (1L << 31)) return DD_ERR_UNSUPPORTED;                 // items are counted in 32 bits
    p.page_log2 = page == 16 ? 4 : page == 32 ? 5 : page == 64 ? 6 : 7;
    cudaStream_t s = (cudaStream_t)stream;
    const int most = N < page ? N : page;                    // new rows in a page
    if (cache->D == 64)
        return most <= 8 ? launch_append<64, 8>(p, s) : most <= 16 ? launch_append<64, 16>(p, s) : most <= 32 ? launch_append<64, 32>(p, s) :
               most <= 64 ? launch_append<64, 64>(p, s) : launch_append<64, 128>(p, s);
    return most <= 4 ? launch_append<128, 4>(p, s) : most <= 16 ? launch_append<128, 16>(p, s) : most <= 32 ? launch_append<128, 32>(p, s) :
           most <= 64 ? launch_append<128, 64>(p, s) : launch_append<128, 128>(p, s);
}
