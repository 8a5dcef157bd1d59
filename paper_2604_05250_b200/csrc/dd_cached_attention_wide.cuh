// dd_cached_attention for more than 32 query rows a key head: tiles of 128 rows by 128 keys on the tensor cores' own memory.
//   warps 0-7   softmax (thread = query row = TMEM lane, warps 4-7 for the tile's second 64 keys); they also prepare the queries and write
//               the result
//   warp  8     copies of keys and values (a lane for each page), scales of the pages
//   warp  9     one thread issues every product
//   warps 10-11 turn a tile's values from e4m3 into f16, which is exact
// Two CTAs share an SM; each takes a contiguous share of all (item, key tile) pairs.
// What bounds it: the chain scores - weights - products of a tile.  The weights go over the scores, since two CTAs fill the tensor memory, so a CTA's
// next scores wait for its products; a tile takes a CTA alone 2.2 us and two of them 1.6 us of the SM, of which the tensor core works 0.55 and
// the exponentials' unit 0.54.  8 x 32 heads, 256 queries over 8192 keys 333 us (826 TFLOP/s of the definition's products, 0.50 of what a
// library's bf16 product reaches); 2 x 32 heads over 4096 keys 60 us, of which some 15 are the ends: share, queries, result, join.
// At 80 registers a thread it spills 196 bytes.
// A row's weights taken before its largest score is known, and anew where they turn out too large: 301 us if none ever did, but 432 with
// heads as peaked as these (scores of a deviation of 8), where some row of 128 outgrows its reference point in most tiles.
//
// Scores: e4m3 products straight from the copied bytes.  A query row, under a power of two that brings its largest entry into (224, 448], is
// the sum of two e4m3 numbers an entry: bf16's eight bits exactly down to 2^-10 of the row's largest entry, and within 2^-18 of that
// for smaller ones.  Twice the products at twice the rate of f16, and no keys to convert.
// Weights relative to a reference point of the row that may lag the row's maximum by a factor of 2^6, times the values' scales (relative to
// a power of two no smaller than any so far, of 2^-100 to 2^100: the range of scales), in f16 with 2^8 on top: nothing overflows, and what underflows is below 2^-32 of the reference.
//
// Included by dd_cached_attention.cu (inside its unnamed namespace).
#pragma once

constexpr int kWideThreads = 384, kWideCopyWarp = 8, kWideMmaWarp = 9;

template <int D>
struct WideShape {
    static constexpr int kHalfBytes = kTileRows * D;             // one of the two parts of the queries
    static constexpr int kTileBytes = kTileKeys * D;             // e4m3
    static constexpr int kBoxBytes = kTileKeys * 128;            // 64 columns of the values in f16
    static constexpr int kKSlots = D == 128 ? 2 : 4, kVSlots = D == 128 ? 1 : 3;
    static constexpr int kQ = 0, kK = 2 * kHalfBytes, kV8 = kK + kKSlots * kTileBytes, kV16 = kV8 + kVSlots * kTileBytes;
    static constexpr int kShared = kV16 + (D / 64) * kBoxBytes;
    struct Shared {
        float4 scale[kKSlots][4];           // of the tile's eight groups of 16 keys: keys' (negative: not there), then values'
        float exchange[kTileRows];          // between the two threads of a row
        uint64_t q_full, s_full, p_full, o_full, v16_full, v16_empty;
        uint64_t k_full[kKSlots], k_empty[kKSlots], v8_full[kVSlots], v8_empty[kVSlots];
        uint32_t tmem;
    };
    static constexpr int kTotal = kShared + (int)sizeof(Shared);
    static_assert(2 * (kTotal + 1024) <= 228 * 1024, "two CTAs on an SM");
};

// Barrier of the eight softmax warps, and whether the predicate held anywhere.
__device__ __forceinline__ bool any_of_256(bool x)
{
    uint32_t r;
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\tbarrier.cta.red.or.pred q, 1, 256, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
                 : "=r"(r) : "r"((uint32_t)x) : "memory");
    return r != 0;
}

template <int D>
__global__ void __launch_bounds__(kWideThreads, 2)
cached_attention_wide_kernel(const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v, const CachedParams p)
{
    using S = WideShape<D>;
    extern __shared__ __align__(1024) unsigned char smem[];
    typename S::Shared &sh = *reinterpret_cast<typename S::Shared *>(smem + S::kShared);
    const int tid = threadIdx.x, warp = warp_uniform(tid >> 5), lane = tid & 31;
    const uint32_t base = smem_u32(smem);
    const uint32_t bar_q = smem_u32(&sh.q_full), bar_s = smem_u32(&sh.s_full), bar_p = smem_u32(&sh.p_full), bar_o = smem_u32(&sh.o_full),
                   bar_v16 = smem_u32(&sh.v16_full), bar_v16_empty = smem_u32(&sh.v16_empty);
    auto bar_k = [&](int s) { return smem_u32(&sh.k_full[0]) + 8 * s; };
    auto bar_k_empty = [&](int s) { return smem_u32(&sh.k_empty[0]) + 8 * s; };
    auto bar_v8 = [&](int s) { return smem_u32(&sh.v8_full[0]) + 8 * s; };
    auto bar_v8_empty = [&](int s) { return smem_u32(&sh.v8_empty[0]) + 8 * s; };
    if (tid == kWideCopyWarp * 32) {
        prefetch_tmap(&tm_k);
        prefetch_tmap(&tm_v);
        mbar_init(bar_q, 256);
        mbar_init(bar_s, 1);
        mbar_init(bar_p, 256);
        mbar_init(bar_o, 1);
        mbar_init(bar_v16, 64);
        mbar_init(bar_v16_empty, 1);
        for (int s = 0; s < S::kKSlots; ++s) { mbar_init(bar_k(s), 33); mbar_init(bar_k_empty(s), 9); }
        for (int s = 0; s < S::kVSlots; ++s) { mbar_init(bar_v8(s), 1); mbar_init(bar_v8_empty(s), 64); }
        fence_mbar_init();
    }
    if (warp == 0) { tmem_alloc(smem_u32(&sh.tmem), 256); tmem_relinquish(); }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = warp_uniform(*reinterpret_cast<volatile uint32_t *>(&sh.tmem));
    constexpr uint32_t kColS = 0, kColO = 128;
    grid_wait();
    unsigned err = 0;
    Cursor now;
    const bool misplaced = base & 1023;     // the swizzles go by the address
    if (misplaced && tid == 0) report(p, kErrPlace);
    // (a wait that has expired before: nothing more is begun; one lane's word for the warp, whose lanes find their share together)
    const Split split(p, lane);
    const bool quiet = warp_uniform(*reinterpret_cast<volatile unsigned int *>(p.status)) == 0;
    const bool work = __syncthreads_and(!misplaced && quiet && find_share(p, lane, split, now));
    clear_empty<D>(p);
    if (!work) {
        if (tid == 0) write_record<D>(p, split, now, false);
    } else if (warp < 8) {
        reg_inc<88>();                      // (2 x 32 heads, 256 queries over 4096 keys: 60.3 us; 80 registers for all 62.8, 96 and 48 62.3)
        // =================================================================== queries, softmax, result
        const int half = warp >> 2, row = (warp & 3) * 32 + lane;
        const uint32_t lane_off = (uint32_t)((warp & 3) * 32) << 16;
        constexpr int kCols = kTileKeys / 2;                     // of this thread in every tile
        // weights go over the first half of this thread's own scores
        const uint32_t tS = tmem + lane_off + kColS + half * kCols, tO = tmem + lane_off + kColO + half * (D / 2);
        int tile = 0, part = 0;                                  // so far, over all items
        for (;; ++part) {
            const int live_rows = min(kTileRows, p.rows - now.rt * kTileRows);
            // ---- the rows as two e4m3 parts, K-major with the copies' swizzle: D / 8 lanes take a row, a warp 16 rows
            {
                constexpr int kLanes = D / 8, kStep = 32 / kLanes, kTimes = 16 / kStep;
                const int x = lane % kLanes, r0 = warp * 16;
                int64_t mine = 0;                                // lane i: where row r0 + i begins
                if (lane < 16) {
                    const int rw = now.rt * kTileRows + r0 + lane, iq = rw / p.G;
                    mine = now.b * p.qs.batch + iq * p.qs.token + (now.h * p.G + rw - iq * p.G) * p.qs.head;
                }
                uint4 raw[kTimes];
                uint32_t top[kTimes];
#pragma unroll
                for (int i = 0; i < kTimes; ++i) {
                    const int from = i * kStep + lane / kLanes;
                    const int64_t at = __shfl_sync(0xFFFFFFFFu, mine, from);
                    raw[i] = make_uint4(0u, 0u, 0u, 0u);
                    if (r0 + from < live_rows) raw[i] = reinterpret_cast<const uint4 *>(p.q + at)[x];
                }
#pragma unroll
                for (int i = 0; i < kTimes; ++i)
                    top[i] = max(max(max(raw[i].x & 0x7FFFu, (raw[i].x >> 16) & 0x7FFFu), max(raw[i].y & 0x7FFFu, (raw[i].y >> 16) & 0x7FFFu)),
                                 max(max(raw[i].z & 0x7FFFu, (raw[i].z >> 16) & 0x7FFFu), max(raw[i].w & 0x7FFFu, (raw[i].w >> 16) & 0x7FFFu)));
                // (each exchange for all the rows before the next: they do not wait for one another)
#pragma unroll
                for (int o = kLanes / 2; o > 0; o /= 2)
#pragma unroll
                    for (int i = 0; i < kTimes; ++i) top[i] = max(top[i], __shfl_xor_sync(0xFFFFFFFFu, top[i], o));
#pragma unroll
                for (int i = 0; i < kTimes; ++i) {
                    const int r = r0 + i * kStep + lane / kLanes;
                    const uint32_t w[4] = {raw[i].x, raw[i].y, raw[i].z, raw[i].w};
                    const int e = min(100, 8 - ((int)(top[i] >> 7) - 127) - ((top[i] & 0x7Fu) > 0x60u));
                    const float up = power_of_two(e);
                    // an entry that is not finite makes the row's scores NaN
                    if (x == 0) sh.exchange[r] = top[i] >= 0x7F80u ? __uint_as_float(0x7FFFFFFFu) : power_of_two(-e) * p.scale_log2;
                    uint32_t hi[2], lo[2];
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        float v[4] = {__uint_as_float(w[2 * k] << 16) * up, __uint_as_float(w[2 * k] & 0xFFFF0000u) * up,
                                      __uint_as_float(w[2 * k + 1] << 16) * up, __uint_as_float(w[2 * k + 1] & 0xFFFF0000u) * up};
                        hi[k] = split_e4m3(v);
                        lo[k] = split_e4m3(v);
                    }
                    unsigned char *to = smem + S::kQ + piece<D>(r, x / 2) + 8 * (x & 1);
                    *reinterpret_cast<uint2 *>(to) = make_uint2(hi[0], hi[1]);
                    *reinterpret_cast<uint2 *>(to + S::kHalfBytes) = make_uint2(lo[0], lo[1]);
                }
            }
            fence_proxy_async_smem();
            mbar_arrive(bar_q);
            named_bar_sync(2, 256);
            const float back = sh.exchange[row];                 // score = product * back * scale of the keys
            const int keys = now.keys;
            float m = -INFINITY, l = 0.f, far = 1.f;             // m: the row's reference point; l: of this thread's keys
            bool any_far = false;
            for (int c = now.c; c < now.end; ++c, ++tile) {
                const int slot = tile % S::kKSlots;
                if (err == 0 && !__all_sync(0xFFFFFFFFu, wait_awake(bar_s, tile & 1))) err = kErrTileS;
                tc_fence_after();
                const int valid = keys - c * kTileKeys - half * kCols;     // of this thread's keys, from the first on
                // 32 scores at a time; read twice, once for the largest and once for the weights
                uint32_t s[32];
                tmem_ld32(tS, s);
                const float *ks = reinterpret_cast<const float *>(sh.scale[slot]) + half * 4, *vs = ks + 8;
                const float4 k0 = sh.scale[slot][half], v0 = sh.scale[slot][2], v1 = sh.scale[slot][3];
                const float vmax = fmaxf(max3(v0.x, v0.y, fmaxf(v0.z, v0.w)), max3(v1.x, v1.y, fmaxf(v1.z, v1.w)));
                const bool masked = valid < kCols || fminf(fminf(k0.x, k0.y), fminf(k0.z, k0.w)) < 0.f;
                const auto in = [&](int i) { return ks[i / 16] >= 0.f && i < valid; };
                // ---- the largest score (one branch for the whole tile: the blocks run into one another)
                float mx = -INFINITY;
                auto largest = [&](auto some) {
#pragma unroll
                    for (int cb = 0; cb < kCols / 32; ++cb) {
                        tmem_wait_ld(s);
                        const float *x = reinterpret_cast<const float *>(s);
#pragma unroll
                        for (int gr = 0; gr < 2; ++gr) {
                            const float f = ks[2 * cb + gr] * back;
                            if constexpr (decltype(some)::value) {
#pragma unroll
                                for (int i = 16 * gr; i < 16 * gr + 16; ++i) mx = fmaxf(mx, in(32 * cb + i) ? x[i] * f : -INFINITY);
                            } else {
                                float a = x[16 * gr], b = x[16 * gr + 1];
#pragma unroll
                                for (int i = 16 * gr + 2; i < 16 * gr + 14; i += 4) { a = max3(a, x[i], x[i + 1]); b = max3(b, x[i + 2], x[i + 3]); }
                                mx = fmaxf(mx, max3(a, b, fmaxf(x[16 * gr + 14], x[16 * gr + 15])) * f);
                            }
                        }
                        tmem_ld32(tS + (cb + 1) % (kCols / 32) * 32, s);         // the next ones; at the end the first again
                    }
                };
                if (masked) largest(std::true_type());
                else largest(std::false_type());
                // ---- the reference points: as long as none is outgrown by more than the lag, the row's other maximum is not needed
                const bool grows = vmax > 0.f && (!any_far || vmax > far), first = c == now.c;
                if (any_of_256(mx > m + kLag) || first || grows) {
                    float shrink = 1.f;
                    if (grows) {
                        const int e = max(-100, min(100, (int)(__float_as_uint(vmax) >> 23) - 127 + ((__float_as_uint(vmax) & 0x7FFFFFu) != 0)));
                        if (any_far) shrink = far * power_of_two(-e);
                        far = power_of_two(e);
                        any_far = true;
                    }
                    if (half == 1) sh.exchange[row] = mx;
                    named_bar_sync(2, 256);
                    if (half == 0) sh.exchange[row] = mx = fmaxf(mx, sh.exchange[row]);
                    named_bar_sync(2, 256);
                    mx = sh.exchange[row];
                    const float m_new = mx > m + kLag ? mx : m;
                    const float alpha = ex2(m - (m_new == -INFINITY ? 0.f : m_new)), both = alpha * shrink;
                    m = m_new;
                    l *= alpha;
                    if (!first && __any_sync(0xFFFFFFFFu, both != 1.f)) {
                        // (the scores on their way are waited for here, and read again)
                        tmem_wait_ld(s);
#pragma unroll
                        for (int cb = 0; cb < D / 64; ++cb) {
                            tmem_ld32(tO + cb * 32, s);
                            tmem_wait_ld(s);
#pragma unroll
                            for (int i = 0; i < 32; ++i) s[i] = __float_as_uint(__uint_as_float(s[i]) * both);
                            tmem_st32(tO + cb * 32, s);
                        }
                        tmem_wait_st();
                        tmem_ld32(tS, s);
                    }
                }
                const float ref = m == -INFINITY ? 0.f : m, near = 256.f * power_of_two(127 - (int)(__float_as_uint(far) >> 23));
                // ---- weights, over the scores (a pair of f16 a column)
                float2 sum = make_float2(0.f, 0.f), sum_b = sum;
                auto weights = [&](auto some) {
#pragma unroll
                    for (int cb = 0; cb < kCols / 32; ++cb) {
                        uint32_t pk[16];
                        tmem_wait_ld(s);
                        const float *y = reinterpret_cast<const float *>(s);
#pragma unroll
                        for (int gr = 0; gr < 2; ++gr) {
                            const float f = ks[2 * cb + gr] * back, v = fmaxf(vs[2 * cb + gr], 0.f) * near;
#pragma unroll
                            for (int i = 16 * gr; i < 16 * gr + 16; i += 2) {
                                const float2 x = __ffma2_rn(make_float2(y[i], y[i + 1]), make_float2(f, f), make_float2(-ref, -ref));
                                float2 w = make_float2(ex2(x.x), ex2(x.y));
                                if constexpr (decltype(some)::value) {
                                    w.x = in(cb * 32 + i) ? w.x : 0.f;
                                    w.y = in(cb * 32 + i + 1) ? w.y : 0.f;
                                }
                                if (i & 2) sum = __fadd2_rn(sum, w);
                                else sum_b = __fadd2_rn(sum_b, w);
                                w = __fmul2_rn(w, make_float2(v, v));
                                pk[i / 2] = half2_bits(w.x, w.y);
                            }
                        }
                        if (cb + 1 < kCols / 32) tmem_ld32(tS + (cb + 1) * 32, s);
                        tmem_st16(tS + cb * 16, pk);
                    }
                };
                if (masked) weights(std::true_type());
                else weights(std::false_type());
                l += (sum.x + sum_b.x) + (sum.y + sum_b.y);
                tmem_wait_st();
                tc_fence_before();
                mbar_arrive(bar_p);
                __syncwarp();
                if (lane == 0) mbar_arrive(bar_k_empty(slot));   // the tile's scales have been read
            }
            // ---- the result, or this part of it: half of the columns each
            named_bar_sync(2, 256);                              // (the last maxima have been read)
            if (half == 1) sh.exchange[row] = l;
            named_bar_sync(2, 256);
            if (half == 0) sh.exchange[row] = l += sh.exchange[row];
            named_bar_sync(2, 256);
            l = sh.exchange[row];
            if (err == 0 && !__all_sync(0xFFFFFFFFu, wait_awake(bar_o, part & 1))) err = kErrTileO;
            tc_fence_after();
            const bool whole = now.c0 == 0 && now.end == now.n, live = row < live_rows;
            float *to = part_of<D>(p, blockIdx.x, now.c0 == 0);
            const int rw = now.rt * kTileRows + row, i_q = rw / p.G;
            __nv_bfloat16 *out = p.out + (now.b * p.os.batch + i_q * p.os.token + (now.h * p.G + rw - i_q * p.G) * p.os.head) + half * (D / 2);
            const bool sectors = (reinterpret_cast<uintptr_t>(out) & 31) == 0;
            const float mine = far * (1.f / 256.f), f = !whole ? mine : m == -INFINITY && l == 0.f ? 0.f : mine / l;
            if (!whole && live && half == 0) *reinterpret_cast<float2 *>(to + p.part_rows * D + 2 * row) = make_float2(m, l);
#pragma unroll
            for (int cb = 0; cb < D / 64; ++cb) {
                uint32_t o[32];
                tmem_ld32(tO + cb * 32, o);
                tmem_wait_ld(o);
                if (!live || err != 0) continue;
                if (whole) {
#pragma unroll
                    for (int c0 = 0; c0 < 32; c0 += 16) {
                        uint32_t w[8];
#pragma unroll
                        for (int h = 0; h < 8; ++h) {
                            __nv_bfloat162 x = __floats2bfloat162_rn(__uint_as_float(o[c0 + 2 * h]) * f, __uint_as_float(o[c0 + 2 * h + 1]) * f);
                            w[h] = *reinterpret_cast<uint32_t *>(&x);
                        }
                        __nv_bfloat16 *dst = out + cb * 32 + c0;
                        if (sectors) st_global_v8(dst, w);
                        else {
                            reinterpret_cast<uint4 *>(dst)[0] = make_uint4(w[0], w[1], w[2], w[3]);
                            reinterpret_cast<uint4 *>(dst)[1] = make_uint4(w[4], w[5], w[6], w[7]);
                        }
                    }
                } else {
                    float4 *dst = reinterpret_cast<float4 *>(to) + (half * (D / 8) + cb * 8) * p.part_rows + row;
#pragma unroll
                    for (int h = 0; h < 8; ++h)
                        dst[h * p.part_rows] = make_float4(__uint_as_float(o[4 * h]) * f, __uint_as_float(o[4 * h + 1]) * f,
                                                           __uint_as_float(o[4 * h + 2]) * f, __uint_as_float(o[4 * h + 3]) * f);
                }
            }
            tc_fence_before();
            if (now.left == 0) break;
            now.next(p);
            named_bar_sync(2, 256);                              // exchange[] has been read
        }
    } else {
        reg_dec<64>();
        if (warp == kWideCopyWarp) {
            copy_tiles<S, D>(p, tm_k, tm_v, base, sh, split, now, lane, err);
            grid_trigger();
        } else if (warp == kWideMmaWarp && elect_one()) {
            // =============================================================== products
            constexpr uint32_t kIdescS = idesc_type0(kTileRows, kTileKeys, false, false), kIdescO = idesc_type0(kTileRows, D, false, true);
            const uint32_t desc_q = desc_low(base + S::kQ, 16), desc_k = desc_low(base + S::kK, 16), desc_v = desc_low(base + S::kV16, S::kBoxBytes);
            int tile = 0, part = 0;
            auto issue_s = [&](int t) {
                const int slot = t % S::kKSlots;
                if (!wait_awake(bar_k(slot), (t / S::kKSlots) & 1)) { err = kErrTileK; return false; }
                tc_fence_after();
                const uint32_t b = desc_k + slot * (S::kTileBytes >> 4);
#pragma unroll
                for (int half = 0; half < 2; ++half)
#pragma unroll
                    for (int ks = 0; ks < D / 32; ++ks)
                        mma_ss_f8(tmem + kColS, desc_q + half * (S::kHalfBytes >> 4) + ks * 2, kRowsHigh<D>, b + ks * 2, kRowsHigh<D>, kIdescS, half > 0 || ks > 0);
                mma_commit(bar_s);
                mma_commit(bar_k_empty(slot));
                return true;
            };
            for (; err == 0; ++part) {
                if (!wait_awake(bar_q, part & 1)) { err = kErrTileQ; break; }
                tc_fence_after();
                if (!issue_s(tile)) break;
                for (int c = now.c; c < now.end; ++c, ++tile) {
                    if (!wait_awake(bar_v16, tile & 1)) { err = kErrTileV; break; }
                    if (!wait_awake(bar_p, tile & 1)) { err = kErrTileP; break; }
                    tc_fence_after();
                    // 16 keys = two groups of 8 rows of 1024 bytes
#pragma unroll
                    for (int ks = 0; ks < kTileKeys / 16; ++ks)
                        mma_ts_f16(tmem + kColO, tmem + kColS + (ks / 4) * 64 + (ks % 4) * 8, desc_v + ks * (2048 >> 4), desc_high<128>(1024), kIdescO, c > now.c || ks > 0);
                    mma_commit(bar_v16_empty);
                    if (c + 1 == now.end) { mma_commit(bar_o); ++tile; break; }
                    if (!issue_s(tile + 1)) break;
                }
                if (err != 0 || now.left == 0) break;
                now.next(p);
            }
        } else if (warp > kWideMmaWarp) {
            // =================================================================== values to f16
            const int ct = tid - (kWideMmaWarp + 1) * 32;
            int tile = 0;
            for (;;) {
                const int keys = now.keys;
                for (int c = now.c; c < now.end && err == 0; ++c, ++tile) {
                    const int slot = tile % S::kVSlots;
                    if (!wait_awake(bar_v8(slot), (tile / S::kVSlots) & 1)) { err = kErrTileV; break; }
                    if (tile > 0 && !wait_awake(bar_v16_empty, (tile - 1) & 1)) { err = kErrTileV; break; }
                    convert_values<D>(smem + S::kV8 + slot * S::kTileBytes, base + S::kV16, ct, keys - c * kTileKeys);
                    fence_proxy_async_smem();
                    mbar_arrive(bar_v16);
                    mbar_arrive(bar_v8_empty(slot));
                }
                if (now.left == 0 || err != 0) break;
                now.next(p);
            }
        }
    }
    if (err != 0) report(p, err);
    __syncwarp();
    if (*reinterpret_cast<volatile unsigned int *>(p.status) != 0)
        // a wait expired somewhere: copies that may still be in flight get time to land before the shared memory is released
#pragma unroll 1
        for (int i = 0; i < 2000; ++i) __nanosleep(1000);
    tc_fence_before();
    __syncthreads();
    if (warp == 0) { __syncwarp(); tmem_dealloc(tmem, 256); }
}
