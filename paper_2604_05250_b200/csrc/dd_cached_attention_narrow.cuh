// dd_cached_attention for up to 32 query rows a key head: keys along the products' 128 rows, queries along their columns, and both
// operands of both products in 8 bits, so that keys and values go to the tensor core as the bytes that were copied.
//   S^T = K Q^T      [128 keys x 2 R columns]: a query entry is the sum of two e4m3 numbers, whose columns the softmax adds
//   O^T += V^T P^T   [D x 3 R columns]: a weight is the sum of three e5m2 numbers, whose columns are added at an item's end
// (R = 16 or 32 rows.)  A product reads its 128-row operand once, whatever the number of columns: the parts cost no second pass.  At a
// tile of 128 keys that is 256 cycles of shared-memory reads and as many for the copies' writes, where the tile's 32 KB take some 1400
// cycles to come from memory.  Values turned into f16 by warps of their own, in another buffer, took 1300 of those (and 1.3 us a tile).
//   4 warps for each 16 rows: softmax (thread = key = TMEM lane of S^T, entry d = lane of O^T); they also prepare their queries and write their
//             result, and know nothing of the other 16 rows'
//   a warp    copies of keys and values (a lane for each page), scales of the pages
//   a warp    one thread issues S^T
//   a warp    one thread issues O^T; the warp clears value rows behind a sequence's end before: 0 x NaN is NaN
// Two CTAs share an SM; each takes a contiguous share of all (item, key tile) pairs.
// What bounds it (D = 128, a graph's replays): bytes for long caches, one token of 16 sequences of up to 16384 keys, 32 heads on 8, 57 us, 6.07
// TB/s, 0.93 of what a copy reaches; for 32 rows of shorter ones a CTA's ends and the softmax's instructions, 16 x 32 heads, 32
// queries over up to 1024 keys 35 us, 2.7 TB/s (IPC 2.1, ALU pipe 42 %, two items a CTA); for few keys the chain of latencies from the lengths
// to the joined result, one token of one sequence of 1024 keys, 32 heads, 9.6 us, of 64 keys (nothing to join) 7.0.
// At 80 registers a thread the form for 32 rows spills 192 bytes, the form for 16 (128 registers) none.
//
// Queries: a row is taken under a power of two that brings its largest entry into (224, 448]; two e4m3 numbers then hold bf16's eight bits
// exactly down to 2^-10 of the row's largest entry, and are within 2^-18 of that for smaller ones.
// Weights are relative to a reference point of the row that may lag its maximum by a factor of 2^5, times the values' scales (relative to
// a power of two no smaller than any so far, of 2^-100 to 2^100: the range of scales), times 2^10: three e5m2 numbers are within 2^-9 of a weight (half a step of bf16),
// and what is lost below their smallest step is at most 2^-27 of the reference's weight.
// A row's maximum is spread over the lanes here, but as long as no weight outgrows the lag it is not needed: the warps agree
// on that by one barrier with a vote, and only where the vote fails (the first tile, and rarely later) the maxima are gathered.
// The sums of weights stay spread over the keys' threads until the item's end.
//
// Included by dd_cached_attention.cu (inside its unnamed namespace).
#pragma once

template <int D, int N>
struct NarrowShape {
    static constexpr int kSoftmax = 4 * (N / 16), kThreads = (kSoftmax + 4) * 32;       // warps of the softmax, threads
    static constexpr int kPartBytes = N * D;                     // one of the two parts of the queries
    static constexpr int kTileBytes = kTileKeys * D;             // e4m3
    static constexpr int kWeightRow = 4 * N;                     // bytes of a key's weights: three parts of N, and a gap
    static constexpr int kKSlots = D == 64 ? 4 : N == 16 ? 3 : 2, kVSlots = D == 64 ? 4 : 2, kPSlots = 2;
    static constexpr int kK = 0, kV8 = kK + kKSlots * kTileBytes, kP = kV8 + kVSlots * kTileBytes, kQ = kP + kPSlots * kTileKeys * kWeightRow;
    static constexpr int kShared = kQ + 2 * kPartBytes;
    static constexpr int kColO = 4 * N, kTmem = N == 16 ? 128 : 256;       // O^T behind two buffers of scores
    struct Shared {
        float4 scale[kKSlots][4];           // of the tile's eight groups of 16 keys: keys' (negative: not there), then values'
        uint64_t q_full, s_full[2], p_full[2], pv_done[2];
        uint64_t k_full[kKSlots], k_empty[kKSlots], v8_full[kVSlots], v8_empty[kVSlots];
        float column[N / 16][4][32];        // a warp's maximum or sum of each column
        // of two query rows at a time: score = product * back * scale of the keys, and the reference points' negatives
        alignas(16) float line[N / 2][4];      // back, back, -ref, -ref
        alignas(16) float move[N / 16][32], alpha[N / 16][32];          // of each column's reference point, and what that makes of its sums
        int64_t q_at[N], out_at[N];       // of each row, from its item's first
        uint32_t tmem;
    };
    static constexpr int kTotal = kShared + (int)sizeof(Shared);
    static_assert(2 * (kTotal + 1024) <= 228 * 1024, "two CTAs on an SM");
};
constexpr float kNarrowLag = 5.f, kNarrowTop = 1024.f;

// A pair of e5m2 numbers nearest to a pair of f16, which become what is left of them.  (e5m2 is the upper half of f16.)
__device__ __forceinline__ uint32_t split_e5m2(__half2 &x)
{
    uint32_t pair, v = *reinterpret_cast<uint32_t *>(&x);
    asm("{\n\t.reg .b16 h;\n\tcvt.rn.satfinite.e5m2x2.f16x2 h, %1;\n\tcvt.u32.u16 %0, h;\n\t}" : "=r"(pair) : "r"(v));
    uint32_t wide = __byte_perm(pair, 0u, 0x1404);
    x = __hsub2(x, *reinterpret_cast<__half2 *>(&wide));
    return pair;
}

// 16 columns, spread over a warp's lanes, joined: lanes c and c + 16 get column c's.
template <typename Op>
__device__ __forceinline__ float join_columns(float (&v)[16], int lane, Op op)
{
#pragma unroll
    for (int half = 8; half > 0; half /= 2) {
        const bool upper = lane & half;
#pragma unroll
        for (int i = 0; i < half; ++i) {
            const float other = __shfl_xor_sync(0xFFFFFFFFu, upper ? v[i] : v[i + half], half);
            v[i] = op(upper ? v[i + half] : v[i], other);
        }
    }
    return op(v[0], __shfl_xor_sync(0xFFFFFFFFu, v[0], 16));
}
// Barrier of four softmax warps, and whether the predicate held anywhere.
__device__ __forceinline__ bool any_of_128(uint32_t barrier, bool x)
{
    uint32_t r;
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\tbarrier.cta.red.or.pred q, %2, 128, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
                 : "=r"(r) : "r"((uint32_t)x), "r"(barrier) : "memory");
    return r != 0;
}
// 16 columns of this thread's lane.
__device__ __forceinline__ void issue_columns(uint32_t taddr, float (&v)[16])
{
    uint32_t *r = reinterpret_cast<uint32_t *>(v);
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
                   "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]) : "r"(taddr) : "memory");
}
// (the values pass through the wait: nothing computed from them moves before it)
__device__ __forceinline__ void wait_columns(float (&v)[16])
{
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+f"(v[0]), "+f"(v[1]), "+f"(v[2]), "+f"(v[3]), "+f"(v[4]), "+f"(v[5]), "+f"(v[6]), "+f"(v[7]), "+f"(v[8]), "+f"(v[9]),
                   "+f"(v[10]), "+f"(v[11]), "+f"(v[12]), "+f"(v[13]), "+f"(v[14]), "+f"(v[15]) :: "memory");
}

template <int D, int N>
__global__ void __launch_bounds__(NarrowShape<D, N>::kThreads, 2)
cached_attention_narrow_kernel(const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v, const CachedParams p)
{
    using S = NarrowShape<D, N>;
    extern __shared__ __align__(1024) unsigned char smem[];
    typename S::Shared &sh = *reinterpret_cast<typename S::Shared *>(smem + S::kShared);
    const int tid = threadIdx.x, warp = warp_uniform(tid >> 5), lane = tid & 31;
    const uint32_t base = smem_u32(smem);
    const uint32_t bar_q = smem_u32(&sh.q_full);
    auto bar_s = [&](int t) { return smem_u32(&sh.s_full[0]) + 8 * (t & 1); };
    auto bar_p = [&](int t) { return smem_u32(&sh.p_full[0]) + 8 * (t & 1); };
    auto bar_pv = [&](int t) { return smem_u32(&sh.pv_done[0]) + 8 * (t & 1); };
    auto bar_k = [&](int s) { return smem_u32(&sh.k_full[0]) + 8 * s; };
    auto bar_k_empty = [&](int s) { return smem_u32(&sh.k_empty[0]) + 8 * s; };
    auto bar_v8 = [&](int s) { return smem_u32(&sh.v8_full[0]) + 8 * s; };
    auto bar_v8_empty = [&](int s) { return smem_u32(&sh.v8_empty[0]) + 8 * s; };
    if (tid == S::kSoftmax * 32) {
        prefetch_tmap(&tm_k);
        prefetch_tmap(&tm_v);
        mbar_init(bar_q, S::kSoftmax * 32);
        for (int s = 0; s < 2; ++s) { mbar_init(bar_s(s), 1); mbar_init(bar_p(s), S::kSoftmax * 32); mbar_init(bar_pv(s), 1); }
        for (int s = 0; s < S::kKSlots; ++s) { mbar_init(bar_k(s), 33); mbar_init(bar_k_empty(s), 1 + S::kSoftmax); }
        for (int s = 0; s < S::kVSlots; ++s) { mbar_init(bar_v8(s), 1); mbar_init(bar_v8_empty(s), 1); }
        fence_mbar_init();
    }
    if (warp == 0) { tmem_alloc(smem_u32(&sh.tmem), S::kTmem); tmem_relinquish(); }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = warp_uniform(*reinterpret_cast<volatile uint32_t *>(&sh.tmem));
    grid_wait();
    unsigned err = 0;
    Cursor now;
    const bool misplaced = base & 1023;                          // the swizzles go by the address
    if (misplaced && tid == 0) report(p, kErrPlace);
    // (a wait that has expired before: nothing more is begun; one lane's word for the warp, whose lanes find their share together)
    const Split split(p, lane);
    const bool quiet = warp_uniform(*reinterpret_cast<volatile unsigned int *>(p.status)) == 0;
    const bool work = __syncthreads_and(!misplaced && quiet && find_share(p, lane, split, now));
    clear_empty<D>(p);
    if (!work) {
        if (tid == 0) write_record<D>(p, split, now, false);
    } else if (warp < S::kSoftmax) {
        reg_inc<N == 16 ? 176 : 96>();
        // =================================================================== queries, softmax, result, of 16 rows
        const int half = N == 16 ? 0 : warp >> 2, w4 = warp & 3, key = tid & 127;
        const uint32_t lane_off = (uint32_t)(w4 * 32) << 16, tO = tmem + lane_off + S::kColO + half * 16, barrier = 1 + 2 * half;
        constexpr int kLanes = D / 8, kRowsAtOnce = 128 / kLanes, kPasses = 16 / kRowsAtOnce;      // lanes of a row of queries
        auto together = [&] { named_bar_sync(barrier + 1, 128); };
        if (key < 16) {
            const int r = half * 16 + key, iq = r / p.G, in_group = r - iq * p.G;
            sh.q_at[r] = iq * p.qs.token + in_group * p.qs.head;
            sh.out_at[r] = iq * p.os.token + in_group * p.os.head;
        }
        together();
        uint4 raw[kPasses];
        auto query = [&](const Cursor &c, int r) {
            return reinterpret_cast<const uint4 *>(p.q + (c.b * p.qs.batch + c.h * (p.G * p.qs.head) + sh.q_at[r])) + key % kLanes;
        };
        auto load_queries = [&](const Cursor &c) {
#pragma unroll
            for (int i = 0; i < kPasses; ++i) {
                const int r = half * 16 + i * kRowsAtOnce + key / kLanes;
                raw[i] = make_uint4(0u, 0u, 0u, 0u);
                if (r < p.rows) raw[i] = *query(c, r);
            }
        };
        // the rows as two e4m3 parts, K-major with the copies' swizzle
        auto place_queries = [&] {
#pragma unroll
            for (int i = 0; i < kPasses; ++i) {
                const int r = half * 16 + i * kRowsAtOnce + key / kLanes, x = key % kLanes;
                const uint32_t w[4] = {raw[i].x, raw[i].y, raw[i].z, raw[i].w};
                uint32_t top = 0;
#pragma unroll
                for (int k = 0; k < 4; ++k) top = max(top, max(w[k] & 0x7FFFu, (w[k] >> 16) & 0x7FFFu));
#pragma unroll
                for (int o = kLanes / 2; o > 0; o /= 2) top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
                const int e = min(100, 8 - ((int)(top >> 7) - 127) - ((top & 0x7Fu) > 0x60u));
                const float up = power_of_two(e);
                // an entry that is not finite makes the row's scores NaN
                if (x == 0) sh.line[r >> 1][r & 1] = top >= 0x7F80u ? __uint_as_float(0x7FFFFFFFu) : power_of_two(-e) * p.scale_log2;
                if (x == 1) sh.line[r >> 1][2 + (r & 1)] = 0.f;
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
                *reinterpret_cast<uint2 *>(to + S::kPartBytes) = make_uint2(lo[0], lo[1]);
            }
            fence_proxy_async_smem();
            mbar_arrive(bar_q);
            together();                                          // line[] is there
        };
        load_queries(now);
        place_queries();
        int tile = 0;                                            // so far, over all items
        for (;;) {
            if (now.left > 0) {                                  // the next item's queries set out, as far as the L2 cache: no registers for them
                Cursor next = now;
                next.next(p);
#pragma unroll
                for (int i = 0; i < kPasses; ++i) {
                    const int r = half * 16 + i * kRowsAtOnce + key / kLanes;
                    if (r < p.rows) asm volatile("prefetch.global.L2 [%0];" ::"l"(query(next, r)));
                }
            }
            const int keys = now.keys;
            // m_col: the reference point of column `lane` % 16; limit: how far a score may be beyond its own.  As long as a column has none (its tiles
            // so far had no key) any key calls for one: its sum must not begin at 0.
            float l[16], m_col = -INFINITY, far = 1.f, limit = -INFINITY;
#pragma unroll
            for (int j = 0; j < 16; ++j) l[j] = 0.f;
            bool any_far = false;
            for (int c = now.c; c < now.end; ++c, ++tile) {
                const int slot = tile % S::kKSlots;
                const bool turn = c + 1 == now.end && now.left > 0;       // to the next item
                if (turn) {
                    Cursor next = now;
                    next.next(p);
                    load_queries(next);
                }
                if (err == 0 && !__all_sync(0xFFFFFFFFu, wait_awake(bar_s(tile), (tile >> 1) & 1))) err = kErrTileS;
                tc_fence_after();
                const float *scales = reinterpret_cast<const float *>(sh.scale[slot]);
                float s[16];
                {
                    float lo[16];
                    issue_columns(tmem + lane_off + (tile & 1) * (2 * N) + half * 16, s);
                    issue_columns(tmem + lane_off + (tile & 1) * (2 * N) + N + half * 16, lo);
                    wait_columns(s);
                    wait_columns(lo);
#pragma unroll
                    for (int j = 0; j < 16; j += 2) {
                        const float2 x = __fadd2_rn(make_float2(s[j], s[j + 1]), make_float2(lo[j], lo[j + 1]));
                        s[j] = x.x; s[j + 1] = x.y;
                    }
                }
                const float ks = scales[key >> 4], vs = fmaxf(scales[8 + (key >> 4)], 0.f);
                const float4 va = sh.scale[slot][2], vb = sh.scale[slot][3];
                const float vmax = fmaxf(max3(va.x, va.y, fmaxf(va.z, va.w)), max3(vb.x, vb.y, fmaxf(vb.z, vb.w)));
                const bool there = ks >= 0.f && key < keys - c * kTileKeys;
                const float2 k2 = make_float2(ks, ks);
                float over = -INFINITY;
#pragma unroll
                for (int j = 0; j < 16; j += 2) {
                    const float2 x = __fmul2_rn(make_float2(s[j], s[j + 1]), k2);
                    const float4 line = *reinterpret_cast<const float4 *>(sh.line[half * 8 + j / 2]);
                    const float2 y = __ffma2_rn(x, make_float2(line.x, line.y), make_float2(line.z, line.w));
                    s[j] = y.x; s[j + 1] = y.y;
                    over = max3(over, y.x, y.y);
                }
                const bool first = c == now.c0, grows = vmax > 0.f && (!any_far || vmax > far);
                if (any_of_128(barrier, there && over > limit) || first || grows) {
                    // ---- the reference points (s is relative to the old ones)
                    float shrink = 1.f;
                    if (grows) {
                        const int e = max(-100, min(100, (int)(__float_as_uint(vmax) >> 23) - 127 + ((__float_as_uint(vmax) & 0x7FFFFFu) != 0)));
                        const float to = power_of_two(e);
                        if (any_far) shrink = far * power_of_two(-e);
                        far = to;
                        any_far = true;
                    }
                    float v[16];
#pragma unroll
                    for (int j = 0; j < 16; ++j) v[j] = there ? s[j] : -INFINITY;
                    sh.column[half][w4][lane] = join_columns(v, lane, [](float a, float b) { return fmaxf(a, b); });
                    together();
                    const float rise = fmaxf(fmaxf(sh.column[half][0][lane], sh.column[half][1][lane]), fmaxf(sh.column[half][2][lane], sh.column[half][3][lane]));
                    // nothing there yet (m_col = -inf): s is relative to 0
                    const float old = m_col;
                    if (old == -INFINITY) m_col = rise;
                    else if (rise > kNarrowLag) m_col = old + rise;
                    if (__all_sync(0xFFFFFFFFu, m_col != -INFINITY)) limit = kNarrowLag;
                    const float move = m_col == -INFINITY ? 0.f : old == -INFINITY ? m_col : m_col - old;
                    if (w4 == 0) {
                        sh.move[half][lane] = move;
                        sh.alpha[half][lane] = old == -INFINITY ? 0.f : ex2(-move);
                        if (lane < 16) sh.line[half * 8 + (lane >> 1)][2 + (lane & 1)] -= move;
                    }
                    together();
#pragma unroll
                    for (int j = 0; j < 16; ++j) {
                        s[j] -= sh.move[half][j];
                        l[j] *= sh.alpha[half][j];
                    }
                    if (!first) {
                        // O^T as it is after the tile before
                        if (err == 0 && !__all_sync(0xFFFFFFFFu, wait_awake(bar_pv(tile - 1), ((tile - 1) >> 1) & 1))) err = kErrTileO;
                        tc_fence_after();
#pragma unroll 1
                        for (int part = 0; part < 3; ++part) {
                            float o[16];
                            issue_columns(tO + part * N, o);
                            wait_columns(o);
#pragma unroll
                            for (int j = 0; j < 16; ++j) o[j] *= sh.alpha[half][j] * shrink;
                            tmem_st16(tO + part * N, reinterpret_cast<const uint32_t(&)[16]>(o));
                            tmem_wait_st();
                        }
                    }
                }
                // the item's last scores have been read: the next item's queries take these ones' place, and its first scores are computed while
                // this item ends
                if (turn) {
                    together();
                    place_queries();
                }
                // ---- weights, once the products with the last ones in their place are done
                constexpr int kBack = S::kPSlots;
                if (err == 0 && tile >= kBack && !__all_sync(0xFFFFFFFFu, wait_awake(bar_pv(tile - kBack), ((tile - kBack) >> 1) & 1))) err = kErrTileO;
                const float vt = vs * (kNarrowTop * power_of_two(127 - (int)(__float_as_uint(far) >> 23)));
                unsigned char *to = smem + S::kP + (tile % S::kPSlots * kTileKeys + key) * S::kWeightRow;
                const int flip = N == 16 ? (key >> 1) & 3 : key & 7;               // of the row's 16-byte pieces: the swizzle
                uint32_t pk[3][4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    uint32_t pair[3][2];
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        const int j = 4 * i + 2 * k;
                        float2 w = make_float2(ex2(s[j]), ex2(s[j + 1]));
                        if (!there) w = make_float2(0.f, 0.f);
                        const float2 sum = __fadd2_rn(make_float2(l[j], l[j + 1]), w);
                        l[j] = sum.x; l[j + 1] = sum.y;
                        w = __fmul2_rn(w, make_float2(vt, vt));
                        __half2 x = __floats2half2_rn(w.x, w.y);
                        pair[0][k] = split_e5m2(x);
                        pair[1][k] = split_e5m2(x);
                        pair[2][k] = split_e5m2(x);
                    }
#pragma unroll
                    for (int part = 0; part < 3; ++part) pk[part][i] = __byte_perm(pair[part][0], pair[part][1], 0x5410);
                }
#pragma unroll
                for (int part = 0; part < 3; ++part)
                    *reinterpret_cast<uint4 *>(to + (((part * (N / 16) + half) ^ flip) << 4)) = make_uint4(pk[part][0], pk[part][1], pk[part][2], pk[part][3]);
                fence_proxy_async_smem();
                tc_fence_before();
                mbar_arrive(bar_p(tile));
                __syncwarp();
                if (lane == 0) mbar_arrive(bar_k_empty(slot));   // the tile's scales have been read
            }
            // ---- the result, or this part of it
            sh.column[half][w4][lane] = join_columns(l, lane, [](float a, float b) { return a + b; });
            together();
            const float total = (sh.column[half][0][lane] + sh.column[half][1][lane]) + (sh.column[half][2][lane] + sh.column[half][3][lane]);
            const bool whole = now.c0 == 0 && now.end == now.n;
            float *part = part_of<D>(p, blockIdx.x, now.c0 == 0);
            const int col = half * 16 + lane;
            if (!whole && w4 == 0 && lane < 16 && col < p.rows) *reinterpret_cast<float2 *>(part + p.part_rows * D + 2 * col) = make_float2(m_col, total);
            if (w4 == 0) sh.alpha[half][lane] = (!whole ? 1.f : m_col == -INFINITY && total == 0.f ? 0.f : 1.f / total) * far * (1.f / kNarrowTop);
            together();
            if (err == 0 && !__all_sync(0xFFFFFFFFu, wait_awake(bar_pv(tile - 1), ((tile - 1) >> 1) & 1))) err = kErrTileO;
            tc_fence_after();
            float o[16];
            {
                float more[2][16];
                issue_columns(tO, o);
                issue_columns(tO + N, more[0]);
                issue_columns(tO + 2 * N, more[1]);
                wait_columns(o);
                wait_columns(more[0]);
                wait_columns(more[1]);
#pragma unroll
                for (int j = 0; j < 16; ++j) o[j] = (o[j] + more[0][j] + more[1][j]) * sh.alpha[half][j];
            }
            const int d = key, rows = p.rows - half * 16;
            if (err == 0 && (D == 128 || w4 < 2)) {
                if (whole) {
                    // two rows at a time: the even lane of a pair takes the first one's two entries, the odd lane the second one's
                    __nv_bfloat16 *head = p.out + (now.b * p.os.batch + now.h * (p.G * p.os.head) + (d & ~1));
#pragma unroll
                    for (int j = 0; j < 16; j += 2) {
                        const float other = __shfl_xor_sync(0xFFFFFFFFu, lane & 1 ? o[j] : o[j + 1], 1);
                        const __nv_bfloat162 x = lane & 1 ? __floats2bfloat162_rn(other, o[j + 1]) : __floats2bfloat162_rn(o[j], other);
                        if (j + (lane & 1) < rows) *reinterpret_cast<__nv_bfloat162 *>(head + sh.out_at[half * 16 + j + (lane & 1)]) = x;
                    }
                } else {
#pragma unroll
                    for (int j = 0; j < 16; ++j)
                        if (j < rows) part[(half * 16 + j) * D + d] = o[j];
                }
            }
            tc_fence_before();
            if (now.left == 0) break;
            now.next(p);
        }
    } else {
        reg_dec<N == 16 ? 80 : 48>();
        if (warp == S::kSoftmax) {
            copy_tiles<S, D>(p, tm_k, tm_v, base, sh, split, now, lane, err);
            grid_trigger();
        } else if (warp == S::kSoftmax + 1) {
            if (elect_one()) {
                // =========================================================== S^T
                constexpr uint32_t kIdesc = idesc_8bit(kTileKeys, 2 * N, false, false, false);
                const uint32_t desc_q = desc_low(base + S::kQ, 16), desc_k = desc_low(base + S::kK, 16);
                int tile = 0;
                for (int item = 0; err == 0; ++item) {
                    if (!wait_awake(bar_q, item & 1)) { err = kErrTileQ; break; }
                    for (int c = now.c; c < now.end; ++c, ++tile) {
                        const int slot = tile % S::kKSlots;
                        if (!wait_awake(bar_k(slot), (tile / S::kKSlots) & 1)) { err = kErrTileK; break; }
                        // the buffer's scores have been read
                        if (tile > 1 && !wait_awake(bar_p(tile), ((tile >> 1) - 1) & 1)) { err = kErrTileP; break; }
                        tc_fence_after();
                        const uint32_t a = desc_k + slot * (S::kTileBytes >> 4);
#pragma unroll
                        for (int ks = 0; ks < D / 32; ++ks)
                            mma_ss_f8(tmem + (tile & 1) * (2 * N), a + ks * 2, kRowsHigh<D>, desc_q + ks * 2, kRowsHigh<D>, kIdesc, ks > 0);
                        mma_commit(bar_s(tile));
                        mma_commit(bar_k_empty(slot));
                    }
                    if (err != 0 || now.left == 0) break;
                    now.next(p);
                }
            }
        } else if (warp == S::kSoftmax + 2) {
            // =============================================================== O^T
            // (D = 64: 128 rows all the same, the upper half the lower one again, which nobody reads)
            constexpr uint32_t kIdesc = idesc_8bit(128, 3 * N, true, true, true);
            constexpr int kValueGroup = 8 * D, kWeightGroup = 8 * S::kWeightRow;       // bytes of 8 keys
            const uint32_t desc_v = desc_low(base + S::kV8, D == 128 ? 16 : 0), desc_p = desc_low(base + S::kP, 16);
            constexpr uint32_t kValueHigh = desc_high<D>(kValueGroup), kWeightHigh = desc_high<S::kWeightRow>(kWeightGroup);
            int tile = 0;
            for (;;) {
                const int keys = now.keys;
                for (int c = now.c; c < now.end; ++c, ++tile) {
                    const int slot = tile % S::kVSlots, valid = keys - c * kTileKeys;
                    if (!__all_sync(0xFFFFFFFFu, wait_awake(bar_v8(slot), (tile / S::kVSlots) & 1))) { err = kErrTileV; break; }
                    if (valid < kTileKeys) {
                        unsigned char *rows = smem + S::kV8 + slot * S::kTileBytes;
                        for (int i = valid * D + lane * 16; i < kTileKeys * D; i += 512) *reinterpret_cast<uint4 *>(rows + i) = make_uint4(0u, 0u, 0u, 0u);
                        fence_proxy_async_smem();
                        __syncwarp();
                    }
                    if (!__all_sync(0xFFFFFFFFu, wait_awake(bar_p(tile), (tile >> 1) & 1))) { err = kErrTileP; break; }
                    tc_fence_after();
                    if (elect_one()) {
                        const uint32_t a = desc_v + slot * (S::kTileBytes >> 4);
#pragma unroll
                        for (int ks = 0; ks < kTileKeys / 32; ++ks)
                            mma_ss_f8(tmem + S::kColO, a + ks * (4 * kValueGroup >> 4), kValueHigh, desc_p + (tile % S::kPSlots * (kTileKeys * S::kWeightRow) + ks * 4 * kWeightGroup >> 4), kWeightHigh, kIdesc, c > now.c || ks > 0);
                        mma_commit(bar_pv(tile));
                        mma_commit(bar_v8_empty(slot));
                    }
                    __syncwarp();
                }
                if (err != 0 || now.left == 0) break;
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
    if (warp == 0) { __syncwarp(); tmem_dealloc(tmem, S::kTmem); }
}
