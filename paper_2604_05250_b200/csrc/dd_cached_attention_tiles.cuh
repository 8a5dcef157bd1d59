// What both kernels of dd_cached_attention share: tiles of 128 keys, their copies, the values' conversion, products of 8-bit operands.
// Included by dd_cached_attention.cu (inside its unnamed namespace).
#pragma once

constexpr float kLag = 6.f;                 // how far (in powers of two) a row's maximum may outgrow its reference point
enum : unsigned { kErrTileK = 0x700, kErrTileV = 0x800, kErrTileS = 0x900, kErrTileP = 0xA00, kErrTileO = 0xB00, kErrTileQ = 0xC00, kErrTileSlot = 0xD00,
                  kErrPlace = 0xE00 };

// Bounded wait as mbar_wait (about a second), whose polls let the hardware hold the warp for a microsecond at a time: some twenty warps of an SM
// wait at any moment, and their polls take issue slots from the others.
__device__ __forceinline__ bool wait_awake(uint32_t bar, uint32_t parity)
{
#pragma unroll 1
    for (uint32_t it = 0; it < (1u << 20); ++it) {
        uint32_t ok;
        asm volatile(
            "{\n\t.reg .pred p;\n\t"
            "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, 1000;\n\t"
            "selp.u32 %0, 1, 0, p;\n\t}"
            : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
        if (ok) return true;
        if (it > 4096) __nanosleep(100);
    }
    return false;
}

// Shared-memory matrix descriptors in two words: the upper one (distance of 8-row groups, swizzle) is a constant, the lower one (address,
// distance of column blocks) takes one 32-bit addition an operand.  As 64-bit values every operand of an unrolled loop had registers of its own.
template <int kSwizzle>
__host__ __device__ constexpr uint32_t desc_high(uint32_t sbo_bytes)
{
    static_assert(kSwizzle == 128 || kSwizzle == 64, "bytes of the swizzle");
    return (sbo_bytes >> 4) | 1u << 14 | (kSwizzle == 128 ? 2u : 4u) << 29;
}
__device__ __forceinline__ uint32_t desc_low(uint32_t addr, uint32_t lbo_bytes) { return ((addr >> 4) & 0x3FFFu) | (lbo_bytes >> 4) << 16; }
// Rows of D bytes, K-major.
template <int D> constexpr uint32_t kRowsHigh = D == 128 ? desc_high<128>(1024) : desc_high<64>(512);

// D[tmem] (+)= A[smem] * B[smem], 8-bit operands, 32 along K
__device__ __forceinline__ void mma_ss_f8(uint32_t d_tmem, uint32_t a_low, uint32_t a_high, uint32_t b_low, uint32_t b_high, uint32_t idesc, bool accumulate)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .b64 a, b;\n\tsetp.ne.b32 p, %6, 0;\n\tmov.b64 a, {%1, %2};\n\tmov.b64 b, {%3, %4};\n\t"
        "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], a, b, %5, p;\n\t}"
        ::"r"(d_tmem), "r"(a_low), "r"(a_high), "r"(b_low), "r"(b_high), "r"(idesc), "r"((uint32_t)accumulate) : "memory");
}
// D[tmem] (+)= A[tmem] * B[smem], f16, 16 along K
__device__ __forceinline__ void mma_ts_f16(uint32_t d_tmem, uint32_t a_tmem, uint32_t b_low, uint32_t b_high, uint32_t idesc, bool accumulate)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .b64 b;\n\tsetp.ne.b32 p, %5, 0;\n\tmov.b64 b, {%2, %3};\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], b, %4, p;\n\t}"
        ::"r"(d_tmem), "r"(a_tmem), "r"(b_low), "r"(b_high), "r"(idesc), "r"((uint32_t)accumulate) : "memory");
}
// Instruction descriptors, fp32 accumulators: A e4m3, B e4m3 or e5m2 (kind::f8f6f4) ...
__host__ __device__ constexpr uint32_t idesc_8bit(int M, int N, bool a_mn_major, bool b_mn_major, bool b_e5m2)
{
    return (1u << 4) | ((b_e5m2 ? 1u : 0u) << 10) | ((a_mn_major ? 1u : 0u) << 15) | ((b_mn_major ? 1u : 0u) << 16) |
           ((uint32_t)(N >> 3) << 17) | ((uint32_t)(M >> 4) << 24);
}
// ... and operand types 0: f16 (kind::f16), e4m3 (kind::f8f6f4).
__host__ __device__ constexpr uint32_t idesc_type0(int M, int N, bool a_mn_major, bool b_mn_major)
{
    return (1u << 4) | ((a_mn_major ? 1u : 0u) << 15) | ((b_mn_major ? 1u : 0u) << 16) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(M >> 4) << 24);
}

// A tile's values from e4m3 (rows of D bytes with the copies' swizzle) to f16 (rows of 128 bytes, 64 columns a box, 128-byte swizzle), by
// 64 threads; rows at and beyond `valid` become zeros: 0 x NaN is NaN.  Not unrolled as a whole: the warps of an SM share its instruction cache, and 1024 items
// of 40 rows over 300 keys took 68 us for 65, 64 x 32 heads with 64 rows over up to 512 keys 126 for 117.
template <int D>
__device__ __forceinline__ void convert_values(const unsigned char *from, uint32_t to, int thread, int valid)
{
    constexpr int kPieces = D / 16, kStep = 64 / kPieces;        // pieces of 16 bytes in a row; keys at a time: 8 or 16
    // The lanes of the second box take the neighbouring key: two boxes' rows of one key share their banks.
    const int c16 = thread % kPieces, key0 = (thread / kPieces) ^ (c16 >> 2);
    const unsigned char *src = from + piece<D>(key0, c16);
    const uint32_t row = to + (c16 >> 2) * (kTileKeys * 128) + key0 * 128;
    const uint32_t dst0 = row + ((((2 * c16) & 7) ^ (key0 & 7)) << 4), dst1 = row + ((((2 * c16 + 1) & 7) ^ (key0 & 7)) << 4);
#pragma unroll 1
    for (int i0 = 0; i0 < kTileKeys / kStep; i0 += 4) {
        uint4 v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = *reinterpret_cast<const uint4 *>(src + (i0 + i) * (kStep * D));
        if (valid < kTileKeys)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (key0 + (i0 + i) * kStep >= valid) v[i] = make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            uint32_t h[8];
            e4m3_to_f16(v[i].x, h[0], h[1]);
            e4m3_to_f16(v[i].y, h[2], h[3]);
            e4m3_to_f16(v[i].z, h[4], h[5]);
            e4m3_to_f16(v[i].w, h[6], h[7]);
            st_shared_v4(dst0 + (i0 + i) * (kStep * 128), h[0], h[1], h[2], h[3]);
            st_shared_v4(dst1 + (i0 + i) * (kStep * 128), h[4], h[5], h[6], h[7]);
        }
    }
}

// The copy warp: keys and values of the CTA's share, tile by tile (a lane for each page), and the scales of their groups of 16 keys.
template <typename S, int D>
__device__ __forceinline__ void copy_tiles(const CachedParams &p, const CUtensorMap &tm_k, const CUtensorMap &tm_v, uint32_t base,
                                           typename S::Shared &sh, const Split &split, Cursor now, int lane, unsigned &err)
{
    auto bar_k = [&](int s) { return smem_u32(&sh.k_full[0]) + 8 * s; };
    auto bar_k_empty = [&](int s) { return smem_u32(&sh.k_empty[0]) + 8 * s; };
    auto bar_v8 = [&](int s) { return smem_u32(&sh.v8_full[0]) + 8 * s; };
    auto bar_v8_empty = [&](int s) { return smem_u32(&sh.v8_empty[0]) + 8 * s; };
    const int pages = kTileKeys >> p.page_log2;          // of a tile: 1 to 8
    const int zero_row = p.num_pages * p.Hkv * p.page;   // beyond the pool: reads as zero
    Cursor ahead = now;                                  // the tile whose page numbers are under way
    // A page that begins at or behind the sequence's end counts as one that is not there, whatever the table has for it: it may be given out
    // ahead or be another sequence's, and its scales must not enter the tile's largest.
    auto fetch_ids = [&](const Cursor &c) {
        if (c.c >= c.end || lane >= pages) return -1;
        const int at = c.c * pages + lane;
        return (unsigned)at << p.page_log2 < (unsigned)c.keys ? __ldg(p.table + (size_t)c.b * p.max_pages + at) : -1;
    };
    auto step = [&] {
        if (++ahead.c < ahead.end || ahead.left == 0) return;
        ahead.next(p);
    };
    int ids_next = fetch_ids(ahead), tile = 0;
    for (; err == 0;) {
        for (; now.c < now.end; ++now.c, ++tile) {
            const int ids = ids_next;
            step();
            ids_next = fetch_ids(ahead);
            const int ks = tile % S::kKSlots, kuse = tile / S::kKSlots, vs = tile % S::kVSlots, vuse = tile / S::kVSlots;
            const bool there = lane < pages && ids >= 0 && ids < p.num_pages;
            const int row = there ? (ids * p.Hkv + now.h) * p.page : zero_row;
            if (kuse > 0 && !__all_sync(0xFFFFFFFFu, wait_awake(bar_k_empty(ks), (kuse - 1) & 1))) { err = kErrTileSlot; break; }
            if (lane == 0) mbar_expect_tx(bar_k(ks), S::kTileBytes);
            __syncwarp();
            if (lane < pages) tma_load_2d(base + S::kK + ks * S::kTileBytes + lane * p.page * D, &tm_k, bar_k(ks), 0, row);
            const int id = __shfl_sync(0xFFFFFFFFu, ids, (lane & 7) * pages >> 3);
            if (lane < 16) {
                float *to = reinterpret_cast<float *>(sh.scale[ks]) + lane;
                if (id >= 0 && id < p.num_pages)
                    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(smem_u32(to)), "l"(p.scale[lane >> 3] + (size_t)id * p.Hkv + now.h) : "memory");
                else {
                    *to = -1.f;
                    __threadfence_block();       // (the arrival below speaks for the copies only)
                }
            }
            asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(bar_k(ks)) : "memory");
            if (vuse > 0 && !__all_sync(0xFFFFFFFFu, wait_awake(bar_v8_empty(vs), (vuse - 1) & 1))) { err = kErrTileSlot; break; }
            if (lane == 0) mbar_expect_tx(bar_v8(vs), S::kTileBytes);
            __syncwarp();
            if (lane < pages) tma_load_2d(base + S::kV8 + vs * S::kTileBytes + lane * p.page * D, &tm_v, bar_v8(vs), 0, row);
        }
        if (err != 0 || now.left == 0) break;
        now.next(p);
    }
    if (lane == 0) write_record<D>(p, split, now, err == 0);
}
