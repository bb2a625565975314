// Attention of new tokens over a paged, quantized cache: the kernel for many rows per KV head (chunks of prompts, drafts under
// grouped queries).  The formulas are those of chunk_attention.cu; here a row's work is enough for the tensor cores to bound it.
//
// An item is 128 or 256 rows (TILES tiles of 128) of one KV head.  Roles of a CTA's warps, handing tiles of 128 tokens on through
// mbarriers:
//   producers (8 warps)  dequantize keys and values into shared memory, binary16 in the 128-byte swizzle, once for all rows of the
//                        item: a thread takes 16 channels of four tokens of one group of keys, whose scales it holds.
//   products (1 thread)  S = Q K^T into tensor memory, then O += P V with P taken from tensor memory; per tile of rows in the order
//                        PV(j), QK(j + 1), so that the scores of one tile are made while the other tile's warps work on theirs.
//   softmax (4 warps a tile)  a thread owns a row: maximum, weights 2^(c s - m + 8), written over its scores as binary16, and the
//                        denominator.  The sum in tensor memory is rescaled only when the maximum has grown by more than 2^6
//                        (weights then reach 2^14, within binary16).
// Channels stand in the order that the dequantization leaves them in (the two codes 16 bits apart in a word are neighbours); the
// queries are stored the same way and the result is put in order when it is written.
// Magnitudes beyond binary16 are noticed on the way, and the segment is done again with bf16 operands.
// 2048 new tokens over 8192 cached ones, 32 / 8 heads of 2 bits: 484 us, 640 TFLOP/s.  The products, the exponentials and
// shared memory at its 128 bytes a cycle each take 2048 cycles for 256 rows and a tile, and do not overlap in full (5450); with four producer warps it took 561 us.
#include "chunk_attention.cuh"

namespace {

constexpr int D = SQUAT_D, T = 128;                  // tokens of a tile
constexpr float P_SHIFT = 8.0f, GROW = 6.0f;
constexpr int OPERAND = T * D * 2;                   // bytes of a tile of 128 rows in shared memory: two halves of 64 channels

template <int TILES>
struct Plan {
    static constexpr int ROWS = 128 * TILES, STAGES = TILES, SOFT = 128 * TILES, PRODUCERS = 256, THREADS = SOFT + PRODUCERS + 128;
    static constexpr int CTAS = TILES == 2 ? 1 : 2;  // to an SM
    static constexpr int TMEM = 256 * TILES;         // columns: scores (and weights) of each tile, then sums of each tile
    // registers of a thread at launch, and of the roles' threads after it
    static constexpr int LAUNCH_REGS = TILES == 2 ? 96 : 64, SOFT_REGS = TILES == 2 ? 136 : 96, PRODUCER_REGS = TILES == 2 ? 80 : 64, PRODUCT_REGS = TILES == 2 ? 48 : 32;
    static_assert(TILES * SOFT_REGS + 2 * PRODUCER_REGS + PRODUCT_REGS == (TILES + 3) * LAUNCH_REGS, "more registers than the block is launched with");
    static constexpr size_t SMEM = 1024 + (size_t)(TILES + 2 * STAGES) * OPERAND;
};

// 128 rows of 64 elements of 16 bits, 128-byte swizzle, groups of 8 rows 1024 bytes apart.  Contraction along the row (queries,
// keys), or across rows (values: 64 channels per row, the next 64 OPERAND / 2 further on).
__device__ __forceinline__ u64 rows_desc(unsigned addr) { return (u64)((addr & 0x3FFFF) >> 4) | ((u64)1 << 16) | ((u64)(1024 >> 4) << 32) | (1ull << 46) | (2ull << 61); }
__device__ __forceinline__ u64 columns_desc(unsigned addr) { return (u64)((addr & 0x3FFFF) >> 4) | ((u64)((OPERAND / 2) >> 4) << 16) | ((u64)(1024 >> 4) << 32) | (1ull << 46) | (2ull << 61); }
// float32 accumulator, both operands binary16 or both bf16, M = N = 128, B with the contraction along its rows or across them
__device__ __forceinline__ unsigned idesc_16(bool bf, bool b_across)
{
    return (1u << 4) | (bf ? (1u << 7) | (1u << 10) : 0u) | (b_across ? 1u << 16 : 0u) | ((128u >> 3) << 17) | ((128u >> 4) << 24);
}
__device__ __forceinline__ void mma_ss(unsigned d, u64 a, u64 b, unsigned idesc, unsigned accumulate)
{
    asm volatile("{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}" ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void mma_ts(unsigned d, unsigned a, u64 b, unsigned idesc, unsigned accumulate)
{
    asm volatile("{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}" ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void tmem_ld32(unsigned addr, float (&r)[32])
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
                 : "=f"(r[0]), "=f"(r[1]), "=f"(r[2]), "=f"(r[3]), "=f"(r[4]), "=f"(r[5]), "=f"(r[6]), "=f"(r[7]), "=f"(r[8]), "=f"(r[9]), "=f"(r[10]), "=f"(r[11]), "=f"(r[12]), "=f"(r[13]),
                   "=f"(r[14]), "=f"(r[15]), "=f"(r[16]), "=f"(r[17]), "=f"(r[18]), "=f"(r[19]), "=f"(r[20]), "=f"(r[21]), "=f"(r[22]), "=f"(r[23]), "=f"(r[24]), "=f"(r[25]), "=f"(r[26]),
                   "=f"(r[27]), "=f"(r[28]), "=f"(r[29]), "=f"(r[30]), "=f"(r[31])
                 : "r"(addr) : "memory");
}
__device__ __forceinline__ void tmem_st32(unsigned addr, const float (&r)[32])
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};"
                 ::"r"(addr), "f"(r[0]), "f"(r[1]), "f"(r[2]), "f"(r[3]), "f"(r[4]), "f"(r[5]), "f"(r[6]), "f"(r[7]), "f"(r[8]), "f"(r[9]), "f"(r[10]), "f"(r[11]), "f"(r[12]), "f"(r[13]), "f"(r[14]),
                   "f"(r[15]), "f"(r[16]), "f"(r[17]), "f"(r[18]), "f"(r[19]), "f"(r[20]), "f"(r[21]), "f"(r[22]), "f"(r[23]), "f"(r[24]), "f"(r[25]), "f"(r[26]), "f"(r[27]), "f"(r[28]), "f"(r[29]),
                   "f"(r[30]), "f"(r[31]) : "memory");
}
__device__ __forceinline__ void tmem_st16(unsigned addr, const uint32_t (&r)[16])
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
                 ::"r"(addr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]),
                   "r"(r[15]) : "memory");
}
__device__ __forceinline__ void tmem_ld_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void mbar_init(unsigned bar, unsigned count) { asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory"); }
__device__ __forceinline__ void mbar_arrive(unsigned bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory"); }
__device__ __forceinline__ void fence_async_smem() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// What a CTA's roles share besides the operands
template <int TILES>
struct Shared {
    u64 k_full[Plan<TILES>::STAGES], k_empty[Plan<TILES>::STAGES], v_full[Plan<TILES>::STAGES], v_empty[Plan<TILES>::STAGES];
    u64 s_full[TILES], p_full[TILES], o_full[TILES];
    unsigned tmem;
    int failed;                                      // a bounded wait ran out: no more waits, the results are not valid
    int wide;                                        // binary16 is too narrow for the segment
    int odd_first, odd_last;                         // range of rows in full precision that hold infinities or NaN among their values
    int v_top, k_top, q_top, q_low;                  // largest magnitudes, as float bits; q_low: the smallest of the rows' largest
    ChunkShared place;
};

// Waits at most once the limit's time in all: after one wait that ran out, none is taken any more.
__device__ __forceinline__ void wait_for(u64 &bar, unsigned parity, int &failed, unsigned *status)
{
    if (*(volatile int *)&failed) return;
    if (mbar_wait(smem_u32(&bar), parity)) return;
    failed = 1;
    atomicOr(status, SQUAT_FLAG_DEVICE_TIMEOUT);
}

// 16 channels of a token in the operand: two 16-byte pieces.  (Eight lanes hold four units of two neighbouring tokens: distinct banks.)
__device__ __forceinline__ void store_unit(unsigned char *operand, int row, int unit, const uint32_t (&r)[8])
{
    unsigned char *base = operand + unit / 4 * (OPERAND / 2) + row * 128;
    const int c = unit % 4 * 2 ^ (row & 7);
    *reinterpret_cast<uint4 *>(base + (c << 4)) = make_uint4(r[0], r[1], r[2], r[3]);
    *reinterpret_cast<uint4 *>(base + ((c ^ 1) << 4)) = make_uint4(r[4], r[5], r[6], r[7]);
}

// 16 bf16 numbers, as loaded, in the operand's order
template <int BITS>
__device__ __forceinline__ void unit_of_bf16(const uint32_t (&x)[8], bool bf, uint32_t (&r)[8])
{
#pragma unroll
    for (int m = 0; m < 8; ++m) {
        const uint32_t v = BITS == 2 ? pair16(x[m / 2], x[4 + m / 2], m) : pair16(x[m / 4 * 4 + m % 4 / 2], x[m / 4 * 4 + 2 + m % 4 / 2], m);
        r[m] = bf ? v : bf16_pair_to_f16(v);
    }
}

// A producer's part of a tile of cached tokens: four tokens, eight apart, of 32 (one page, one group of keys), 16 channels each.  Keys
// and values are asked for a tile ahead: the keys of the next tile while this one's values are made, and the other way round.
constexpr int UNITS = 4, APART = 8;
template <int BITS, int G, bool M16>
struct Producer {
    static constexpr int ROW = D * BITS / 8, NG = D / G;
    const CodeBias<BITS> bias;
    int sub, unit;                                   // the first of its tokens, its channels
    uint32_t code[2][UNITS][BITS / 2];                   // keys, values
    uint4 ks[M16 ? 2 : 4], kz[M16 ? 2 : 4];          // the unit's scales and zero-points (keys)
    float vs[UNITS], vz[UNITS];                              // the tokens' (values)

    __device__ __forceinline__ void load_codes(int side, const unsigned char *codes, long long tok)
    {
        const unsigned char *from = codes + (tok + sub) * ROW + unit * (2 * BITS);
#pragma unroll
        for (int i = 0; i < UNITS; ++i) {
            if (BITS == 2) code[side][i][0] = __ldg(reinterpret_cast<const uint32_t *>(from + APART * i * ROW));
            else {
                const uint2 v = __ldg(reinterpret_cast<const uint2 *>(from + APART * i * ROW));
                code[side][i][0] = v.x; code[side][i][BITS / 2 - 1] = v.y;
            }
        }
    }
    __device__ __forceinline__ void load_keys(const PagePool &pool, long long tok)
    {
        load_codes(0, pool.kc, tok);
        const long long at = (tok / G * D + 16 * unit) * (M16 ? 2 : 4) / 16;
#pragma unroll
        for (int i = 0; i < (M16 ? 2 : 4); ++i) {
            ks[i] = __ldg(static_cast<const uint4 *>(pool.ks) + at + i);
            kz[i] = __ldg(static_cast<const uint4 *>(pool.kz) + at + i);
        }
    }
    __device__ __forceinline__ void load_values(const PagePool &pool, long long tok)
    {
        load_codes(1, pool.vc, tok);
        const long long at = (tok + sub) * NG + 16 * unit / G;
#pragma unroll
        for (int i = 0; i < UNITS; ++i) {
            vs[i] = M16 ? __half2float(__ldg(static_cast<const __half *>(pool.vs) + at + APART * i * NG)) : __ldg(static_cast<const float *>(pool.vs) + at + APART * i * NG);
            vz[i] = M16 ? __half2float(__ldg(static_cast<const __half *>(pool.vz) + at + APART * i * NG)) : __ldg(static_cast<const float *>(pool.vz) + at + APART * i * NG);
        }
    }
    // register m of a unit holds channels lo_of(m) and lo_of(m) + HALF
    static constexpr int HALF = BITS == 2 ? 8 : 4;
    __device__ __forceinline__ static constexpr int lo_of(int m) { return BITS == 2 ? m : m / 4 * 8 + m % 4; }
    __device__ __forceinline__ __half2 pair(int side, int i, int m) const { return BITS == 2 ? bias.codes(code[side][i][0], m) : bias.codes(code[side][i][m / 4 * (BITS / 2 - 1)], m % 4); }
    __device__ __forceinline__ float code_at(int side, int i, int c) const
    {
        return BITS == 2 ? code_float<BITS>(code[side][i][0], c) : code_float<BITS>(code[side][i][c / 8 * (BITS / 2 - 1)], c % 8);
    }
    __device__ __forceinline__ static float meta(const uint4 *x, int c)
    {
        const uint4 &v = x[c / (M16 ? 8 : 4)];
        const int w = M16 ? c % 8 / 2 : c % 4;
        const uint32_t u = w == 0 ? v.x : w == 1 ? v.y : w == 2 ? v.z : v.w;
        return M16 ? __half2float(__ushort_as_half((unsigned short)(u >> (16 * (c & 1))))) : __uint_as_float(u);
    }
    __device__ __forceinline__ static uint32_t meta_word(const uint4 *x, int c)      // (binary16) channels c, c + 1
    {
        const uint4 &v = x[c / 8];
        const int w = c % 8 / 2;
        return w == 0 ? v.x : w == 1 ? v.y : w == 2 ? v.z : v.w;
    }
    __device__ __forceinline__ static __half2 meta_pair(const uint4 *x, int m)
    {
        const int lo = lo_of(m);
        if (M16) return as_half2(pair16(meta_word(x, lo & ~1), meta_word(x, (lo + HALF) & ~1), lo));
        return __floats2half2_rn(meta(x, lo), meta(x, lo + HALF));
    }
    template <bool BF>
    __device__ __forceinline__ void store_keys(unsigned char *to, int row, __half2 &s_top, __half2 &z_top) const
    {
        if (!BF) {
            __half2 s2[8], z2[8];
#pragma unroll
            for (int m = 0; m < 8; ++m) {
                s2[m] = meta_pair(ks, m);
                z2[m] = meta_pair(kz, m);
                s_top = __hmax2(s_top, __habs2(s2[m]));
                z_top = __hmax2(z_top, __habs2(z2[m]));
            }
#pragma unroll
            for (int i = 0; i < UNITS; ++i) {
                uint32_t y[8];
#pragma unroll
                for (int m = 0; m < 8; ++m) y[m] = as_u32(__hfma2(pair(0, i, m), s2[m], z2[m]));
                store_unit(to, row + APART * i, unit, y);
            }
        } else {
#pragma unroll
            for (int i = 0; i < UNITS; ++i) {
                uint32_t y[8];
#pragma unroll
                for (int m = 0; m < 8; ++m) {
                    const int lo = lo_of(m), hi = lo + HALF;
                    y[m] = pack16<true>(fmaf(code_at(0, i, lo), meta(ks, lo), meta(kz, lo)), fmaf(code_at(0, i, hi), meta(ks, hi), meta(kz, hi)));
                }
                store_unit(to, row + APART * i, unit, y);
            }
        }
    }
    template <bool BF>
    __device__ __forceinline__ void store_values(unsigned char *to, int row, float &s_top, float &z_top) const
    {
#pragma unroll
        for (int i = 0; i < UNITS; ++i) {
            uint32_t y[8];
            if (!BF) {
                const __half2 s2 = __float2half2_rn(vs[i]), z2 = __float2half2_rn(vz[i]);
                s_top = fmaxf(s_top, fabsf(vs[i]));      // (as stored: binary16 may make zeros of them)
                z_top = fmaxf(z_top, fabsf(vz[i]));
#pragma unroll
                for (int m = 0; m < 8; ++m) y[m] = as_u32(__hfma2(pair(1, i, m), s2, z2));
            } else {
#pragma unroll
                for (int m = 0; m < 8; ++m) y[m] = pack16<true>(fmaf(code_at(1, i, lo_of(m)), vs[i], vz[i]), fmaf(code_at(1, i, lo_of(m) + HALF), vs[i], vz[i]));
            }
            store_unit(to, row + APART * i, unit, y);
        }
    }
};

// A CTA's way along the line of items.
struct Walk {
    ChunkPlace pl;
    ChunkSeq sq;
    long long at, end;
};
struct Segment {                                     // tiles [ta, tb) of an item
    int ta, tb, n, tiles, steps, row0, n_rows, last, ct, most;
};
template <int ROWS>
__device__ __forceinline__ bool walk_segment(const ChunkParams &p, Walk &w, Segment &sg)
{
    while (w.at < w.end) {
        sg.tiles = chunk_tiles<ROWS, T>(p, w.sq, w.pl.qt);
        const int begin = w.pl.at, stop = (int)min((long long)p.start + sg.tiles, begin + (w.end - w.at));
        sg.ta = max(begin - p.start, 0);
        sg.tb = max(stop - p.start, 0);
        sg.n = sg.tb - sg.ta;
        sg.steps = stop - begin;
        if (sg.n > 0) {
            sg.row0 = w.pl.qt * ROWS;
            sg.n_rows = min(ROWS, w.sq.nq * p.qpk - sg.row0);
            sg.last = sg.row0 + sg.n_rows - 1;
            sg.ct = (w.sq.cached + T - 1) / T;
            sg.most = chunk_sees(p, w.sq, sg.last / p.qpk);
            return true;
        }
        w.at += sg.steps;
        if (w.at < w.end) chunk_next<ROWS>(p, w.pl, w.sq);
    }
    return false;
}
template <int ROWS>
__device__ __forceinline__ void walk_on(const ChunkParams &p, Walk &w, const Segment &sg)
{
    w.at += sg.steps;
    if (w.at < w.end) chunk_next<ROWS>(p, w.pl, w.sq);
}
// All roles: the segment begins (its queries may be stored), its queries are there, its sums have been taken; whether it is done again in bf16.
template <int TILES>
__device__ __forceinline__ void segment_begins(Shared<TILES> &sh)
{
    if (threadIdx.x == 0) {
        sh.wide = 0;
        sh.odd_first = 0x7fffffff;
        sh.odd_last = -1;
        sh.v_top = sh.k_top = sh.q_top = 0;
        sh.q_low = 0x7f800000;
    }
    __syncthreads();
}
template <int TILES>
__device__ __forceinline__ bool too_wide(const ChunkParams &p, Shared<TILES> &sh, bool bf)
{
    if (bf) return false;
    const float q_top = __int_as_float(*(volatile int *)&sh.q_top), q_low = __int_as_float(*(volatile int *)&sh.q_low);
    const float k_top = __int_as_float(*(volatile int *)&sh.k_top), v_top = __int_as_float(*(volatile int *)&sh.v_top);
    return *(volatile int *)&sh.wide || !(k_top < 4096.0f) || !(v_top < 65000.0f) || (v_top < 0x1p-8f && v_top > 0.0f) || chunk_too_low(p, false, q_top, q_low, k_top);
}
template <int TILES>
__device__ __forceinline__ bool segment_again(const ChunkParams &p, Shared<TILES> &sh, bool bf)
{
    __syncthreads();
    tc_fence_after();
    const bool again = too_wide(p, sh, bf);
    __syncthreads();
    return again;
}
template <int N>
__device__ __forceinline__ void more_registers() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }
template <int N>
__device__ __forceinline__ void fewer_registers() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }

// 64 columns of a row's scores at a time; past the first `lim` of the tile they are -infinity.  (Loops of 64 columns, and the rare
// cases apart: the roles' loops together have to stay within the instruction cache, or fetching them is what takes the time.)
template <bool MASKED>
__device__ __forceinline__ void load_scores(unsigned s_addr, int half, int lim, float (&x)[32], float (&y)[32])
{
    tmem_ld32(s_addr + 64 * half, x);
    tmem_ld32(s_addr + 64 * half + 32, y);
    tmem_ld_wait();
    if (MASKED) {
        const int left = lim - 64 * half;
#pragma unroll
        for (int i = 0; i < 32; ++i) {
            x[i] = i < left ? x[i] : -INFINITY;
            y[i] = i + 32 < left ? y[i] : -INFINITY;
        }
    }
}
template <bool MASKED>
__device__ __forceinline__ float row_max(unsigned s_addr, int lim)
{
    float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll 1
    for (int half = 0; half < 2; ++half) {
        float x[32], y[32];
        load_scores<MASKED>(s_addr, half, lim, x, y);
#pragma unroll
        for (int i = 0; i < 32; ++i) mx[i & 3] = fmaxf(fmaxf(mx[i & 3], x[i]), y[i]);
    }
    return fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3]));
}
// The weights 2^(c s + base), written over the scores; returns their sum.
template <bool MASKED, bool BF>
__device__ __forceinline__ float row_weights(unsigned s_addr, int lim, float c, float base)
{
    const u64 c2 = pack2(c, c), base2 = pack2(base, base);
    u64 sum2[2] = {0, 0};
#pragma unroll 1
    for (int half = 0; half < 2; ++half) {
        float x[32], y[32];
        load_scores<MASKED>(s_addr, half, lim, x, y);
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            uint32_t w[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                float y0, y1;
                unpack2(ffma2(k ? pack2(y[2 * i], y[2 * i + 1]) : pack2(x[2 * i], x[2 * i + 1]), c2, base2), y0, y1);
                y0 = exp2_fast(y0);
                y1 = exp2_fast(y1);
                sum2[i & 1] = fadd2(sum2[i & 1], pack2(y0, y1));
                w[i] = pack16<BF>(y0, y1);
            }
            tmem_st16(s_addr + 32 * half + 16 * k, w);
        }
    }
    sum2[0] = fadd2(sum2[0], sum2[1]);
    return lo_of(sum2[0]) + hi_of(sum2[0]);
}

// A segment's tiles for the rows of row tile t.
template <int TILES, bool BF>
__device__ __forceinline__ void softmax_tiles(const ChunkParams &p, const Segment &sg, Shared<TILES> &sh, int cached, int sees, int t, unsigned turns, unsigned s_addr, unsigned o_addr, float &m, float &l)
{
    const float c = p.scale_log2;
    m = -INFINITY;
    l = 0.0f;
#pragma unroll 1
    for (int j = 0; j < sg.n; ++j) {
        const int tile = sg.ta + j, lim = tile < sg.ct ? cached - tile * T : sees - (tile - sg.ct) * T;
        const bool masked = __any_sync(0xffffffffu, lim < T);
        wait_for(sh.s_full[t], (turns + j) & 1, sh.failed, p.status);
        tc_fence_after();
        const float mx = c * (masked ? row_max<true>(s_addr, lim) : row_max<false>(s_addr, lim));
        if (j == 0) m = mx;
        else if (__any_sync(0xffffffffu, mx > m + GROW)) {
            const float top = mx > m + GROW ? mx : m, use = top == -INFINITY ? 0.0f : top, f = exp2_fast(m - use);
            m = top;
            l *= f;
#pragma unroll 1
            for (int b = 0; b < 4; ++b) {
                float x[32];
                tmem_ld32(o_addr + 32 * b, x);
                tmem_ld_wait();
#pragma unroll
                for (int i = 0; i < 32; ++i) x[i] *= f;
                tmem_st32(o_addr + 32 * b, x);
            }
        }
        const float base = P_SHIFT - (m == -INFINITY ? 0.0f : m);
        l += masked ? row_weights<true, BF>(s_addr, lim, c, base) : row_weights<false, BF>(s_addr, lim, c, base);
        tmem_st_wait();
        tc_fence_before();
        mbar_arrive(smem_u32(&sh.p_full[t]));
    }
}

template <int BITS, int TILES>
__device__ __forceinline__ void softmax_role(const ChunkParams &p, Walk w, Shared<TILES> &sh, unsigned char *q_sm, unsigned tmem)
{
    using S = Plan<TILES>;
    const int tid = threadIdx.x, warp = tid >> 5, t = warp / 4, r = tid;
    unsigned turns = 0, segments = 0;                // scores of the row tile, and segments, so far
    Segment sg;
    while (walk_segment<S::ROWS>(p, w, sg)) {
        for (bool bf = false;; bf = true) {
            segment_begins(sh);
            {
                float top = 0.0f;
#pragma unroll
                for (int u = 0; u < 8; ++u) {
                    uint32_t x[8] = {0, 0, 0, 0, 0, 0, 0, 0}, y[8];
                    if (r < sg.n_rows) {
                        const __nv_bfloat16 *from = p.q + (long long)(w.sq.q0 + (sg.row0 + r) / p.qpk) * p.qt + (long long)(w.pl.h * p.qpk + (sg.row0 + r) % p.qpk) * p.qh + 16 * u;
                        const uint4 a = ldg128(from), b = ldg128(from + 8);
                        x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
                    }
#pragma unroll
                    for (int i = 0; i < 8; ++i) top = fmaxf(top, fmaxf(fabsf(bf16lo_to_f32(x[i])), fabsf(bf16hi_to_f32(x[i]))));
                    unit_of_bf16<BITS>(x, bf, y);
                    unsigned char *base = q_sm + r / 128 * OPERAND + u / 4 * (OPERAND / 2) + r % 128 * 128;
                    *reinterpret_cast<uint4 *>(base + ((u % 4 * 2 ^ (r & 7)) << 4)) = make_uint4(y[0], y[1], y[2], y[3]);
                    *reinterpret_cast<uint4 *>(base + (((u % 4 * 2 + 1) ^ (r & 7)) << 4)) = make_uint4(y[4], y[5], y[6], y[7]);
                }
                if (!(top < 4096.0f)) sh.wide = 1;
                const float q_top = warp_max(top), q_low = warp_min(top > 0.0f ? top : INFINITY);
                if (tid % 32 == 0) {
                    atomicMax(&sh.q_top, __float_as_int(q_top));
                    atomicMin(&sh.q_low, __float_as_int(q_low));
                }
                fence_async_smem();
            }
            __syncthreads();
            const unsigned s_addr = tmem + 128 * t + ((unsigned)(warp % 4 * 32) << 16), o_addr = tmem + 128 * (TILES + t) + ((unsigned)(warp % 4 * 32) << 16);
            const int sees = chunk_sees(p, w.sq, min(sg.row0 + r, sg.last) / p.qpk);
            float m, l;
            if (!bf) softmax_tiles<TILES, false>(p, sg, sh, w.sq.cached, sees, t, turns, s_addr, o_addr, m, l);
            else softmax_tiles<TILES, true>(p, sg, sh, w.sq.cached, sees, t, turns, s_addr, o_addr, m, l);
            wait_for(sh.o_full[t], segments & 1, sh.failed, p.status);
            tc_fence_after();
            if (!too_wide(p, sh, bf)) {                 // (known: the last tile was handed on after it)
                const bool whole = sg.ta == 0 && sg.tb == sg.tiles;
                const long long slot = 2LL * blockIdx.x + (sg.ta == 0 ? 1 : 0);
                const int row = sg.row0 + r, q_row = w.sq.q0 + row / p.qpk, hq = w.pl.h * p.qpk + row % p.qpk;
                const float inv = l == 0.0f ? 0.0f : 1.0f / l;
                const int odd_first = max(sh.odd_first, (max(sg.ta, sg.ct) - sg.ct) * T), odd_last = min(sh.odd_last, sees - 1);
#pragma unroll 1
                for (int b = 0; b < 4; ++b) {
                    float x[32];
                    __syncwarp();
                    tmem_ld32(o_addr + 32 * b, x);
                    tmem_ld_wait();
                    if (r >= sg.n_rows) continue;
                    float y[32];                 // in the order of the channels
#pragma unroll
                    for (int i = 0; i < 32; ++i) {
                        const int e = i % 16, at_reg = BITS == 2 ? 2 * (e % 8) + e / 8 : e / 8 * 8 + 2 * (e % 4) + e % 8 / 4;
                        y[i] = l == 0.0f ? 0.0f : x[i / 16 * 16 + at_reg];
                    }
                    for (int u = odd_first; u <= odd_last; ++u) {       // rare: infinities and NaN that the row sees
                        const __nv_bfloat16 *v = p.v_new + (long long)(w.sq.k0 + u) * p.vnt + (long long)w.pl.h * p.vnh + 32 * b;
#pragma unroll
                        for (int i = 0; i < 32; ++i) {
                            const float o = __bfloat162float(v[i]);
                            if (!(fabsf(o) < INFINITY)) y[i] += o;
                        }
                    }
                    if (whole) {
                        uint32_t w[16];
#pragma unroll
                        for (int i = 0; i < 16; ++i) w[i] = pack16<true>(y[2 * i] * inv, y[2 * i + 1] * inv);
                        uint4 *to = reinterpret_cast<uint4 *>(p.out + (long long)q_row * p.ot + (long long)hq * p.oh + 32 * b);
#pragma unroll
                        for (int i = 0; i < 4; ++i) to[i] = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
                    } else {
                        float4 *to = reinterpret_cast<float4 *>(p.part + (slot * S::ROWS + r) * D + 32 * b);
#pragma unroll
                        for (int i = 0; i < 8; ++i) to[i] = make_float4(y[4 * i], y[4 * i + 1], y[4 * i + 2], y[4 * i + 3]);
                    }
                }
                if (r < sg.n_rows) {
                    if (!whole) *reinterpret_cast<float2 *>(p.ml + (slot * S::ROWS + r) * 2) = make_float2(m, l);
                    else if (p.lse) p.lse[(long long)q_row * p.Hq + hq] = l == 0.0f ? -INFINITY : (m - P_SHIFT + log2f(l)) * 0.6931471805599453f;
                }
            }
            tc_fence_before();
            turns += sg.n;
            ++segments;
            if (!segment_again(p, sh, bf)) break;
        }
        walk_on<S::ROWS>(p, w, sg);
    }
}

// A segment's tiles of keys and values.
template <int BITS, int G, bool M16, int TILES, bool BF>
__device__ __forceinline__ void producer_tiles(const ChunkParams &p, const Walk &w, const Segment &sg, Shared<TILES> &sh, Producer<BITS, G, M16> &pr, int group32, unsigned kv,
                                               unsigned char *k_sm, unsigned char *v_sm)
{
    using S = Plan<TILES>;
    const int row0_sm = 32 * group32 + pr.sub;
    // the first of the thread's 32 tokens of a tile in the pool; -1: past the cached tokens, or on a page outside the pool (keys and
    // values of zero in their place)
    auto place = [&](int t) -> long long {
        const int tk = t * T + 32 * group32;
        if (t >= min(sg.tb, sg.ct) || tk >= w.sq.cached) return -1;
        const int pg = tk / p.pool.page_tokens;
        const int page = __ldg(p.page_table + (long long)w.pl.seq * p.table_stride + pg);
        if ((unsigned)page >= (unsigned)p.pool.n_pages) {
            atomicOr(p.status, SQUAT_FLAG_PAGES);
            return -1;
        }
        return (long long)page * p.pool.page_stride + (long long)w.pl.h * p.pool.head_stride + (tk - pg * p.pool.page_tokens);
    };
    __half2 ks_top = __float2half2_rn(0.0f), kz_top = ks_top;
    float k_top = 0.0f, v_top = 0.0f, vs_top = 0.0f, vz_top = 0.0f;
    // what the segment's magnitudes were: before the last tile is handed on, so that who waits for its sums knows them
    auto publish = [&]() {
        if (BF) return;
        constexpr float L = float((1 << BITS) - 1);
        auto top = [](__half2 x) { const float2 f = __half22float2(x); return fmaxf(f.x, f.y); };
        atomicMax(&sh.k_top, __float_as_int(fmaxf(fmaf(L, top(ks_top), top(kz_top)), k_top)));
        atomicMax(&sh.v_top, __float_as_int(fmaxf(fmaf(L, vs_top, vz_top), v_top)));
    };
    long long tok = place(sg.ta), next = place(sg.ta + 1);
    if (tok >= 0) {
        pr.load_keys(p.pool, tok);
        pr.load_values(p.pool, tok);
    }
#pragma unroll 1
    for (int j = 0; j < sg.n; ++j) {
        const int tile = sg.ta + j, stage = (kv + j) % S::STAGES;
        const unsigned parity = (((kv + j) / S::STAGES) & 1) ^ 1;
        unsigned char *k_to = k_sm + stage * OPERAND, *v_to = v_sm + stage * OPERAND;
        if (tile < sg.ct) {
            const uint32_t zero[8] = {0, 0, 0, 0, 0, 0, 0, 0};
            wait_for(sh.k_empty[stage], parity, sh.failed, p.status);
            if (tok >= 0) pr.template store_keys<BF>(k_to, row0_sm, ks_top, kz_top);
            else
#pragma unroll
                for (int i = 0; i < UNITS; ++i) store_unit(k_to, row0_sm + APART * i, pr.unit, zero);
            fence_async_smem();
            mbar_arrive(smem_u32(&sh.k_full[stage]));
            if (next >= 0) pr.load_keys(p.pool, next);
            wait_for(sh.v_empty[stage], parity, sh.failed, p.status);
            if (tok >= 0) pr.template store_values<BF>(v_to, row0_sm, vs_top, vz_top);
            else
#pragma unroll
                for (int i = 0; i < UNITS; ++i) store_unit(v_to, row0_sm + APART * i, pr.unit, zero);
            if (j == sg.n - 1) publish();
            fence_async_smem();
            mbar_arrive(smem_u32(&sh.v_full[stage]));
            if (next >= 0) pr.load_values(p.pool, next);
            tok = next;
            next = place(tile + 2);
        } else {
            // rows in full precision
            const int u0 = (tile - sg.ct) * T + row0_sm;
#pragma unroll
            for (int side = 0; side < 2; ++side) {
                const __nv_bfloat16 *src = side == 0 ? p.k_new : p.v_new;
                const long long st = side == 0 ? p.knt : p.vnt, shd = side == 0 ? p.knh : p.vnh;
                if (side == 0) wait_for(sh.k_empty[stage], parity, sh.failed, p.status);
                else wait_for(sh.v_empty[stage], parity, sh.failed, p.status);
#pragma unroll 2
                for (int i = 0; i < UNITS; ++i) {
                    const int u = u0 + APART * i;
                    uint32_t x[8] = {0, 0, 0, 0, 0, 0, 0, 0}, y[8];
                    if (u < sg.most) {
                        const __nv_bfloat16 *from = src + (long long)(w.sq.k0 + u) * st + (long long)w.pl.h * shd + 16 * pr.unit;
                        const uint4 a = ldg128(from), b = ldg128(from + 8);
                        x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
                    }
                    bool odd = false;
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        if (side == 1 && bf16_pair_not_finite(x[e])) {     // a row that does not see it must not meet it
                            odd = true;
                            if ((x[e] & 0x7f80u) == 0x7f80u) x[e] &= 0xffff0000u;
                            if ((x[e] & 0x7f800000u) == 0x7f800000u) x[e] &= 0x0000ffffu;
                        }
                        const float lo = fabsf(bf16lo_to_f32(x[e])), hi = fabsf(bf16hi_to_f32(x[e]));
                        if (side == 0) k_top = fmaxf(k_top, fmaxf(lo < INFINITY ? lo : 0.0f, hi < INFINITY ? hi : 0.0f));
                        else v_top = fmaxf(v_top, fmaxf(lo, hi));
                    }
                    if (odd) {
                        atomicMin(&sh.odd_first, u);
                        atomicMax(&sh.odd_last, u);
                    }
                    unit_of_bf16<BITS>(x, BF, y);
                    store_unit(side == 0 ? k_to : v_to, row0_sm + APART * i, pr.unit, y);
                }
                if (side == 1 && j == sg.n - 1) publish();
                fence_async_smem();
                mbar_arrive(smem_u32(side == 0 ? &sh.k_full[stage] : &sh.v_full[stage]));
            }
        }
    }
}

template <int BITS, int G, bool M16, int TILES>
__device__ __forceinline__ void producer_role(const ChunkParams &p, Walk w, Shared<TILES> &sh, unsigned char *k_sm, unsigned char *v_sm)
{
    using S = Plan<TILES>;
    const int pt = threadIdx.x - S::SOFT, group32 = pt / 64;
    Producer<BITS, G, M16> pr;
    pr.sub = (pt >> 2 & 1) | (pt >> 4 & 1) << 1 | (pt >> 5 & 1) << 2;
    pr.unit = (pt & 3) | (pt >> 3 & 1) << 2;
    unsigned kv = 0;                                 // tiles so far
    Segment sg;
    while (walk_segment<S::ROWS>(p, w, sg)) {
        for (bool bf = false;; bf = true) {
            segment_begins(sh);
            __syncthreads();
            if (!bf) producer_tiles<BITS, G, M16, TILES, false>(p, w, sg, sh, pr, group32, kv, k_sm, v_sm);
            else producer_tiles<BITS, G, M16, TILES, true>(p, w, sg, sh, pr, group32, kv, k_sm, v_sm);
            kv += sg.n;
            if (!segment_again(p, sh, bf)) break;
        }
        walk_on<S::ROWS>(p, w, sg);
    }
}

template <int TILES>
__device__ __forceinline__ void product_role(const ChunkParams &p, Walk w, Shared<TILES> &sh, unsigned char *q_sm, unsigned char *k_sm, unsigned char *v_sm, unsigned tmem, bool issues)
{
    using S = Plan<TILES>;
    unsigned kv = 0, turns = 0;
    Segment sg;
    while (walk_segment<S::ROWS>(p, w, sg)) {
        for (bool bf = false;; bf = true) {
            segment_begins(sh);
            __syncthreads();
            if (issues) {
                const unsigned id_s = idesc_16(bf, false), id_o = idesc_16(bf, true);
                auto scores = [&](int t, int stage) {
                    const u64 a = rows_desc(smem_u32(q_sm + t * OPERAND)), b = rows_desc(smem_u32(k_sm + stage * OPERAND));
#pragma unroll
                    for (int s = 0; s < 8; ++s) {
                        const int off = (s / 4 * (OPERAND / 2) + s % 4 * 32) >> 4;
                        mma_ss(tmem + 128 * t, a + off, b + off, id_s, s > 0);
                    }
                };
                wait_for(sh.k_full[kv % S::STAGES], (kv / S::STAGES) & 1, sh.failed, p.status);
                tc_fence_after();
                if (elect_one()) {
#pragma unroll
                    for (int t = 0; t < TILES; ++t) {
                        scores(t, kv % S::STAGES);
                        tc_commit(smem_u32(&sh.s_full[t]));
                    }
                    tc_commit(smem_u32(&sh.k_empty[kv % S::STAGES]));
                }
                __syncwarp();
#pragma unroll 1
                for (int j = 0; j < sg.n; ++j) {
                    const int stage = (kv + j) % S::STAGES, next = (kv + j + 1) % S::STAGES;
#pragma unroll
                    for (int t = 0; t < TILES; ++t) {
                        if (t == 0) wait_for(sh.v_full[stage], ((kv + j) / S::STAGES) & 1, sh.failed, p.status);
                        wait_for(sh.p_full[t], (turns + j) & 1, sh.failed, p.status);
                        tc_fence_after();
                        if (elect_one()) {
                            const u64 b = columns_desc(smem_u32(v_sm + stage * OPERAND));
#pragma unroll
                            for (int s = 0; s < 8; ++s) mma_ts(tmem + 128 * (TILES + t), tmem + 128 * t + 8 * s, b + (s * 2048 >> 4), id_o, j > 0 || s > 0);
                            if (t == TILES - 1) tc_commit(smem_u32(&sh.v_empty[stage]));
                            if (j + 1 == sg.n) tc_commit(smem_u32(&sh.o_full[t]));
                        }
                        __syncwarp();
                        if (j + 1 == sg.n) continue;
                        if (t == 0) {
                            wait_for(sh.k_full[next], ((kv + j + 1) / S::STAGES) & 1, sh.failed, p.status);
                            tc_fence_after();
                        }
                        if (elect_one()) {
                            scores(t, next);
                            tc_commit(smem_u32(&sh.s_full[t]));
                            if (t == TILES - 1) tc_commit(smem_u32(&sh.k_empty[next]));
                        }
                        __syncwarp();
                    }
                }
            }
            kv += sg.n;
            turns += sg.n;
            if (!segment_again(p, sh, bf)) break;
        }
        walk_on<S::ROWS>(p, w, sg);
    }
}

template <int BITS, int G, bool M16, int TILES>
__global__ void __launch_bounds__(Plan<TILES>::THREADS, Plan<TILES>::CTAS) chunk_matrix_kernel(const __grid_constant__ ChunkParams params)
{
    using S = Plan<TILES>;
    extern __shared__ unsigned char smem_raw[];
    __shared__ Shared<TILES> sh;
    unsigned char *q_sm = smem_raw + (1024 - (smem_u32(smem_raw) & 1023)) % 1024, *k_sm = q_sm + TILES * OPERAND, *v_sm = k_sm + S::STAGES * OPERAND;
    const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0);
    constexpr int SOFT_WARPS = S::SOFT / 32, MMA_WARP = SOFT_WARPS + S::PRODUCERS / 32;
    ChunkParams p = params;
    grid_wait(p.q, p.q_start, p.cached_len, p.page_table, p.new_start, p.new_len, p.k_new, p.v_new);
    long long per, total;
    chunk_share<S::ROWS, T>(p, sh.place, per, total);
    Walk w;
    w.at = per * blockIdx.x;
    if (w.at >= total) return;
    w.end = min(w.at + per, total);
    chunk_locate<S::ROWS, T, 1>(p, sh.place, w.at, per);
    w.pl = sh.place.found[0];
    w.sq = chunk_seq(p, w.pl.seq);
    if (warp == MMA_WARP) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&sh.tmem)), "r"((unsigned)S::TMEM) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    if (tid == 0) {
        for (int i = 0; i < S::STAGES; ++i) {
            mbar_init(smem_u32(&sh.k_full[i]), S::PRODUCERS);
            mbar_init(smem_u32(&sh.v_full[i]), S::PRODUCERS);
            mbar_init(smem_u32(&sh.k_empty[i]), 1);
            mbar_init(smem_u32(&sh.v_empty[i]), 1);
        }
        for (int t = 0; t < TILES; ++t) {
            mbar_init(smem_u32(&sh.s_full[t]), 1);
            mbar_init(smem_u32(&sh.p_full[t]), 128);
            mbar_init(smem_u32(&sh.o_full[t]), 1);
        }
        sh.failed = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const unsigned tmem = __shfl_sync(0xffffffffu, sh.tmem, 0);
    // registers: the three roles' shares add up to what the block was launched with
    if (warp < SOFT_WARPS) {
        more_registers<S::SOFT_REGS>();
        softmax_role<BITS, TILES>(p, w, sh, q_sm, tmem);
    } else if (warp < MMA_WARP) {
        if (S::PRODUCER_REGS < S::LAUNCH_REGS) fewer_registers<S::PRODUCER_REGS>();
        producer_role<BITS, G, M16, TILES>(p, w, sh, k_sm, v_sm);
    } else {
        fewer_registers<S::PRODUCT_REGS>();
        product_role<TILES>(p, w, sh, q_sm, k_sm, v_sm, tmem, warp == MMA_WARP);
    }
    tc_fence_before();
    __syncthreads();
    if (warp == MMA_WARP) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"((unsigned)S::TMEM) : "memory");
}

template <int BITS, int G, bool M16, int TILES>
int launch_matrix(const ChunkParams &p, cudaStream_t st)
{
    using S = Plan<TILES>;
    static std::atomic<unsigned long long> allowed{0};
    const void *kernel = reinterpret_cast<const void *>(chunk_matrix_kernel<BITS, G, M16, TILES>);
    if (!allowed.load(std::memory_order_acquire)) {  // the roles' registers are taken out of the block's: a build with fewer would wait for them for good
        cudaFuncAttributes a;
        SQUAT_CUDA(cudaFuncGetAttributes(&a, kernel));
        if (a.numRegs != S::LAUNCH_REGS) return SQUAT_ERR_UNSUPPORTED;
    }
    const int rc = squat_allow_smem(kernel, S::SMEM, allowed);
    if (rc != SQUAT_OK) return rc;
    return squat_launch(chunk_matrix_kernel<BITS, G, M16, TILES>, p.n_workers, S::THREADS, S::SMEM, st, p);
}
template <int TILES>
int launch_matrix_tiles(const ChunkParams &p, int bits, int meta16, cudaStream_t st)
{
#define SQ_C(BB, GG) return meta16 ? launch_matrix<BB, GG, true, TILES>(p, st) : launch_matrix<BB, GG, false, TILES>(p, st)
    if (bits == 2) { if (p.G == 32) SQ_C(2, 32); if (p.G == 64) SQ_C(2, 64); SQ_C(2, 128); }
    if (p.G == 32) SQ_C(4, 32);
    if (p.G == 64) SQ_C(4, 64);
    SQ_C(4, 128);
#undef SQ_C
}

}  // namespace

int squat_launch_chunk_matrix(const ChunkParams &p, int tiles, int bits, int meta16, cudaStream_t st)
{
    return tiles == 2 ? launch_matrix_tiles<2>(p, bits, meta16, st) : launch_matrix_tiles<1>(p, bits, meta16, st);
}
