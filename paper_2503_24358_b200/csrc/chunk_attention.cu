// Attention of new tokens over a paged, quantized cache (squat_chunk_attention): the kernel for few rows per KV head (decode
// steps, drafted tokens), and the sum of an item's parts.
//
//   out_r = sum_t p_rt v_t / sum_t p_rt,   p_rt = 2^(c <q_r, k_t> - m_r),   c = softmax scale / ln 2,   m_r the running maximum
//
// The cache's bytes bound it, if the two to four instructions that a code costs can be issued meanwhile.  So nothing is
// staged for the tensor core: the operands of mma.sync m16n8k16 are made in the registers where it wants them.
//   - The 16 rows of an item are the M side.  A warp takes 32 tokens at a time (they lie in one page and one group of keys) and
//     keeps its own maximum, denominator and sum; a CTA's warps are joined at the end.
//   - Scores: lane (g, q) holds token 8 n + g, channels 32 q .. 32 q + 31: a contiguous quarter of its codes.  Which of them
//     stand at which of the 16 steps of the contraction is free, as long as the queries agree: the two codes 16 bits apart in a
//     word become a pair of binary16 numbers by one logic instruction (their bits under the exponent of 2^(10 - s) make 2^(10 - s) + code),
//     one subtraction, and one multiply-add with the channel pair's scale and zero-point.
//   - Values: the same lane holds tokens 16 k + 2 q, + 1, + 8, + 9, channels 16 g .. 16 g + 15.  The halves of two tokens' words
//     are joined first, so a pair is one channel of two tokens, which is the order of this operand.
//   - A step's codes and metadata come through shared memory by cp.async, a few steps ahead.
// Binary16 keeps 11 significant bits, three more than bf16: the result's own rounding to bf16 is what is left.  Magnitudes
// beyond its range (or values that all lie below 2^-8, where it would lose them) are noticed on the way, and the
// segment is done again with bf16 operands.  Weights carry a factor of 2^8, so that those down to 2^-32 of the largest are not lost.
#include "chunk_attention.cuh"

namespace {

constexpr int D = SQUAT_D;
constexpr int THREADS = 128, WARPS = 4, STEP = 32;   // tokens per warp and step
constexpr int R = CHUNK_ROWS;
constexpr float P_SHIFT = 8.0f;

template <int BITS, int G, bool M16>
struct Stage {                                       // one step's part of the cache, in shared memory
    static constexpr int MS = M16 ? 2 : 4, ROW = D * BITS / 8, NG = D / G;
    static constexpr int QUARTER = 32 * MS + 16;     // key metadata: padded, so that the four quarters fall on distinct banks
    static constexpr int KC = 0, VC = STEP * ROW, KS = 2 * STEP * ROW, KZ = KS + 4 * QUARTER, VS = KZ + 4 * QUARTER, VZ = VS + STEP * NG * MS;
    static constexpr int BYTES = VZ + STEP * NG * MS;
    static constexpr int STAGES = 3;
};
constexpr int MERGE_ROW = D + 4;
constexpr int MERGE_BYTES = WARPS * R * (MERGE_ROW + 2) * 4;

__device__ __forceinline__ void cp16(unsigned dst, const void *src)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

template <bool BF>
__device__ __forceinline__ void mma16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    if (BF)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// what a warp has seen of the magnitudes
struct Range {
    __half2 ks, kz, vs, vz;                          // quantized scales and zero-points
    float k, v;                                      // rows in full precision
};

struct Acc {
    float m[2], l[2], o[16][4];
};

// One 32-token step's softmax: scores s[n][.] (columns 8 n + 2 q, + 1 of rows g and g + 8) become weights, packed as the A operand.
template <bool BF>
__device__ __forceinline__ void softmax_step(Acc &acc, float (&s)[4][4], float scale_log2, uint32_t (&pa)[2][4])
{
    float corr[2], base[2];
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        float mx = -INFINITY;
#pragma unroll
        for (int n = 0; n < 4; ++n) mx = max_nan(mx, max_nan(s[n][2 * r], s[n][2 * r + 1]));
        mx = max_nan(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
        mx = max_nan(mx, __shfl_xor_sync(0xffffffffu, mx, 2));
        const float m = max_nan(acc.m[r], mx * scale_log2), use = m == -INFINITY ? 0.0f : m;
        corr[r] = exp2_fast(acc.m[r] - use);
        acc.m[r] = m;
        base[r] = P_SHIFT - use;
        acc.l[r] *= corr[r];
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        acc.o[i][0] *= corr[0]; acc.o[i][1] *= corr[0];
        acc.o[i][2] *= corr[1]; acc.o[i][3] *= corr[1];
    }
#pragma unroll
    for (int n = 0; n < 4; ++n) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            s[n][e] = exp2_fast(fmaf(s[n][e], scale_log2, base[e >> 1]));
            acc.l[e >> 1] += s[n][e];
        }
        pa[n >> 1][(n & 1) * 2] = pack16<BF>(s[n][0], s[n][1]);
        pa[n >> 1][(n & 1) * 2 + 1] = pack16<BF>(s[n][2], s[n][3]);
    }
}

// A step of cached tokens, staged at `st`.
template <int BITS, int G, bool M16, bool BF>
__device__ __forceinline__ void cached_step(const unsigned char *st, const uint32_t (&qf)[8][4], float scale_log2, Acc &acc, Range &range)
{
    using S = Stage<BITS, G, M16>;
    const int lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3;
    constexpr int HALF = BITS == 2 ? 8 : 4;          // codes in half a word; a pair is (c, c + HALF) of a word
    float s[4][4];
#pragma unroll
    for (int n = 0; n < 4; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) s[n][e] = 0.0f;
    {
        const unsigned char *ks = st + S::KS + q * S::QUARTER, *kz = st + S::KZ + q * S::QUARTER;
        uint32_t s2[16], z2[16];
        if (!BF) {
            if (M16) {
                uint32_t a[16], b[16];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    *reinterpret_cast<uint4 *>(a + 4 * i) = reinterpret_cast<const uint4 *>(ks)[i];
                    *reinterpret_cast<uint4 *>(b + 4 * i) = reinterpret_cast<const uint4 *>(kz)[i];
                }
#pragma unroll
                for (int m = 0; m < 16; ++m) {
                    const int lo = m / HALF * 2 * HALF + m % HALF, hi = lo + HALF;
                    s2[m] = pair16(a[lo / 2], a[hi / 2], lo);
                    z2[m] = pair16(b[lo / 2], b[hi / 2], lo);
                }
            } else {
                float a[32], b[32];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    *reinterpret_cast<float4 *>(a + 4 * i) = reinterpret_cast<const float4 *>(ks)[i];
                    *reinterpret_cast<float4 *>(b + 4 * i) = reinterpret_cast<const float4 *>(kz)[i];
                }
#pragma unroll
                for (int m = 0; m < 16; ++m) {
                    const int lo = m / HALF * 2 * HALF + m % HALF, hi = lo + HALF;
                    s2[m] = pack16<false>(a[lo], a[hi]);
                    z2[m] = pack16<false>(b[lo], b[hi]);
                }
            }
#pragma unroll
            for (int m = 0; m < 16; ++m) {
                range.ks = __hmax2(range.ks, __habs2(as_half2(s2[m])));
                range.kz = __hmax2(range.kz, __habs2(as_half2(z2[m])));
            }
        }
#pragma unroll
        for (int n = 0; n < 4; ++n) {
            uint32_t w[BITS];
            const unsigned char *from = st + S::KC + (8 * n + g) * S::ROW + q * (S::ROW / 4);
            if (BITS == 2) {
                const uint2 v = *reinterpret_cast<const uint2 *>(from);
                w[0] = v.x; w[1] = v.y;
            } else {
                const uint4 v = *reinterpret_cast<const uint4 *>(from);
                w[0] = v.x; w[1] = v.y; w[BITS - 2] = v.z; w[BITS - 1] = v.w;
            }
            uint32_t b[16];
#pragma unroll
            for (int m = 0; m < 16; ++m) {
                if (!BF) {
                    b[m] = as_u32(__hfma2(code_pair<BITS>(w[m / HALF], m % HALF), as_half2(s2[m]), as_half2(z2[m])));
                } else {
                    const int lo = m / HALF * 2 * HALF + m % HALF, hi = lo + HALF;
                    float y[2];
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const int c = e ? hi : lo;
                        const float sc = M16 ? __half2float(reinterpret_cast<const __half *>(ks)[c]) : reinterpret_cast<const float *>(ks)[c];
                        const float zr = M16 ? __half2float(reinterpret_cast<const __half *>(kz)[c]) : reinterpret_cast<const float *>(kz)[c];
                        y[e] = fmaf(code_float<BITS>(w[m / HALF], m % HALF + e * HALF), sc, zr);
                    }
                    b[m] = pack16<true>(y[0], y[1]);
                }
            }
#pragma unroll
            for (int kk = 0; kk < 8; ++kk) mma16<BF>(s[n], qf[kk], b[2 * kk], b[2 * kk + 1]);
        }
    }
    uint32_t pa[2][4];
    softmax_step<BF>(acc, s, scale_log2, pa);
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) {
        uint32_t w[4][BITS / 2];                     // 16 channels of the lane's four tokens
        float sc[4], zr[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int t = 16 * kt + 2 * q + (j & 1) + 8 * (j >> 1);
            const unsigned char *from = st + S::VC + t * S::ROW + g * (S::ROW / 8);
            if (BITS == 2) w[j][0] = *reinterpret_cast<const uint32_t *>(from);
            else {
                const uint2 v = *reinterpret_cast<const uint2 *>(from);
                w[j][0] = v.x; w[j][BITS / 2 - 1] = v.y;
            }
            const int at = t * S::NG + g * 16 / G;
            sc[j] = M16 ? __half2float(reinterpret_cast<const __half *>(st + S::VS)[at]) : reinterpret_cast<const float *>(st + S::VS)[at];
            zr[j] = M16 ? __half2float(reinterpret_cast<const __half *>(st + S::VZ)[at]) : reinterpret_cast<const float *>(st + S::VZ)[at];
        }
        __half2 s2[2], z2[2];
        uint32_t both[2][BITS];                      // halves of the words of two tokens
        if (!BF) {
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                s2[e] = __floats2half2_rn(sc[2 * e], sc[2 * e + 1]);
                z2[e] = __floats2half2_rn(zr[2 * e], zr[2 * e + 1]);
                range.vs = __hmax2(range.vs, __habs2(s2[e]));
                range.vz = __hmax2(range.vz, __habs2(z2[e]));
#pragma unroll
                for (int i = 0; i < BITS; ++i) both[e][i] = pair16(w[2 * e][i / 2], w[2 * e + 1][i / 2], i);
            }
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            uint32_t b[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                if (!BF) b[e] = as_u32(__hfma2(code_pair<BITS>(both[e][i / HALF], i % HALF), s2[e], z2[e]));
                else {
                    constexpr int PER = 2 * HALF;
                    b[e] = pack16<true>(fmaf(code_float<BITS>(w[2 * e][i / PER], i % PER), sc[2 * e], zr[2 * e]),
                                        fmaf(code_float<BITS>(w[2 * e + 1][i / PER], i % PER), sc[2 * e + 1], zr[2 * e + 1]));
                }
            }
            mma16<BF>(acc.o[i], pa[kt], b[0], b[1]);
        }
    }
}

// A step of rows in full precision: rows u0 .. u0 + 31 of the sequence, of which row g of the item sees the first sees[0], row
// g + 8 the first sees[1], and none more than `most`.
template <int BITS, bool BF>
__device__ __forceinline__ void full_step(const ChunkParams &p, const ChunkSeq &sq, int h, int u0, int most, const int (&sees)[2],
                                          const uint32_t (&qf)[8][4], Acc &acc, Range &range)
{
    constexpr int HALF = BITS == 2 ? 8 : 4;
    const int lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3;
    float s[4][4];
#pragma unroll
    for (int n = 0; n < 4; ++n) {
        const int u = u0 + 8 * n + g;
        uint32_t x[16];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            uint4 v = make_uint4(0, 0, 0, 0);
            if (u < most) v = ldg128(p.k_new + (long long)(sq.k0 + u) * p.knt + (long long)h * p.knh + 32 * q + 8 * i);
            x[4 * i] = v.x; x[4 * i + 1] = v.y; x[4 * i + 2] = v.z; x[4 * i + 3] = v.w;
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) s[n][e] = 0.0f;
        if (!BF)
#pragma unroll
            for (int i = 0; i < 16; ++i) {            // infinities and NaN are the same in either type
                const float lo = fabsf(bf16lo_to_f32(x[i])), hi = fabsf(bf16hi_to_f32(x[i]));
                range.k = fmaxf(range.k, fmaxf(lo < INFINITY ? lo : 0.0f, hi < INFINITY ? hi : 0.0f));
            }
        uint32_t b[16];
#pragma unroll
        for (int m = 0; m < 16; ++m) {
            const int lo = m / HALF * 2 * HALF + m % HALF;
            b[m] = pair16(x[lo / 2], x[(lo + HALF) / 2], lo);
            if (!BF) b[m] = bf16_pair_to_f16(b[m]);
        }
#pragma unroll
        for (int kk = 0; kk < 8; ++kk) mma16<BF>(s[n], qf[kk], b[2 * kk], b[2 * kk + 1]);
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (u0 + 8 * n + 2 * q + (e & 1) >= sees[e >> 1]) s[n][e] = -INFINITY;
    }
    uint32_t pa[2][4];
    softmax_step<BF>(acc, s, p.scale_log2, pa);
    bool odd = false;                                // an infinity or NaN among the lane's values
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) {
        uint32_t w[4][8];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int u = u0 + 16 * kt + 2 * q + (j & 1) + 8 * (j >> 1);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                uint4 v = make_uint4(0, 0, 0, 0);
                if (u < most) v = ldg128(p.v_new + (long long)(sq.k0 + u) * p.vnt + (long long)h * p.vnh + 16 * g + 8 * i);
                w[j][4 * i] = v.x; w[j][4 * i + 1] = v.y; w[j][4 * i + 2] = v.z; w[j][4 * i + 3] = v.w;
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if (bf16_pair_not_finite(w[j][i])) {  // a row that does not see it must not meet it: its weight of zero would not do
                    odd = true;
                    if ((w[j][i] & 0x7f80u) == 0x7f80u) w[j][i] &= 0xffff0000u;
                    if ((w[j][i] & 0x7f800000u) == 0x7f800000u) w[j][i] &= 0x0000ffffu;
                }
                if (!BF) range.v = fmaxf(range.v, fmaxf(fabsf(bf16lo_to_f32(w[j][i])), fabsf(bf16hi_to_f32(w[j][i]))));
            }
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            uint32_t b0 = pair16(w[0][i / 2], w[1][i / 2], i), b1 = pair16(w[2][i / 2], w[3][i / 2], i);
            if (!BF) { b0 = bf16_pair_to_f16(b0); b1 = bf16_pair_to_f16(b1); }
            mma16<BF>(acc.o[i], pa[kt], b0, b1);
        }
    }
    if (__any_sync(0xffffffffu, odd)) {              // rare: the rows that see such a value get it
#pragma unroll 1
        for (int u = u0; u < min(u0 + STEP, most); ++u) {
            const __nv_bfloat16 *v = p.v_new + (long long)(sq.k0 + u) * p.vnt + (long long)h * p.vnh + 32 * q;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const float x = __bfloat162float(v[16 * e + i]);
                    if (fabsf(x) < INFINITY) continue;
                    if (u < sees[0]) acc.o[i][e] += x;
                    if (u < sees[1]) acc.o[i][2 + e] += x;
                }
            }
        }
    }
}

// Tiles [ta, tb) of an item by one warp: 32 tokens of every tile.  Returns whether binary16 was too narrow.
template <int BITS, int G, bool M16, bool BF>
__device__ __forceinline__ bool run_segment(const ChunkParams &p, const ChunkPlace &pl, const ChunkSeq &sq, int ta, int tb, unsigned char *stages, Acc &acc)
{
    using S = Stage<BITS, G, M16>;
    constexpr int HALF = BITS == 2 ? 8 : 4;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, q = lane & 3;
    const int rows = sq.nq * p.qpk, row0 = pl.qt * R;
    const int ct = (sq.cached + CHUNK_TILE - 1) / CHUNK_TILE;
    Range range = {};
    acc.m[0] = acc.m[1] = -INFINITY;
    acc.l[0] = acc.l[1] = 0.0f;
#pragma unroll
    for (int i = 0; i < 16; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc.o[i][e] = 0.0f;

    // ---- the cached steps of this warp: tile ta + i, tokens 32 warp .. of it
    const int c_end = min(tb, ct);
    int steps = max(c_end - ta, 0);
    if (steps > 0 && (c_end - 1) * CHUNK_TILE + STEP * warp >= sq.cached) --steps;           // the last tile may end before this warp's tokens
    int page_off = 0;                                // lane i: where step (32 b + i)'s tokens are
    long long page_tok = 0;
    auto look_up = [&](int first) {
        const int i = first + lane;
        if (i < steps) {
            const int t = (ta + i) * CHUNK_TILE + STEP * warp, at = t / p.pool.page_tokens;
            int page = __ldg(p.page_table + (long long)pl.seq * p.table_stride + at);
            if ((unsigned)page >= (unsigned)p.pool.n_pages) {
                atomicOr(p.status, SQUAT_FLAG_PAGES);
                page = 0;
            }
            page_off = t - at * p.pool.page_tokens;
            page_tok = (long long)page * p.pool.page_stride + (long long)pl.h * p.pool.head_stride + page_off;
        }
    };
    const unsigned stage0 = smem_u32(stages);
    auto load = [&](int i) {                         // step i into its stage
        if (i < steps) {
            const long long tok = __shfl_sync(0xffffffffu, page_tok, i & 31);
            const unsigned dst = stage0 + i % S::STAGES * S::BYTES;
            const unsigned char *kc = p.pool.kc + tok * S::ROW, *vc = p.pool.vc + tok * S::ROW;
#pragma unroll
            for (int j = 0; j < BITS; ++j) {
                cp16(dst + S::KC + (32 * j + lane) * 16, kc + (32 * j + lane) * 16);
                cp16(dst + S::VC + (32 * j + lane) * 16, vc + (32 * j + lane) * 16);
            }
            constexpr int KP = D * S::MS / 16, PER_Q = KP / 4;        // pieces of a row of key metadata, and of a quarter
            const unsigned char *ks = static_cast<const unsigned char *>(p.pool.ks) + tok / G * (D * S::MS), *kz = static_cast<const unsigned char *>(p.pool.kz) + tok / G * (D * S::MS);
            if (M16) {
                const int j = lane % KP;
                cp16(dst + (lane < KP ? S::KS : S::KZ) + j / PER_Q * S::QUARTER + j % PER_Q * 16, (lane < KP ? ks : kz) + j * 16);
            } else {
                cp16(dst + S::KS + lane / PER_Q * S::QUARTER + lane % PER_Q * 16, ks + lane * 16);
                cp16(dst + S::KZ + lane / PER_Q * S::QUARTER + lane % PER_Q * 16, kz + lane * 16);
            }
            constexpr int VP = STEP * S::NG * S::MS / 16;             // pieces of the value scales: 4 .. 32
            const unsigned char *vs = static_cast<const unsigned char *>(p.pool.vs) + tok * (S::NG * S::MS), *vz = static_cast<const unsigned char *>(p.pool.vz) + tok * (S::NG * S::MS);
            if (VP == 32) {
                cp16(dst + S::VS + lane * 16, vs + lane * 16);
                cp16(dst + S::VZ + lane * 16, vz + lane * 16);
            } else if (lane < 2 * VP) {
                const int j = lane % VP;
                cp16(dst + (lane < VP ? S::VS : S::VZ) + j * 16, (lane < VP ? vs : vz) + j * 16);
            }
        }
        cp_commit();
    };
    if (steps > 0) {
        look_up(0);
#pragma unroll
        for (int i = 0; i < S::STAGES - 1; ++i) load(i);
    }

    // ---- queries: rows g and g + 8, channels 32 q .. + 31, in the order of the key operand
    uint32_t qf[8][4];
    float q_max = 0.0f;
#pragma unroll
    for (int e = 0; e < 2; ++e) {
        const int r = row0 + g + 8 * e;
        uint32_t x[16];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            uint4 v = make_uint4(0, 0, 0, 0);
            if (r < rows) v = ldg128(p.q + (long long)(sq.q0 + r / p.qpk) * p.qt + (long long)(pl.h * p.qpk + r % p.qpk) * p.qh + 32 * q + 8 * i);
            x[4 * i] = v.x; x[4 * i + 1] = v.y; x[4 * i + 2] = v.z; x[4 * i + 3] = v.w;
        }
#pragma unroll
        for (int m = 0; m < 16; ++m) {
            const int lo = m / HALF * 2 * HALF + m % HALF;
            uint32_t v = pair16(x[lo / 2], x[(lo + HALF) / 2], lo);
            if (!BF) {
                q_max = fmaxf(q_max, fmaxf(fabsf(bf16lo_to_f32(v)), fabsf(bf16hi_to_f32(v))));
                v = bf16_pair_to_f16(v);
            }
            qf[m / 2][(m & 1) * 2 + e] = v;
        }
    }

#pragma unroll 1
    for (int i = 0; i < steps; ++i) {
        cp_wait<S::STAGES - 2>();
        __syncwarp();
        cached_step<BITS, G, M16, BF>(stages + i % S::STAGES * S::BYTES, qf, p.scale_log2, acc, range);
        __syncwarp();
        if ((i + S::STAGES - 1) % 32 == 0) look_up(i + S::STAGES - 1);
        load(i + S::STAGES - 1);
    }
    cp_wait<0>();
    __syncwarp();

    // ---- rows in full precision
    const int last = min(rows, row0 + R) - 1, most = chunk_sees(p, sq, last / p.qpk);
    const int sees[2] = {chunk_sees(p, sq, min(row0 + g, last) / p.qpk), chunk_sees(p, sq, min(row0 + g + 8, last) / p.qpk)};
#pragma unroll 1
    for (int t = max(ta, ct); t < tb; ++t) {
        const int u0 = (t - ct) * CHUNK_TILE + STEP * warp;
        if (u0 < most) full_step<BITS, BF>(p, sq, pl.h, u0, most, sees, qf, acc, range);
    }
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        acc.l[r] += __shfl_xor_sync(0xffffffffu, acc.l[r], 1);
        acc.l[r] += __shfl_xor_sync(0xffffffffu, acc.l[r], 2);
    }
    if (BF) return false;
    constexpr float L = float((1 << BITS) - 1);
    auto top = [](__half2 x) { const float2 f = __half22float2(x); return fmaxf(f.x, f.y); };
    // 2^12 for queries and keys: what falls below 2^-25 of binary16 is then less than 2^-13 of a score's unit even in 128 products
    const float k_top = fmaxf(fmaf(L, top(range.ks), top(range.kz)), range.k), v_top = fmaxf(fmaf(L, top(range.vs), top(range.vz)), range.v);
    const bool wide = !(q_max < 4096.0f) || !(k_top < 4096.0f) || !(v_top < 65000.0f);
    const float v_low = fmaxf(fmaxf(top(range.vs), top(range.vz)), range.v);
    return __any_sync(0xffffffffu, wide) || (!__any_sync(0xffffffffu, v_low >= 0x1p-8f) && __any_sync(0xffffffffu, v_low > 0.0f));
}

template <int BITS, int G, bool M16>
__global__ void __launch_bounds__(THREADS, 2) chunk_rows_kernel(const __grid_constant__ ChunkParams params)
{
    using S = Stage<BITS, G, M16>;
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ ChunkShared sh;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, q = lane & 3;
    ChunkParams p = params;
    grid_wait(p.q, p.q_start, p.cached_len, p.page_table, p.new_start, p.new_len, p.k_new, p.v_new);
    long long per, total;
    chunk_share<R>(p, sh, per, total);
    long long at = per * blockIdx.x;
    if (at >= total) return;
    const long long end = min(at + per, total);
    ChunkPlace pl = chunk_locate<R>(p, sh, at);
    ChunkSeq sq = chunk_seq(p, pl.seq);
    float *o_sm = reinterpret_cast<float *>(smem), *ml_sm = o_sm + WARPS * R * MERGE_ROW;
    while (at < end) {
        const int tiles = chunk_tiles<R>(p, sq, pl.qt), ta = pl.tile, tb = (int)min((long long)tiles, ta + (end - at));
        Acc acc;
        const bool narrow = run_segment<BITS, G, M16, false>(p, pl, sq, ta, tb, smem + warp * S::STAGES * S::BYTES, acc);
        if (__syncthreads_or(narrow)) run_segment<BITS, G, M16, true>(p, pl, sq, ta, tb, smem + warp * S::STAGES * S::BYTES, acc);
        __syncthreads();                             // the stages become the place where the warps meet
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            float *row = o_sm + (warp * R + g + 8 * e) * MERGE_ROW + 32 * q;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                *reinterpret_cast<float4 *>(row + 4 * j) = make_float4(acc.o[4 * j][2 * e], acc.o[4 * j + 1][2 * e], acc.o[4 * j + 2][2 * e], acc.o[4 * j + 3][2 * e]);
                *reinterpret_cast<float4 *>(row + 16 + 4 * j) = make_float4(acc.o[4 * j][2 * e + 1], acc.o[4 * j + 1][2 * e + 1], acc.o[4 * j + 2][2 * e + 1], acc.o[4 * j + 3][2 * e + 1]);
            }
            if (q == 0) {
                ml_sm[(warp * R + g + 8 * e) * 2] = acc.m[e];
                ml_sm[(warp * R + g + 8 * e) * 2 + 1] = acc.l[e];
            }
        }
        __syncthreads();
        const bool whole = ta == 0 && tb == tiles;
        const int row0 = pl.qt * R, n_rows = min(R, sq.nq * p.qpk - row0);
        const long long slot = 2LL * blockIdx.x + (ta == 0 ? 1 : 0);
#pragma unroll 1
        for (int r = 0; r < n_rows; ++r) {
            float m = -INFINITY, l = 0.0f, o = 0.0f;
#pragma unroll
            for (int w = 0; w < WARPS; ++w) m = max_nan(m, ml_sm[(w * R + r) * 2]);
            const float use = m == -INFINITY ? 0.0f : m;
#pragma unroll
            for (int w = 0; w < WARPS; ++w) {
                const float f = exp2_fast(ml_sm[(w * R + r) * 2] - use);
                l = fmaf(f, ml_sm[(w * R + r) * 2 + 1], l);
                o = fmaf(f, o_sm[(w * R + r) * MERGE_ROW + tid], o);
            }
            if (whole) {
                const int row = row0 + r, j = sq.q0 + row / p.qpk, hq = pl.h * p.qpk + row % p.qpk;
                p.out[(long long)j * p.ot + (long long)hq * p.oh + tid] = __float2bfloat16_rn(l == 0.0f ? 0.0f : o / l);
                if (p.lse && tid == 0) p.lse[(long long)j * p.Hq + hq] = l == 0.0f ? -INFINITY : (m - P_SHIFT + log2f(l)) * 0.6931471805599453f;
            } else {
                p.part[(slot * R + r) * D + tid] = o;
                if (tid == 0) *reinterpret_cast<float2 *>(p.ml + (slot * R + r) * 2) = make_float2(m, l);
            }
        }
        __syncthreads();
        at += tb - ta;
        if (at < end) chunk_next<R>(p, pl, sq);
    }
}

// CTA c: the item that CTA c of the main kernel began and did not finish, if there is one.  A warp takes a row, four channels a lane.
template <int ROWS>
__global__ void __launch_bounds__(D) chunk_combine_kernel(const __grid_constant__ ChunkParams params)
{
    __shared__ ChunkShared sh;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    ChunkParams p = params;
    grid_wait(p.q, p.q_start, p.cached_len, p.page_table, p.new_start, p.new_len, p.k_new, p.v_new);
    long long per, total;
    chunk_share<ROWS>(p, sh, per, total);
    const long long c = blockIdx.x, border = (c + 1) * per;
    if (border >= total) return;
    const ChunkPlace pl = chunk_locate<ROWS>(p, sh, border);
    const long long first = border - pl.tile;        // the item's first tile
    if (pl.tile == 0 || first < c * per) return;
    const ChunkSeq sq = chunk_seq(p, pl.seq);
    const long long parts = (first + chunk_tiles<ROWS>(p, sq, pl.qt) - 1) / per - c + 1;
    const int row0 = pl.qt * ROWS, n_rows = min(ROWS, sq.nq * p.qpk - row0);
#pragma unroll 1
    for (int r = blockIdx.y * 4 + warp; r < n_rows; r += gridDim.y * 4) {
        float m = -INFINITY, l = 0.0f;
        float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        constexpr int AT_ONCE = 8;                   // parts whose loads are in flight together
#pragma unroll 1
        for (long long i0 = 0; i0 < parts; i0 += AT_ONCE) {
            float2 v[AT_ONCE];
            float4 x[AT_ONCE];
#pragma unroll
            for (int i = 0; i < AT_ONCE; ++i) {
                const bool in = i0 + i < parts;
                const long long at = ((i0 + i == 0 ? 2 * c + 1 : 2 * (c + i0 + i)) * ROWS + r);
                v[i] = in ? *reinterpret_cast<const float2 *>(p.ml + at * 2) : make_float2(-INFINITY, 0.0f);
                x[i] = in ? *reinterpret_cast<const float4 *>(p.part + at * D + 4 * lane) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            }
            float mn = m;
#pragma unroll
            for (int i = 0; i < AT_ONCE; ++i) mn = max_nan(mn, v[i].x);
            const float use = mn == -INFINITY ? 0.0f : mn, f0 = exp2_fast(m - use);
            l *= f0;
            o.x *= f0; o.y *= f0; o.z *= f0; o.w *= f0;
#pragma unroll
            for (int i = 0; i < AT_ONCE; ++i) {
                const float f = exp2_fast(v[i].x - use);
                l = fmaf(f, v[i].y, l);
                o.x = fmaf(f, x[i].x, o.x); o.y = fmaf(f, x[i].y, o.y); o.z = fmaf(f, x[i].z, o.z); o.w = fmaf(f, x[i].w, o.w);
            }
            m = mn;
        }
        const int row = row0 + r, j = sq.q0 + row / p.qpk, hq = pl.h * p.qpk + row % p.qpk;
        const float inv = l == 0.0f ? 0.0f : 1.0f / l;
        *reinterpret_cast<uint2 *>(p.out + (long long)j * p.ot + (long long)hq * p.oh + 4 * lane) = make_uint2(pack16<true>(o.x * inv, o.y * inv), pack16<true>(o.z * inv, o.w * inv));
        if (p.lse && lane == 0) p.lse[(long long)j * p.Hq + hq] = l == 0.0f ? -INFINITY : (m - P_SHIFT + log2f(l)) * 0.6931471805599453f;
    }
}

template <int BITS, int G, bool M16>
int launch_rows(const ChunkParams &p, cudaStream_t st)
{
    using S = Stage<BITS, G, M16>;
    constexpr size_t smem = WARPS * S::STAGES * S::BYTES > MERGE_BYTES ? WARPS * S::STAGES * S::BYTES : MERGE_BYTES;
    static std::atomic<unsigned long long> allowed{0};
    const int rc = squat_allow_smem(reinterpret_cast<const void *>(chunk_rows_kernel<BITS, G, M16>), smem, allowed);
    if (rc != SQUAT_OK) return rc;
    return squat_launch(chunk_rows_kernel<BITS, G, M16>, p.n_cta, THREADS, smem, st, p);
}

}  // namespace

int squat_launch_chunk_rows(const ChunkParams &p, int bits, int meta16, cudaStream_t st)
{
#define SQ_C(BB, GG) return meta16 ? launch_rows<BB, GG, true>(p, st) : launch_rows<BB, GG, false>(p, st)
    if (bits == 2) { if (p.G == 32) SQ_C(2, 32); if (p.G == 64) SQ_C(2, 64); SQ_C(2, 128); }
    if (p.G == 32) SQ_C(4, 32);
    if (p.G == 64) SQ_C(4, 64);
    SQ_C(4, 128);
#undef SQ_C
}

namespace {

// The kernels of a call: rows of the sequences with at most few_rows rows per KV head go to the kernel for few rows, those of the
// others to the kernel for many, in tiles of 128 or 256.
struct ChunkKernels {
    bool rows;
    int tiles;                                       // 0: no kernel for many rows
};
constexpr int FEW_ROWS = 16;

ChunkKernels kernels_for(long long n_q, long long n_seqs, long long max_q, int qpk)
{
    ChunkKernels k;
    const long long most = max_q * qpk;
    k.tiles = most <= FEW_ROWS ? 0 : most <= 128 ? 1 : 2;
    k.rows = k.tiles == 0 || n_q != n_seqs * max_q;  // sequences of one length, all of them in the other kernel
    return k;
}
int matrix_ctas(int tiles) { return squat_sm_count() * (tiles == 2 ? 1 : 2); }
size_t part_floats(int n_cta, int rows) { return 2 * (size_t)n_cta * rows * (D + 2); }
void use_part(ChunkParams &p, float *at, int n_cta, int rows)
{
    p.n_cta = n_cta;
    p.part = at;
    p.ml = at + 2 * (size_t)n_cta * rows * D;
}

}  // namespace

size_t squat_chunk_workspace_floats(int n_q, int n_q_heads, int n_kv_heads, int max_q)
{
    (void)n_q;
    size_t n = part_floats(2 * squat_sm_count(), CHUNK_ROWS);
    const int tiles = kernels_for(0, 0, max_q, n_q_heads / n_kv_heads).tiles;
    if (tiles) n += part_floats(matrix_ctas(tiles), 128 * tiles);
    return n;
}

int squat_launch_chunk_attention(ChunkParams p, const squat_page_pool *pool, float *workspace, int max_q, cudaStream_t st)
{
    p.pool = page_pool_of(pool);
    p.G = pool->group_size;
    p.H = pool->n_kv_heads;
    p.qpk = p.Hq / p.H;
    p.status = squat_status_word();
    if (!p.status) return SQUAT_ERR_CUDA;
    const ChunkKernels k = kernels_for(p.n_q, p.n_seqs, max_q, p.qpk);
    ChunkParams few = p, many = p;
    few.min_rows = 1;
    few.max_rows = k.tiles ? FEW_ROWS : 0x7fffffff;
    few.min_tiles = 2;
    use_part(few, workspace, 2 * squat_sm_count(), CHUNK_ROWS);
    many.min_rows = k.rows ? FEW_ROWS + 1 : 1;
    many.max_rows = 0x7fffffff;
    many.min_tiles = 4;
    int rc = SQUAT_OK;
    if (k.tiles) {
        use_part(many, workspace + part_floats(few.n_cta, CHUNK_ROWS), matrix_ctas(k.tiles), 128 * k.tiles);
        rc = squat_launch_chunk_matrix(many, k.tiles, pool->bits, pool->meta16, st);
    }
    if (rc == SQUAT_OK && k.rows) rc = squat_launch_chunk_rows(few, pool->bits, pool->meta16, st);
    if (rc == SQUAT_OK && k.tiles == 1) rc = squat_launch(chunk_combine_kernel<128>, dim3((unsigned)many.n_cta, 8), D, 0, st, many);
    if (rc == SQUAT_OK && k.tiles == 2) rc = squat_launch(chunk_combine_kernel<256>, dim3((unsigned)many.n_cta, 16), D, 0, st, many);
    if (rc == SQUAT_OK && k.rows) rc = squat_launch(chunk_combine_kernel<CHUNK_ROWS>, dim3((unsigned)few.n_cta, 1), D, 0, st, few);
    return rc;
}
