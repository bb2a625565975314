// Attention of new tokens over a paged, quantized cache (squat_chunk_attention): the kernel for few rows per KV head (decode
// steps, drafted tokens), and the sum of an item's parts.
//
//   out_r = sum_t p_rt v_t / sum_t p_rt,   p_rt = 2^(c <q_r, k_t> - m_r),   c = softmax scale / ln 2,   m_r the running maximum
//
// The cache's bytes bound it, if the two instructions that a code costs can be issued meanwhile.  So nothing is staged for
// the tensor core: the operands of mma.sync m16n8k16 are made in the registers where it wants them, the dequantized ones once for
// up to 24 rows, 8 rows a product (the tcgen05 form wants them in shared or tensor memory, and 128 rows to fill it).
//   - A warp works by itself: it takes 32 tokens at a time (they lie in one page and one group of keys) of its own share of the work.
//     (Warps that shared an item waited for one another at its end: a quarter of all stalls.)
//   - Scores, transposed: tokens are the 16 side.  Lane (g, q) holds tokens g and g + 8, channels 32 q .. 32 q + 31: a contiguous
//     quarter of their codes.  Which of them stand at which of the steps of the contraction is free, as long as the queries agree: the two
//     codes 16 bits apart in a word become a pair of binary16 numbers by one logic instruction (their bits under the exponent of 2^(10 - s)
//     make 2^(10 - s) + code), one subtraction, and one multiply-add with the channel pair's scale and zero-point.
//   - The weights' 8 x 8 blocks are transposed by movmatrix into the other operand of the second product.
//   - Values, transposed: channels are the 16 side.  Lane (g, q) holds tokens 16 k + 2 q, + 1, + 8, + 9, channels 16 g .. 16 g + 15.
//     The halves of two tokens' words are joined first, so a pair is one channel of two tokens, which is the order of this operand.
//     Its sums stand at the lane that holds the rows' maxima.
//   - A step's codes and metadata come through shared memory by cp.async, a step ahead.
// The loops are rolled where the registers allow it: straight-line code of a step, met once by a short sequence, takes longer to be
// fetched than to be executed.
// 64 sequences of up to 4096 tokens, one new token each, 32 heads with keys of their own, 2 bits: 235 us, 2.6 TB/s of codes and metadata: 870
// instructions for 32 tokens of a head, issued at 60 % of the slots by 14 warps an SM.  16 sequences of up to 8160 tokens, 24 rows for each
// of 8 heads: 81 us, 1310 instructions, at 45 % of the slots: 255 registers leave 8 warps an SM, which wait for one another's latencies.
// Binary16 keeps 11 significant bits, three more than bf16: the result's own rounding to bf16 is what is left.  Magnitudes
// beyond its range (or values that all lie below 2^-8, where it would lose them, or keys and queries of which it would lose what
// matters: chunk_too_low) are noticed on the way, and the segment is done again with bf16 operands.  Weights carry a factor of 2^8, so that those down to 2^-32 of the largest are not lost.
#include "chunk_attention.cuh"

namespace {

constexpr int D = SQUAT_D;
constexpr int THREADS = 128, WARPS = 4, STEP = 32, STAGES = 2;     // tokens per warp and step, steps in shared memory
constexpr float P_SHIFT = 8.0f;

template <int BITS, bool M16>
struct Stage {                                       // one step's part of the cache, in shared memory
    static constexpr int MS = M16 ? 2 : 4, ROW = D * BITS / 8;
    static constexpr int QUARTER = 32 * MS + 16;     // key metadata: padded, so that the four quarters fall on distinct banks
    static constexpr int KC = 0, VC = STEP * ROW, KS = 2 * STEP * ROW, KZ = KS + 4 * QUARTER, VS = KZ + 4 * QUARTER, VZ = VS + STEP * 4 * MS;
    static constexpr int BYTES = VZ + STEP * 4 * MS;
};
// CTAs to an SM, by registers.  Four of 8 rows: 64 ragged sequences, 32 heads with keys of their own, 235 us (three 247); on 8 KV heads 89
// (three 87).  Three of 16 rows: 16 sequences of up to 8160 tokens 87 us, with 400 to 500 bytes of spills a thread (two, without: 79).
template <int NT>
constexpr int CTAS = NT == 1 ? 4 : NT == 2 ? 3 : 2;

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
// 8 x 8 block of 16-bit numbers, lane (g, q) holding columns 2 q, 2 q + 1 of row g: transposed
__device__ __forceinline__ uint32_t transposed(uint32_t x)
{
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}

// What a lane has seen of the magnitudes.
struct Range {
    __half2 ks, kz;                                  // largest of the keys' scales and of their zero-points
    float k;                                         // largest finite one among keys in full precision
    float v;                                         // largest of the values' scales and zero-points, and of the finite ones in full precision
    float score;                                     // largest score of cached tokens
    int odd_first, odd_last;                         // range of rows in full precision with infinities or NaN among their values
};

// The other operand of the scores: rows 8 t + g, the lane's 16 pairs of channels, in the warp's own shared memory.
template <int NT>
struct Queries {
    static constexpr int BYTES = NT * 16 * 32 * 4;
    uint32_t *smem;                                  // the lane's place: [t][pair / 4][lane][4]
    __device__ __forceinline__ void put(int t, const uint32_t (&x)[16]) const
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) *reinterpret_cast<uint4 *>(smem + (t * 4 + i) * 128) = make_uint4(x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]);
    }
    __device__ __forceinline__ void get(int t, int four, uint32_t (&b)[4]) const       // pairs 4 four .. + 3
    {
        const uint4 v = *reinterpret_cast<const uint4 *>(smem + (t * 4 + four) * 128);
        b[0] = v.x; b[1] = v.y; b[2] = v.z; b[3] = v.w;
    }
};

// Rows 8 t + 2 q and 8 t + 2 q + 1: maximum, denominator, and sums of channels 16 g + i and 16 g + i + 8 (o[t][i]: row, row + 1, each)
template <int NT>
struct Acc {
    float m[NT][2], l[NT][2], o[NT][8][4];
};

// One 32-token step's softmax: scores s[t][k] (tokens 16 k + g, + 8 of the lane's two rows) become weights, packed as the operand of the
// second product.
template <int NT, bool BF>
__device__ __forceinline__ void softmax_step(Acc<NT> &acc, float (&s)[NT][2][4], float scale_log2, uint32_t (&pb)[NT][2][2])
{
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        float base[2], corr[2];
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            float mx = max_nan(max_nan(s[t][0][r], s[t][0][2 + r]), max_nan(s[t][1][r], s[t][1][2 + r]));
#pragma unroll
            for (int o = 4; o < 32; o <<= 1) mx = max_nan(mx, __shfl_xor_sync(0xffffffffu, mx, o));
            const float m = max_nan(acc.m[t][r], mx * scale_log2), use = m == -INFINITY ? 0.0f : m;
            corr[r] = exp2_fast(acc.m[t][r] - use);
            acc.m[t][r] = m;
            base[r] = P_SHIFT - use;
            acc.l[t][r] *= corr[r];
        }
        if (__any_sync(0xffffffffu, corr[0] != 1.0f || corr[1] != 1.0f)) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                acc.o[t][i][0] *= corr[0]; acc.o[t][i][2] *= corr[0];
                acc.o[t][i][1] *= corr[1]; acc.o[t][i][3] *= corr[1];
            }
        }
#pragma unroll
        for (int k = 0; k < 2; ++k) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                s[t][k][e] = exp2_fast(fmaf(s[t][k][e], scale_log2, base[e & 1]));
                acc.l[t][e & 1] += s[t][k][e];
            }
            pb[t][k][0] = transposed(pack16<BF>(s[t][k][0], s[t][k][1]));
            pb[t][k][1] = transposed(pack16<BF>(s[t][k][2], s[t][k][3]));
        }
    }
}

// The key metadata of a step in the operand's order, binary16, in the place of the first half of what was loaded: for a quarter of the channels
// eight 16-byte pieces, scales of two neighbouring pairs (channels lo, lo + HALF and lo + 1, lo + 1 + HALF) and their zero-points.  A
// lane makes one of them for the eight lanes that use it.
constexpr int PAIRS_QUARTER = 8 * 16 + 16;           // padded: the four quarters fall on distinct banks
template <int BITS, bool M16>
__device__ __forceinline__ void order_key_meta(unsigned char *st, Range &range)
{
    using S = Stage<BITS, M16>;
    constexpr int HALF = BITS == 2 ? 8 : 4;          // codes in half a word; a pair is (c, c + HALF) of a word
    const int lane = threadIdx.x & 31, quarter = lane >> 3, m = 2 * (lane & 7), lo = m / HALF * 2 * HALF + m % HALF;
    uint32_t y[4];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
        const unsigned char *from = st + (e ? S::KZ : S::KS) + quarter * S::QUARTER;
        if (M16) {
            const uint32_t a = reinterpret_cast<const uint32_t *>(from)[lo / 2], b = reinterpret_cast<const uint32_t *>(from)[(lo + HALF) / 2];
            y[2 * e] = pair16(a, b, 0);
            y[2 * e + 1] = pair16(a, b, 1);
        } else {
            const float2 a = reinterpret_cast<const float2 *>(from)[lo / 2], b = reinterpret_cast<const float2 *>(from)[(lo + HALF) / 2];
            y[2 * e] = pack16<false>(a.x, b.x);
            y[2 * e + 1] = pack16<false>(a.y, b.y);
        }
    }
    range.ks = __hmax2(range.ks, __hmax2(__habs2(as_half2(y[0])), __habs2(as_half2(y[1]))));
    range.kz = __hmax2(range.kz, __hmax2(__habs2(as_half2(y[2])), __habs2(as_half2(y[3]))));
    __syncwarp();
    *reinterpret_cast<uint4 *>(st + S::KS + quarter * PAIRS_QUARTER + (lane & 7) * 16) = make_uint4(y[0], y[1], y[2], y[3]);
    __syncwarp();
}
template <bool M16>
__device__ __forceinline__ float meta_at(const unsigned char *from, int i)
{
    return M16 ? __half2float(reinterpret_cast<const __half *>(from)[i]) : reinterpret_cast<const float *>(from)[i];
}

// For few rows it is less to scale the queries than the codes (16 products a row of eight rather than 128 differences and multiply-adds).
template <int NT>
constexpr bool folds = NT <= 2;

// A step of cached tokens, staged at `st`.
template <int BITS, bool M16, int NT, bool BF>
__device__ __forceinline__ void cached_step(unsigned char *st, const CodeBias<BITS> &bias, int g_shift, const Queries<NT> &queries, float scale_log2, Acc<NT> &acc, Range &range)
{
    using S = Stage<BITS, M16>;
    const int lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3;
    constexpr int HALF = BITS == 2 ? 8 : 4;
    float s[NT][2][4];
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int e = 0; e < 4; ++e) s[t][k][e] = 0.0f;
    if (!BF) order_key_meta<BITS, M16>(st, range);
    constexpr bool FOLD = !BF && folds<NT>;
    {
        float alike[NT][4];
        if (FOLD)
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e) alike[t][e] = 0.0f;
        const unsigned char *ks = st + S::KS + q * S::QUARTER, *kz = st + S::KZ + q * S::QUARTER, *kc = st + S::KC + g * S::ROW + q * (S::ROW / 4);
#pragma unroll 1
        for (int wd = 0; wd < BITS; ++wd) {          // a word of codes: HALF pairs
            uint32_t w[4];                           // of tokens g, g + 8, g + 16, g + 24
#pragma unroll
            for (int e = 0; e < 4; ++e) w[e] = *reinterpret_cast<const uint32_t *>(kc + 8 * e * S::ROW + 4 * wd);
#pragma unroll
            for (int four = 0; four < HALF / 4; ++four) {
                uint32_t b4[NT][4];
#pragma unroll
                for (int t = 0; t < NT; ++t) queries.get(t, wd * (HALF / 4) + four, b4[t]);
#pragma unroll
                for (int two = 0; two < 2; ++two) {  // a product contracts two pairs of every lane of a quad
                    const int c = 4 * four + 2 * two, lo = wd * 2 * HALF + c;
                    __half2 s2[2], z2[2];
                    if (!BF) {
                        const uint4 v = *reinterpret_cast<const uint4 *>(st + S::KS + q * PAIRS_QUARTER + (wd * (HALF / 2) + 2 * four + two) * 16);
                        s2[0] = as_half2(v.x); s2[1] = as_half2(v.y);
                        z2[0] = as_half2(v.z); z2[1] = as_half2(v.w);
                    }
                    uint32_t b[NT][2];
#pragma unroll
                    for (int t = 0; t < NT; ++t) { b[t][0] = b4[t][2 * two]; b[t][1] = b4[t][2 * two + 1]; }
                    if (FOLD) {
                        // sum q (z + s c) = sum q z - sum (q s) B + sum (q s) (B + c): the first two are the same for every token, so they
                        // are products with rows that are all alike, made once for both halves
                        const uint32_t za[4] = {as_u32(z2[0]), as_u32(z2[0]), as_u32(z2[1]), as_u32(z2[1])};
                        const uint32_t b0 = code_bias<BITS>(c) | 0x80008000u, b1 = code_bias<BITS>(c + 1) | 0x80008000u, ba[4] = {b0, b0, b1, b1};
#pragma unroll
                        for (int t = 0; t < NT; ++t) {
                            mma16<false>(alike[t], za, b[t][0], b[t][1]);
                            b[t][0] = as_u32(__hmul2(as_half2(b[t][0]), s2[0]));
                            b[t][1] = as_u32(__hmul2(as_half2(b[t][1]), s2[1]));
                            mma16<false>(alike[t], ba, b[t][0], b[t][1]);
                        }
                    }
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        uint32_t a[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e) {        // token g or g + 8 of the half, the first or the second pair
                            const uint32_t word = w[2 * k + (e & 1)];
                            const int ce = c + (e >> 1);
                            if (FOLD) {
                                a[e] = bias.biased(word, ce);
                            } else if (!BF) {
                                a[e] = as_u32(__hfma2(bias.codes(word, ce), s2[e >> 1], z2[e >> 1]));
                            } else {
                                const int l = lo + (e >> 1), h = l + HALF;
                                a[e] = pack16<true>(fmaf(code_float<BITS>(word, ce), meta_at<M16>(ks, l), meta_at<M16>(kz, l)),
                                                    fmaf(code_float<BITS>(word, ce + HALF), meta_at<M16>(ks, h), meta_at<M16>(kz, h)));
                            }
                        }
#pragma unroll
                        for (int t = 0; t < NT; ++t) mma16<BF>(s[t][k], a, b[t][0], b[t][1]);
                    }
                }
            }
        }
        if (FOLD)
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int k = 0; k < 2; ++k)
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[t][k][e] += alike[t][e & 1];
    }
    if (!BF)
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
                for (int e = 0; e < 4; ++e) range.score = max_nan(range.score, fabsf(s[t][k][e]));
    uint32_t pb[NT][2][2];
    softmax_step<NT, BF>(acc, s, scale_log2, pb);
#pragma unroll 1
    for (int k = 0; k < 2; ++k) {
        uint32_t b[NT][2];
#pragma unroll
        for (int t = 0; t < NT; ++t) { b[t][0] = k ? pb[t][1][0] : pb[t][0][0]; b[t][1] = k ? pb[t][1][1] : pb[t][0][1]; }
        uint32_t w[4][BITS / 2];                     // 16 channels of the lane's four tokens
        float sc[4], zr[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int t = 16 * k + 2 * q + (j & 1) + 8 * (j >> 1);
            const unsigned char *from = st + S::VC + t * S::ROW + g * (S::ROW / 8);
            if (BITS == 2) w[j][0] = *reinterpret_cast<const uint32_t *>(from);
            else {
                const uint2 v = *reinterpret_cast<const uint2 *>(from);
                w[j][0] = v.x; w[j][BITS / 2 - 1] = v.y;
            }
            const int at = (t * D + 16 * g) >> g_shift;
            sc[j] = meta_at<M16>(st + S::VS, at);
            zr[j] = meta_at<M16>(st + S::VZ, at);
            if (!BF) range.v = fmaxf(range.v, fmaxf(fabsf(sc[j]), fabsf(zr[j])));      // (as stored: binary16 may make zeros of them)
        }
        __half2 s2[2], z2[2];
        uint32_t both[2][BITS];                      // halves of the words of two tokens
        if (!BF) {
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                s2[e] = __floats2half2_rn(sc[2 * e], sc[2 * e + 1]);
                z2[e] = __floats2half2_rn(zr[2 * e], zr[2 * e + 1]);
#pragma unroll
                for (int i = 0; i < BITS; ++i) both[e][i] = pair16(w[2 * e][i / 2], w[2 * e + 1][i / 2], i);
            }
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            uint32_t a[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {            // tokens 2 q, 2 q + 1 or the later two (e >> 1), channel i or i + 8 (e & 1)
                const int c = i + 8 * (e & 1), j = e >> 1;
                if (!BF) a[e] = as_u32(__hfma2(bias.codes(both[j][c / HALF], c % HALF), s2[j], z2[j]));
                else {
                    constexpr int PER = 2 * HALF;
                    a[e] = pack16<true>(fmaf(code_float<BITS>(w[2 * j][c / PER], c % PER), sc[2 * j], zr[2 * j]),
                                        fmaf(code_float<BITS>(w[2 * j + 1][c / PER], c % PER), sc[2 * j + 1], zr[2 * j + 1]));
                }
            }
#pragma unroll
            for (int t = 0; t < NT; ++t) mma16<BF>(acc.o[t][i], a, b[t][0], b[t][1]);
        }
    }
}

// A step of rows in full precision: rows u0 .. u0 + 31 of the sequence, none from `most` on; row (t, r) of the lane sees the first
// sees[t][r].
template <int BITS, int NT, bool BF>
__device__ __forceinline__ void full_step(const ChunkParams &p, const ChunkSeq &sq, int h, int u0, int most, const int (&sees)[NT][2],
                                       const Queries<NT> &queries, Acc<NT> &acc, Range &range)
{
    constexpr int HALF = BITS == 2 ? 8 : 4;
    const int lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3;
    float s[NT][2][4];
#pragma unroll 1
    for (int k = 0; k < 2; ++k) {
        uint32_t x[2][16];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int u = u0 + 16 * k + 8 * e + g;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                uint4 v = make_uint4(0, 0, 0, 0);
                if (u < most) v = ldg128(p.k_new + (long long)(sq.k0 + u) * p.knt + (long long)h * p.knh + 32 * q + 8 * i);
                x[e][4 * i] = v.x; x[e][4 * i + 1] = v.y; x[e][4 * i + 2] = v.z; x[e][4 * i + 3] = v.w;
            }
        }
        float d[NT][4];
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e) d[t][e] = 0.0f;
#pragma unroll
        for (int four = 0; four < 4; ++four) {
            uint32_t b[NT][4];
#pragma unroll
            for (int t = 0; t < NT; ++t) queries.get(t, four, b[t]);
#pragma unroll
            for (int two = 0; two < 2; ++two) {
                uint32_t a[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int m = 4 * four + 2 * two + (e >> 1), lo = m / HALF * 2 * HALF + m % HALF;
                    a[e] = pair16(x[e & 1][lo / 2], x[e & 1][(lo + HALF) / 2], lo);
                    if (!BF) {                        // infinities and NaN are the same in either type
                        const float v0 = fabsf(bf16lo_to_f32(a[e])), v1 = fabsf(bf16hi_to_f32(a[e]));
                        range.k = fmaxf(range.k, fmaxf(v0 < INFINITY ? v0 : 0.0f, v1 < INFINITY ? v1 : 0.0f));
                        a[e] = bf16_pair_to_f16(a[e]);
                    }
                }
#pragma unroll
                for (int t = 0; t < NT; ++t) mma16<BF>(d[t], a, b[t][2 * two], b[t][2 * two + 1]);
            }
        }
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float v = u0 + 16 * k + g + 8 * (e >> 1) < sees[t][e & 1] ? d[t][e] : -INFINITY;
                if (k == 0) s[t][0][e] = v;
                else s[t][1][e] = v;
            }
    }
    uint32_t pb[NT][2][2];
    softmax_step<NT, BF>(acc, s, p.scale_log2, pb);
    bool odd = false;                                // an infinity or NaN among the lane's values
#pragma unroll 1
    for (int k = 0; k < 2; ++k) {
        uint32_t b[NT][2];
#pragma unroll
        for (int t = 0; t < NT; ++t) { b[t][0] = k ? pb[t][1][0] : pb[t][0][0]; b[t][1] = k ? pb[t][1][1] : pb[t][0][1]; }
        uint32_t w[4][8];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int u = u0 + 16 * k + 2 * q + (j & 1) + 8 * (j >> 1);
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
        for (int i = 0; i < 8; ++i) {
            uint32_t a[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int c = i + 8 * (e & 1), j = e >> 1;
                a[e] = pair16(w[2 * j][c / 2], w[2 * j + 1][c / 2], c);
                if (!BF) a[e] = bf16_pair_to_f16(a[e]);
            }
#pragma unroll
            for (int t = 0; t < NT; ++t) mma16<BF>(acc.o[t][i], a, b[t][0], b[t][1]);
        }
    }
    if (__any_sync(0xffffffffu, odd)) {
        range.odd_first = min(range.odd_first, u0);
        range.odd_last = min(u0 + STEP, most) - 1;
    }
}

// Rare: infinities and NaN among the values of rows [first, last], which were left out of the products, for the rows that see them.
template <int NT>
__device__ __noinline__ void add_not_finite(const __nv_bfloat16 *v0, long long stride, int first, int last, const int *sees, float *o)
{
#pragma unroll 1
    for (int u = first; u <= last; ++u)
#pragma unroll 1
        for (int i = 0; i < 32 * NT; ++i) {          // tile of rows i / 32, channel i / 4 mod 8 (or that + 8), row i mod 2 of the lane's
            const float x = __bfloat162float(v0[u * stride + i / 4 % 8 + 8 * (i >> 1 & 1)]);
            if (!(fabsf(x) < INFINITY) && u < sees[i / 32 * 2 + (i & 1)]) o[i] += x;
        }
}

// Steps [ta, tb) of an item.  Returns whether binary16 was too narrow.
template <int BITS, bool M16, int NT, bool BF>
__device__ __forceinline__ bool run_segment(const ChunkParams &p, const ChunkPlace &pl, const ChunkSeq &sq, int ta, int tb, unsigned char *stages, uint32_t *q_sm, Acc<NT> &acc, Range &range)
{
    using S = Stage<BITS, M16>;
    constexpr int HALF = BITS == 2 ? 8 : 4, R = 8 * NT;
    const int lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3;
    const int rows = sq.nq * p.qpk, row0 = pl.qt * R, g_shift = 31 - __clz(p.G);
    const int ct = sq.cached / STEP;                 // (the group size, and so a length, is a multiple of it)
    range = {};
    range.odd_first = 0x7fffffff;
    range.odd_last = -1;
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        acc.m[t][0] = acc.m[t][1] = -INFINITY;
        acc.l[t][0] = acc.l[t][1] = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc.o[t][i][e] = 0.0f;
    }

    // ---- cached steps
    const int steps = max(min(tb, ct) - ta, 0);
    long long page_tok = 0;                          // lane i: where the tokens of step 32 b + i are; -1: on a page outside the pool
    auto look_up = [&](int first) {
        const int i = first + lane;
        if (i < steps) {
            const int t = (ta + i) * STEP, at = t / p.pool.page_tokens;
            const int page = __ldg(p.page_table + (long long)pl.seq * p.table_stride + at);
            if ((unsigned)page >= (unsigned)p.pool.n_pages) {
                atomicOr(p.status, SQUAT_FLAG_PAGES);
                page_tok = -1;
            } else page_tok = (long long)page * p.pool.page_stride + (long long)pl.h * p.pool.head_stride + (t - at * p.pool.page_tokens);
        }
    };
    const unsigned stage0 = smem_u32(stages);
    auto load = [&](int i) {                         // step i into its stage
        if (i < steps) {
            const long long tok = __shfl_sync(0xffffffffu, page_tok, i & 31);
            if (tok < 0) {                           // no page of anybody's is read: keys and values of zero
#pragma unroll 1
                for (int j = lane; j < S::BYTES / 16; j += 32) reinterpret_cast<uint4 *>(stages + i % STAGES * S::BYTES)[j] = make_uint4(0, 0, 0, 0);
                cp_commit();
                return;
            }
            const unsigned dst = stage0 + i % STAGES * S::BYTES;
            const unsigned char *kc = p.pool.kc + tok * S::ROW, *vc = p.pool.vc + tok * S::ROW;
#pragma unroll
            for (int j = 0; j < BITS; ++j) {
                cp16(dst + S::KC + (32 * j + lane) * 16, kc + (32 * j + lane) * 16);
                cp16(dst + S::VC + (32 * j + lane) * 16, vc + (32 * j + lane) * 16);
            }
            constexpr int KP = D * S::MS / 16, PER_Q = KP / 4;        // pieces of a row of key metadata, and of a quarter
            const unsigned char *ks = static_cast<const unsigned char *>(p.pool.ks) + (tok >> g_shift) * (D * S::MS), *kz = static_cast<const unsigned char *>(p.pool.kz) + (tok >> g_shift) * (D * S::MS);
            if (M16) {
                const int j = lane % KP;
                cp16(dst + (lane < KP ? S::KS : S::KZ) + j / PER_Q * S::QUARTER + j % PER_Q * 16, (lane < KP ? ks : kz) + j * 16);
            } else {
                cp16(dst + S::KS + lane / PER_Q * S::QUARTER + lane % PER_Q * 16, ks + lane * 16);
                cp16(dst + S::KZ + lane / PER_Q * S::QUARTER + lane % PER_Q * 16, kz + lane * 16);
            }
            const int ng = D >> g_shift;                              // value groups of a token: 1, 2 or 4
            if (lane < 2 * S::MS * ng) {                              // 16-byte pieces of 32 tokens' scales
                const unsigned char *vs = static_cast<const unsigned char *>(p.pool.vs) + tok * (ng * S::MS), *vz = static_cast<const unsigned char *>(p.pool.vz) + tok * (ng * S::MS);
                cp16(dst + S::VS + lane * 16, vs + lane * 16);
                cp16(dst + S::VZ + lane * 16, vz + lane * 16);
            }
        }
        cp_commit();
    };
    if (steps > 0) {
        look_up(0);
#pragma unroll
        for (int i = 0; i < STAGES - 1; ++i) load(i);
    }

    // ---- queries: rows 8 t + g, channels 32 q .. + 31, in the order of the key operand
    Queries<NT> queries;
    queries.smem = q_sm + 4 * lane;
    float q_max = 0.0f, q_low = INFINITY;
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const int r = row0 + 8 * t + g;
        float q_row = 0.0f;
        uint32_t x[16];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            uint4 v = make_uint4(0, 0, 0, 0);
            if (r < rows) v = ldg128(p.q + (long long)(sq.q0 + r / p.qpk) * p.qt + (long long)(pl.h * p.qpk + r % p.qpk) * p.qh + 32 * q + 8 * i);
            x[4 * i] = v.x; x[4 * i + 1] = v.y; x[4 * i + 2] = v.z; x[4 * i + 3] = v.w;
        }
        uint32_t y[16];
#pragma unroll
        for (int m = 0; m < 16; ++m) {
            const int lo = m / HALF * 2 * HALF + m % HALF;
            y[m] = pair16(x[lo / 2], x[(lo + HALF) / 2], lo);
            if (!BF) {
                q_row = fmaxf(q_row, fmaxf(fabsf(bf16lo_to_f32(y[m])), fabsf(bf16hi_to_f32(y[m]))));
                y[m] = bf16_pair_to_f16(y[m]);
            }
        }
        if (!BF) {
            q_row = fmaxf(q_row, __shfl_xor_sync(0xffffffffu, q_row, 1));
            q_row = fmaxf(q_row, __shfl_xor_sync(0xffffffffu, q_row, 2));
            q_max = fmaxf(q_max, q_row);
            if (q_row > 0.0f) q_low = fminf(q_low, q_row);
        }
        queries.put(t, y);
    }

    const CodeBias<BITS> bias;
#pragma unroll 1
    for (int i = 0; i < steps; ++i) {
        cp_wait<STAGES - 2>();
        __syncwarp();
        if ((i + STAGES - 1) % 32 == 0) look_up(i + STAGES - 1);
        load(i + STAGES - 1);                        // into the stage of the step before this one
        cached_step<BITS, M16, NT, BF>(stages + i % STAGES * S::BYTES, bias, g_shift, queries, p.scale_log2, acc, range);
        __syncwarp();
    }
    cp_wait<0>();
    __syncwarp();

    // ---- rows in full precision
    const int last = min(rows, row0 + R) - 1, most = chunk_sees(p, sq, last / p.qpk);
    int sees[NT][2];
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int r = 0; r < 2; ++r) sees[t][r] = chunk_sees(p, sq, min(row0 + 8 * t + 2 * q + r, last) / p.qpk);
#pragma unroll 1
    for (int t = max(ta, ct); t < tb; ++t) {
        const int u0 = (t - ct) * STEP;
        if (u0 < most) full_step<BITS, NT, BF>(p, sq, pl.h, u0, most, sees, queries, acc, range);
    }
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int r = 0; r < 2; ++r)
#pragma unroll
            for (int o = 4; o < 32; o <<= 1) acc.l[t][r] += __shfl_xor_sync(0xffffffffu, acc.l[t][r], o);
    if (BF) return false;
    // Dequantized keys and values beyond binary16 have become infinities, and so have scores or sums.  Queries count as beyond it from 2^12
    // on, as in the kernel for many rows.
    constexpr float L = float((1 << BITS) - 1);
    const float2 ks = __half22float2(range.ks), kz = __half22float2(range.kz);
    const float k_top = warp_max(fmaxf(fmaf(L, fmaxf(ks.x, ks.y), fmaxf(kz.x, kz.y)), range.k));
    bool wide = chunk_too_low(p, folds<NT>, warp_max(q_max), warp_min(q_low), k_top);
    wide |= !(q_max < 4096.0f) || !(range.k < 65000.0f) || !(range.score < INFINITY);
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) wide |= !(fabsf(acc.o[t][i][e]) < INFINITY) && acc.m[t][e & 1] < INFINITY;      // (a row with an infinite score of its own has no sum)
    return __any_sync(0xffffffffu, wide) || (!__any_sync(0xffffffffu, range.v >= 0x1p-8f) && __any_sync(0xffffffffu, range.v > 0.0f));
}

template <int BITS, bool M16, int NT>
__global__ void __launch_bounds__(THREADS, CTAS<NT>) chunk_rows_kernel(const __grid_constant__ ChunkParams params)
{
    using S = Stage<BITS, M16>;
    constexpr int R = 8 * NT;
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ ChunkShared sh;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, q = lane & 3;
    ChunkParams p = params;
    chunk_wait(p);
    long long per, total;
    chunk_share<R, STEP>(p, sh, per, total);
    const long long worker = (long long)blockIdx.x * WARPS + warp;
    long long at = per * worker;
    if (per * blockIdx.x * WARPS >= total) return;
    chunk_locate<R, STEP, WARPS>(p, sh, per * blockIdx.x * WARPS, per);
    if (at >= total) return;                         // from here on every warp is by itself
    const long long end = min(at + per, total);
    ChunkPlace pl = sh.found[warp];
    ChunkSeq sq = chunk_seq(p, pl.seq);
    unsigned char *stages = smem + warp * STAGES * S::BYTES;
    uint32_t *q_sm = reinterpret_cast<uint32_t *>(smem + WARPS * STAGES * S::BYTES + warp * Queries<NT>::BYTES);
    while (at < end) {
        const int tiles = chunk_tiles<R, STEP>(p, sq, pl.qt), begin = pl.at, stop = (int)min((long long)p.start + tiles, begin + (end - at));
        const int ta = max(begin - p.start, 0), tb = max(stop - p.start, 0);
        if (ta < tb) {
            Acc<NT> acc;
            Range range;
            if (run_segment<BITS, M16, NT, false>(p, pl, sq, ta, tb, stages, q_sm, acc, range)) run_segment<BITS, M16, NT, true>(p, pl, sq, ta, tb, stages, q_sm, acc, range);
            const int row0 = pl.qt * R, n_rows = min(R, sq.nq * p.qpk - row0);
            if (range.odd_first <= range.odd_last) {
                float o[32 * NT];
                int sees[2 * NT];
#pragma unroll
                for (int i = 0; i < 32 * NT; ++i) o[i] = acc.o[i / 32][i / 4 % 8][i % 4];
#pragma unroll
                for (int i = 0; i < 2 * NT; ++i) sees[i] = chunk_sees(p, sq, min(row0 + i / 2 * 8 + 2 * q + i % 2, sq.nq * p.qpk - 1) / p.qpk);
                add_not_finite<NT>(p.v_new + (long long)sq.k0 * p.vnt + (long long)pl.h * p.vnh + 16 * g, p.vnt, range.odd_first, range.odd_last, sees, o);
#pragma unroll
                for (int i = 0; i < 32 * NT; ++i) acc.o[i / 32][i / 4 % 8][i % 4] = o[i];
            }
            const bool whole = ta == 0 && tb == tiles;
            const long long slot = 2 * worker + (ta == 0 ? 1 : 0);
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    const int row = 8 * t + 2 * q + r;
                    if (row >= n_rows) continue;
                    float y[16];                     // channels 16 g ..
#pragma unroll
                    for (int i = 0; i < 16; ++i) y[i] = acc.o[t][i % 8][i / 8 * 2 + r];
                    const float m = acc.m[t][r], l = acc.l[t][r];
                    if (whole) {
                        const int j = sq.q0 + (row0 + row) / p.qpk, hq = pl.h * p.qpk + (row0 + row) % p.qpk;
                        const float inv = l == 0.0f ? 0.0f : 1.0f / l;
                        uint32_t w[8];
#pragma unroll
                        for (int i = 0; i < 8; ++i) w[i] = pack16<true>(y[2 * i] * inv, y[2 * i + 1] * inv);
                        uint4 *to = reinterpret_cast<uint4 *>(p.out + (long long)j * p.ot + (long long)hq * p.oh + 16 * g);
                        to[0] = make_uint4(w[0], w[1], w[2], w[3]);
                        to[1] = make_uint4(w[4], w[5], w[6], w[7]);
                        if (p.lse && g == 0) p.lse[(long long)j * p.Hq + hq] = l == 0.0f ? -INFINITY : (m - P_SHIFT + log2f(l)) * 0.6931471805599453f;
                    } else {
                        float4 *to = reinterpret_cast<float4 *>(p.part + (slot * R + row) * D + 16 * g);
#pragma unroll
                        for (int i = 0; i < 4; ++i) to[i] = make_float4(y[4 * i], y[4 * i + 1], y[4 * i + 2], y[4 * i + 3]);
                        if (g == 0) *reinterpret_cast<float2 *>(p.ml + (slot * R + row) * 2) = make_float2(m, l);
                    }
                }
            __syncwarp();
        }
        at += stop - begin;
        if (at < end) chunk_next<R>(p, pl, sq);
    }
}

// The item that worker c = blockIdx.x began and did not finish, if there is one.  A warp takes a row, four channels a lane: all the
// row's parts where they are few (BY_ROWS: parts of CTAs' work, of many rows), else every fourth, eight at once, which are joined.
template <int ROWS, int U, bool BY_ROWS>
__global__ void __launch_bounds__(D) chunk_combine_kernel(const __grid_constant__ ChunkParams params)
{
    __shared__ ChunkShared sh;
    __shared__ float4 o_sm[BY_ROWS ? 1 : 4][32];
    __shared__ float2 ml_sm[4];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    // The kernel for few rows lets this one begin when itself has waited for what came earlier, so lengths are there to be read; its
    // parts are waited for below.
    ChunkParams p = params;
    if (BY_ROWS) grid_wait(p.q_start, p.cached_len, p.new_start, p.new_len);
    long long per, total;
    chunk_share<ROWS, U>(p, sh, per, total);
    const long long c = blockIdx.x, border = (c + 1) * per;
    if (border < total) chunk_locate<ROWS, U, 1>(p, sh, border, per);
    if (!BY_ROWS) grid_wait(p.part, p.ml);
    if (border >= total) return;
    const ChunkPlace pl = sh.found[0];
    const long long first = border - pl.at + p.start;        // place of the item's first tile
    if (first >= border || first < c * per) return;
    const ChunkSeq sq = chunk_seq(p, pl.seq);
    const long long parts = (first + chunk_tiles<ROWS, U>(p, sq, pl.qt) - 1) / per - c + 1;
    const int row0 = pl.qt * ROWS, n_rows = min(ROWS, sq.nq * p.qpk - row0);
    constexpr int STRIDE = BY_ROWS ? 1 : 4, AT_ONCE = 8;     // parts of a warp: every STRIDE-th, so many in flight together
#pragma unroll 1
    for (int r = BY_ROWS ? blockIdx.y * 4 + warp : blockIdx.y; r < n_rows; r += gridDim.y * (BY_ROWS ? 4 : 1)) {
        float m = -INFINITY, l = 0.0f;
        float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 1
        for (long long i0 = BY_ROWS ? 0 : warp; i0 < parts; i0 += AT_ONCE * STRIDE) {
            float2 v[AT_ONCE];
            float4 x[AT_ONCE];
#pragma unroll
            for (int i = 0; i < AT_ONCE; ++i) {
                const long long part = i0 + STRIDE * i, at = ((part == 0 ? 2 * c + 1 : 2 * (c + part)) * ROWS + r);
                const bool in = part < parts;
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
        if (!BY_ROWS) {
            __syncthreads();                         // (the row before this one has been read)
            o_sm[warp][lane] = o;
            if (lane == 0) ml_sm[warp] = make_float2(m, l);
            __syncthreads();
            if (warp != 0) continue;
            float mn = m;
#pragma unroll
            for (int w = 1; w < 4; ++w) mn = max_nan(mn, ml_sm[w].x);
            const float use = mn == -INFINITY ? 0.0f : mn, f0 = exp2_fast(m - use);
            l *= f0;
            o.x *= f0; o.y *= f0; o.z *= f0; o.w *= f0;
#pragma unroll
            for (int w = 1; w < 4; ++w) {
                const float f = exp2_fast(ml_sm[w].x - use);
                const float4 x = o_sm[w][lane];
                l = fmaf(f, ml_sm[w].y, l);
                o.x = fmaf(f, x.x, o.x); o.y = fmaf(f, x.y, o.y); o.z = fmaf(f, x.z, o.z); o.w = fmaf(f, x.w, o.w);
            }
            m = mn;
        }
        const int row = row0 + r, j = sq.q0 + row / p.qpk, hq = pl.h * p.qpk + row % p.qpk;
        const float inv = l == 0.0f ? 0.0f : 1.0f / l;
        *reinterpret_cast<uint2 *>(p.out + (long long)j * p.ot + (long long)hq * p.oh + 4 * lane) = make_uint2(pack16<true>(o.x * inv, o.y * inv), pack16<true>(o.z * inv, o.w * inv));
        if (p.lse && lane == 0) p.lse[(long long)j * p.Hq + hq] = l == 0.0f ? -INFINITY : (m - P_SHIFT + log2f(l)) * 0.6931471805599453f;
    }
}

template <int BITS, bool M16, int NT>
constexpr int ROWS_SMEM = WARPS * (STAGES * Stage<BITS, M16>::BYTES + Queries<NT>::BYTES);
// CTAs of an instance to an SM: as many as its registers allow, if shared memory (228 KB, 1 KB of it for every CTA) holds them.  (For 4-bit
// codes with float32 metadata and 8 rows it holds three.  Work shared out among four of them: 64 ragged sequences of up to 4096 tokens x 32
// heads 327 us, a quarter of the CTAs after the others; among three 285.)
template <int BITS, bool M16, int NT>
constexpr int FITTING = [] {
    int n = CTAS<NT>;
    while (n * (ROWS_SMEM<BITS, M16, NT> + (int)sizeof(ChunkShared) + 1024) > 228 * 1024) --n;
    return n;
}();
template <int NT>
int fitting(int bits, int meta16)
{
    return bits == 2 ? meta16 ? FITTING<2, true, NT> : FITTING<2, false, NT> : meta16 ? FITTING<4, true, NT> : FITTING<4, false, NT>;
}
template <int BITS, bool M16, int NT>
int launch_rows(const ChunkParams &p, cudaStream_t st)
{
    constexpr int smem = ROWS_SMEM<BITS, M16, NT>;
    static std::atomic<unsigned long long> allowed{0};
    const int rc = squat_allow_smem(reinterpret_cast<const void *>(chunk_rows_kernel<BITS, M16, NT>), smem, allowed);
    if (rc != SQUAT_OK) return rc;
    return squat_launch(chunk_rows_kernel<BITS, M16, NT>, p.n_workers / WARPS, THREADS, smem, st, p);
}
template <int NT>
int launch_rows_tiles(const ChunkParams &p, int bits, int meta16, cudaStream_t st)
{
    if (bits == 2) return meta16 ? launch_rows<2, true, NT>(p, st) : launch_rows<2, false, NT>(p, st);
    return meta16 ? launch_rows<4, true, NT>(p, st) : launch_rows<4, false, NT>(p, st);
}

// The kernels of a call.  Sequences with at most FEW_ROWS rows per KV head go to the kernel for few rows (8 `eights` of them share an
// item), the others to the kernel for many, in tiles of 128 or 256.  Both sides, us a call, 32 / 8 heads, 2 bits: 16 sequences of up to 8160
// tokens, 16 rows 84 and 119, 24 rows 81 and 122, 32 rows (in an instance of four times eight rows, which is not built) 105 and 114, 48 rows
// 163 and 138; two such sequences, 24 rows 54 and 47, 32 rows 69 and 46; 32 of 2048 tokens at 4 bits, 24 rows 69 and 86, 32 rows 89 and 83.
// So the border lies lower for a few long sequences than for many; their number is not looked at.
struct ChunkKernels {
    int eights;                                      // 0: no kernel for few rows
    int tiles;                                       // 0: no kernel for many rows
};
constexpr int FEW_ROWS = 24;

ChunkKernels kernels_for(long long n_q, long long n_seqs, long long max_q, int qpk)
{
    ChunkKernels k;
    const long long most = max_q * qpk, rows = most <= FEW_ROWS ? most : qpk;
    k.tiles = most <= FEW_ROWS ? 0 : most <= 128 ? 1 : 2;
    k.eights = rows <= 8 ? 1 : rows <= 16 ? 2 : 3;
    // sequences of one length, all of them in the other kernel; or heads that share keys in such numbers that one query is many rows
    if (k.tiles && (n_q == n_seqs * max_q || qpk > FEW_ROWS)) k.eights = 0;
    return k;
}
int rows_workers(int eights, int bits, int meta16)
{
    return WARPS * squat_sm_count() * (eights == 1 ? fitting<1>(bits, meta16) : eights == 2 ? fitting<2>(bits, meta16) : fitting<3>(bits, meta16));
}
int rows_workers(int eights) { return WARPS * squat_sm_count() * (eights == 1 ? CTAS<1> : eights == 2 ? CTAS<2> : CTAS<3>); }      // of any pool
int matrix_workers(int tiles) { return squat_sm_count() * (tiles == 2 ? 1 : 2); }
size_t part_floats(int workers, int rows) { return 2 * (size_t)workers * rows * (D + 2); }
// Workers, at most as many as the longest sequences that the page table can hold would give work to, and their parts.
void use_part(ChunkParams &p, float *at, int workers, int rows, int tile, int together)
{
    const double tokens = (double)p.table_stride * p.pool.page_tokens + p.n_new, row_tiles = (double)p.n_q * p.qpk / rows + p.n_seqs;
    const double most = row_tiles * p.H * (p.start + tokens / tile + 2.0) / p.min_tiles + 1.0;
    p.n_workers = most < workers ? ((int)most + together - 1) / together * together : workers;
    p.part = at;
    p.ml = at + 2 * (size_t)workers * rows * D;
}
template <int ROWS>
int launch_combine(const ChunkParams &p, cudaStream_t st)
{
    // (a CTA for every row that a decode step has; more rows than that in turns of four)
    if constexpr (ROWS >= 128) return squat_launch(chunk_combine_kernel<ROWS, 128, true>, dim3((unsigned)p.n_workers, ROWS / 16), D, 0, st, p);
    else return squat_launch(chunk_combine_kernel<ROWS, STEP, false>, dim3((unsigned)p.n_workers, (unsigned)(p.qpk < ROWS / 4 ? p.qpk : ROWS / 4)), D, 0, st, p);
}

}  // namespace

size_t squat_chunk_workspace_floats(int n_q_heads, int n_kv_heads, int max_q)
{
    const ChunkKernels k = kernels_for(-1, 1, max_q, n_q_heads / n_kv_heads);
    return part_floats(rows_workers(k.eights), 8 * k.eights) + (k.tiles ? part_floats(matrix_workers(k.tiles), 128 * k.tiles) : 0);
}

int squat_launch_chunk_attention(ChunkParams p, const squat_page_pool *pool, float *workspace, int max_q, cudaStream_t st)
{
    p.pool = page_pool_of(pool);
    p.G = pool->group_size;
    p.H = pool->n_kv_heads;
    p.qpk = p.Hq / p.H;
    p.levels = (float)(1 << pool->bits);
    p.status = squat_status_word();
    if (!p.status) return SQUAT_ERR_CUDA;
    const ChunkKernels k = kernels_for(p.n_q, p.n_seqs, max_q, p.qpk);
    ChunkParams few = p, many = p;
    int rc = SQUAT_OK;
    if (k.tiles) {
        many.min_rows = k.eights ? FEW_ROWS + 1 : 1;
        many.max_rows = 0x7fffffff;
        // us a call, 32 / 8 heads: 256 new tokens over 1024 at min_tiles 2 / 4 / 8: 49 / 53 / 62, 1024 without a cache 80 / 80 / 89; 24 mixed
        // sequences at start 0 / 1 / 2 / 4: 215 / 200 / 188 / 177, 8 chunks of 256 72 / 62 / 62 / 63, 2048 over 8192 483 / 495 / 483 / 479
        many.min_tiles = 4;
        many.start = 2;
        use_part(many, workspace, matrix_workers(k.tiles), 128 * k.tiles, 128, 1);
        workspace += part_floats(matrix_workers(k.tiles), 128 * k.tiles);
        rc = squat_launch_chunk_matrix(many, k.tiles, pool->bits, pool->meta16, st);
    }
    if (rc == SQUAT_OK && k.eights) {
        few.min_rows = 1;
        few.max_rows = k.tiles ? FEW_ROWS : 0x7fffffff;
        // us a call: 16 sequences of up to 512 tokens at min_tiles 1 / 3 / 6 / 12: 24 / 22 / 25 / 35, one of 256 13.5 / 15.9 / 20 / 27, one of
        // 32768 52 / 52 / 45 / 44; 64 of up to 4096, 32 heads with keys of their own, at start 0 / 1 / 2 / 4: 320 / 263 / 235 / 213, 24 rows
        // of 16 sequences 85 / 84 / 81 / 80
        few.min_tiles = 3;
        few.start = 2;
        use_part(few, workspace, rows_workers(k.eights, pool->bits, pool->meta16), 8 * k.eights, STEP, WARPS);
        switch (k.eights) {
            case 1: rc = launch_rows_tiles<1>(few, pool->bits, pool->meta16, st); break;
            case 2: rc = launch_rows_tiles<2>(few, pool->bits, pool->meta16, st); break;
            default: rc = launch_rows_tiles<3>(few, pool->bits, pool->meta16, st); break;
        }
    }
    if (rc == SQUAT_OK && k.tiles) rc = k.tiles == 1 ? launch_combine<128>(many, st) : launch_combine<256>(many, st);
    if (rc == SQUAT_OK && k.eights)
        rc = k.eights == 1 ? launch_combine<8>(few, st) : k.eights == 2 ? launch_combine<16>(few, st) : launch_combine<24>(few, st);
    return rc;
}
