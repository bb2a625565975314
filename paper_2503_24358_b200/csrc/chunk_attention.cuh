// Attention of new tokens over a paged cache: parameters, and how the work is dealt out (chunk_attention.cu, chunk_attention_mma.cu).
//
// An item is (sequence, KV head, R rows), a row being a query of one of the KV head's query heads: row r of a sequence is query
// r / qpk of head h qpk + r mod qpk.  Its work is tiles of U tokens: the sequence's cached tokens, then as many of its rows in
// full precision as the item's last query sees.  What an item costs besides (its queries, its first loads, its result) counts
// as `start` tiles in front of them.  All items stand in one line, and worker w (a CTA, or a warp) takes places [w per, (w + 1) per)
// of it, whatever sequences they belong to: a long sequence among short ones, or a single one, is spread over the GPU without the
// host knowing a length.  An item that begins and ends within a worker's places is finished there; of one that crosses a border,
// every worker leaves (sum, maximum, denominator) in the workspace and chunk_combine_kernel adds them up.  A worker has at most two
// such parts: of the item that it begins in the middle of (slot 2 w), and of the one that it begins and does not finish (slot 2 w + 1).
#pragma once
#include "pages.cuh"

struct ChunkParams {
    const __nv_bfloat16 *q;
    __nv_bfloat16 *out;
    float *lse;
    long long qt, qh, ot, oh;                        // element strides
    PagePool pool;
    int G;
    int n_q, Hq, H, qpk, n_seqs, table_stride, n_new, causal;
    const int *q_start, *cached_len, *page_table, *new_start, *new_len;
    const __nv_bfloat16 *k_new, *v_new;
    long long knt, knh, vnt, vnh;
    float scale_log2;                                // softmax scale / ln 2
    float levels;                                    // of a code: L + 1
    int min_rows, max_rows;                          // the kernel's sequences: those with so many rows
    int n_workers, min_tiles, start;                 // who share the work, the least that one takes, and what an item costs besides its tiles
    float *part, *ml;                                // [2 n_workers][R][D], [2 n_workers][R][2]
    unsigned *status;
};

struct ChunkSeq {
    int nq, q0, cached, nk, k0;
};
__device__ __forceinline__ ChunkSeq chunk_seq(const ChunkParams &p, int i)
{
    ChunkSeq s;
    const int a = __ldg(p.q_start + i), b = __ldg(p.q_start + i + 1), c = __ldg(p.cached_len + i);
    const int k0 = p.n_new > 0 ? __ldg(p.new_start + i) : 0, nk = p.n_new > 0 ? __ldg(p.new_len + i) : 0;
    s.q0 = min(max(a, 0), p.n_q);
    s.nq = max(min(b, p.n_q) - s.q0, 0);
    const long long room = p.pool.n_pages > 0 ? (long long)p.table_stride * p.pool.page_tokens : 0;
    s.cached = (int)min((long long)max(c, 0), room);
    s.cached &= -p.G;                                // (a power of two)
    s.k0 = min(max(k0, 0), p.n_new);
    s.nk = min(max(nk, 0), p.n_new - s.k0);
    if (s.q0 != a || s.q0 + s.nq != b || s.cached != c || s.k0 != k0 || s.nk != nk) atomicOr(p.status, SQUAT_FLAG_PAGES);
    const long long rows = (long long)s.nq * p.qpk;
    if (rows < p.min_rows || rows > p.max_rows) s.nq = 0;
    return s;
}
// rows in full precision that query j sees
__device__ __forceinline__ int chunk_sees(const ChunkParams &p, const ChunkSeq &s, int j)
{
    return p.causal ? min(max(s.nk - s.nq + j + 1, 0), s.nk) : s.nk;
}
template <int R>
__device__ __forceinline__ int chunk_row_tiles(const ChunkParams &p, const ChunkSeq &s) { return (int)(((long long)s.nq * p.qpk + R - 1) / R); }
// tiles of the sequence's rows qt R .. of one head; at least one, which writes the zeros of rows that see nothing
template <int R, int U>
__device__ __forceinline__ int chunk_tiles(const ChunkParams &p, const ChunkSeq &s, int qt)
{
    const int last = (int)(min((long long)s.nq * p.qpk, (long long)(qt + 1) * R) - 1) / p.qpk;
    const int n = (s.cached + U - 1) / U + (chunk_sees(p, s, last) + U - 1) / U;
    return max(n, 1);
}
template <int R, int U>
__device__ __forceinline__ long long chunk_head_tiles(const ChunkParams &p, const ChunkSeq &s)
{
    const int n = chunk_row_tiles<R>(p, s);
    long long sum = 0;
    for (int qt = 0; qt < n; ++qt) sum += p.start + chunk_tiles<R, U>(p, s, qt);
    return sum;
}

// A place in the line: item and place within it.
struct ChunkPlace {
    int seq, h, qt, at;
};
struct ChunkShared {
    long long sums[33];
    ChunkPlace found[4];
};

// As grid_wait, but the kernel behind (the sum of the parts) may begin only now: it reads the lengths before it waits itself.
__device__ __forceinline__ void chunk_wait(ChunkParams &p)
{
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("" : "+l"(p.q), "+l"(p.q_start), "+l"(p.cached_len), "+l"(p.page_table), "+l"(p.new_start), "+l"(p.new_len), "+l"(p.k_new), "+l"(p.v_new)::"memory");
}

// All threads of the CTA (a multiple of 32, at most 1024) call this.  per: places per worker, total: of all sequences.
template <int R, int U>
__device__ __forceinline__ void chunk_share(const ChunkParams &p, ChunkShared &sm, long long &per, long long &total)
{
    long long mine = 0;
    for (int i = threadIdx.x; i < p.n_seqs; i += blockDim.x) {
        const ChunkSeq s = chunk_seq(p, i);
        mine += chunk_head_tiles<R, U>(p, s) * p.H;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) mine += __shfl_xor_sync(0xffffffffu, mine, o);
    if ((threadIdx.x & 31) == 0) sm.sums[threadIdx.x >> 5] = mine;
    __syncthreads();
    total = 0;
    for (int w = 0; w < (int)blockDim.x >> 5; ++w) total += sm.sums[w];
    per = max((total + p.n_workers - 1) / p.n_workers, (long long)p.min_tiles);
    __syncthreads();
}
// The items that hold places first, first + per, .. of the line, N of them (those behind its end stay unknown), in sm.found.
template <int R, int U, int N>
__device__ __forceinline__ void chunk_locate(const ChunkParams &p, ChunkShared &sm, long long first, long long per)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    long long before = 0;
    for (int base = 0; base < p.n_seqs; base += blockDim.x) {
        const int i = base + threadIdx.x;
        ChunkSeq s = {};
        long long head = 0, sum;
        if (i < p.n_seqs) {
            s = chunk_seq(p, i);
            head = chunk_head_tiles<R, U>(p, s);
        }
        sum = head * p.H;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long v = __shfl_up_sync(0xffffffffu, sum, o);
            if (lane >= o) sum += v;
        }
        if (lane == 31) sm.sums[warp] = sum;
        __syncthreads();
        long long end = before + sum;
        for (int w = 0; w < warp; ++w) end += sm.sums[w];
        const long long begin = end - head * p.H;
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const long long at = first + k * per;
            if (head > 0 && at >= begin && at < end) {
                // (a sequence's places mostly fit 32 bits, whose division is a tenth of the other)
                const unsigned long long off = at - begin;
                const int in_head = (off | (unsigned long long)head) >> 32 ? (int)(off / head) : (int)((unsigned)off / (unsigned)head);
                long long rest = (long long)off - in_head * head;
                int qt = 0;
                for (int n; rest >= (n = p.start + chunk_tiles<R, U>(p, s, qt)); ++qt) rest -= n;
                sm.found[k] = {i, in_head, qt, (int)rest};
            }
        }
        for (int w = 0; w < warps; ++w) before += sm.sums[w];
        __syncthreads();
        if (before > first + (N - 1) * per) break;
    }
}
// To the next item.
template <int R>
__device__ __forceinline__ void chunk_next(const ChunkParams &p, ChunkPlace &w, ChunkSeq &s)
{
    w.at = 0;
    if (++w.qt < chunk_row_tiles<R>(p, s)) return;
    w.qt = 0;
    if (++w.h < p.H) return;
    w.h = 0;
    do {
        if (++w.seq >= p.n_seqs) return;
        s = chunk_seq(p, w.seq);
    } while (s.nq == 0);
}

// ---- pairs of 16-bit numbers
template <bool BF>
__device__ __forceinline__ uint32_t pack16(float lo, float hi)
{
    if (BF) {
        const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
        return *reinterpret_cast<const uint32_t *>(&v);
    }
    const __half2 v = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&v);
}
__device__ __forceinline__ __half2 as_half2(uint32_t x) { return *reinterpret_cast<const __half2 *>(&x); }
__device__ __forceinline__ uint32_t as_u32(__half2 x) { return *reinterpret_cast<const uint32_t *>(&x); }
__device__ __forceinline__ uint32_t prmt(uint32_t a, uint32_t b, uint32_t sel) { return __byte_perm(a, b, sel); }
// elements i of a and b (two to a word), as a pair
__device__ __forceinline__ uint32_t pair16(uint32_t a, uint32_t b, int i) { return prmt(a, b, i & 1 ? 0x7632 : 0x5410); }
__device__ __forceinline__ float exp2_fast(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// Code c of the low half of `word` and of the high half under the exponent of 2^(10 - s), s the bit where it stands (after one shift
// for the upper codes): a pair of binary16 numbers, bias + code.
template <int BITS>
__device__ __forceinline__ constexpr int code_shift(int c) { return BITS * (c < (BITS == 2 ? 5 : 2) ? c : c - (BITS == 2 ? 5 : 2)); }
template <int BITS>
__device__ __forceinline__ constexpr uint32_t code_bias(int c) { return (uint32_t)(25 - code_shift<BITS>(c)) * 0x04000400u; }
// The biases in registers, where the compiler has to keep them: mask (its immediate) and bias are then one logic instruction, not two.
template <int BITS>
struct CodeBias {
    static constexpr int IN_PLACE = BITS == 2 ? 5 : 2;      // codes whose bits lie within a binary16's significand as they are
    uint32_t at[IN_PLACE];
    __device__ __forceinline__ CodeBias()
    {
#pragma unroll
        for (int c = 0; c < IN_PLACE; ++c) asm volatile("mov.b32 %0, %1;" : "=r"(at[c]) : "r"(code_bias<BITS>(c)));
    }
    __device__ __forceinline__ uint32_t biased(uint32_t word, int c) const
    {
        const uint32_t src = c < IN_PLACE ? word : word >> (BITS * IN_PLACE), mask = ((1u << BITS) - 1u) * 0x00010001u << code_shift<BITS>(c);
        uint32_t d;
        asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(d) : "r"(src), "r"(mask), "r"(at[c % IN_PLACE]));
        return d;
    }
    // the codes themselves
    __device__ __forceinline__ __half2 codes(uint32_t word, int c) const { return __hsub2(as_half2(biased(word, c)), as_half2(code_bias<BITS>(c))); }
};
template <int BITS>
__device__ __forceinline__ float code_float(uint32_t word, int pos) { return (float)(word >> (BITS * pos) & ((1u << BITS) - 1u)); }

__device__ __forceinline__ uint32_t bf16_pair_to_f16(uint32_t x) { return pack16<false>(bf16lo_to_f32(x), bf16hi_to_f32(x)); }
__device__ __forceinline__ bool bf16_pair_not_finite(uint32_t x) { return (x & 0x7f80u) == 0x7f80u || (x & 0x7f800000u) == 0x7f800000u; }

// Whether scores may have lost digits in binary16 that bf16 operands keep.  Below 2^-14 binary16 rounds by up to 2^-25 however small the
// number is: a key's scale (times a code of at most L) and zero-point, a query, and with `fold` the product of a query and a scale.  Over
// 128 channels an exponent is off by `off` at most; q_top: the largest query, k_top: L times the largest scale and the largest
// zero-point together (or the largest key in full precision).  Where that matters, bf16, whose keys are off by 2^-9 of themselves, is
// the better choice once the largest key, the largest channel of a query (q_low: the smallest such one among the rows, zeros apart) or
// their product is so small that 2^-25, L + 1 times for a key, is more than 2^-9 of it: below (L + 1) 2^-16, for k_top, which may be
// four times the largest key, (L + 1) 2^-14.
__device__ __forceinline__ bool chunk_too_low(const ChunkParams &p, bool fold, float q_top, float q_low, float k_top)
{
    const float off = p.scale_log2 * 128.0f * 0x1p-25f * (p.levels * q_top + k_top + (fold ? p.levels : 0.0f)), least = p.levels * 0x1p-14f;
    return !(off <= 0x1p-9f) && (k_top < least || q_low < 0x1p-16f || (fold && q_low * k_top < least));
}

int squat_launch_chunk_matrix(const ChunkParams &p, int tiles, int bits, int meta16, cudaStream_t st);
