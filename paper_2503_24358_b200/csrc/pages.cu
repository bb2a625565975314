// Groups of keys and values quantized into the pages of a paged cache, and read back (squat_pages_write, squat_pages_read).
//
//   Delta = (M - m) RN(1 / L),   c = clamp(rint((x - z) / Delta), 0, L),   x' = z + Delta c     (z = m; or both rounded to binary16)
//
// Delta is a product of binary32 numbers: its last bit may differ from the rounded quotient that the quantizers of contiguous
// caches store.  Codes are decided by the stored grid, so this is no error of theirs; within L 2^-22 steps of the middle between two
// levels they may be the neighbours of a contiguous cache's.  M and m: over G tokens per channel (keys) or G channels per token (values).
//
// Keys: a group is G rows of 256 or 512 contiguous bytes.  16 threads hold a row, eight channels each, eight rows to a thread; the
// minima of a thread's rows (bf16: of channel pairs, packed), of the halves of a warp, then of the group's 2 to 8 warps.  Values: a
// thread holds 32 channels of a token, as the quantizer of contiguous caches does; groups of 64 and 128 are 2 and 4 lanes.
//
// Decisions.  t is bracketed by (x - z) r (1 +- 2^-20), r the hardware reciprocal of Delta (1 ulp); adding 1.5 * 2^23 rounds both
// ends to integers, ties to even, and where they agree that integer is the code.  Both ends are packed by shifted adds; the ends
// differ by one level at most, so the difference of the packed words has a bit for every element that is open (structural with
// bf16 data).  Those are decided one by one (patch).
//
// Bound: HBM (x is read once, codes and metadata are written once; a group's codes are one contiguous span of its page) for what is read
// back: 65536 tokens of 32 heads as bf16 250 us, 5.4 TB/s.  Writes are at neither limit: 131072 tokens of 8 heads, keys and values in
// bf16, 2 bits: 148 us, 4.5 TB/s, 64 % of the issue slots, 21 warps an SM (values alone 72 us).  With a handle: the key kernel (rank 8
// 216 us, dense 331 us for these) into the workspace, 38 us to place its output, and the values: 327 and 443 us.
#include <type_traits>
#include "pages.cuh"

namespace {

constexpr int D = SQUAT_D;
constexpr float kMagic = 12582912.0f;   // 1.5 * 2^23
constexpr int READ_THREADS = 256;
constexpr int ROWS = 8;                 // rows of a group per thread
// groups and threads of a CTA: 64 tokens and 128 threads, or (G = 128) twice as many
template <int G>
struct Cta {
    static constexpr int TOKENS = G < 64 ? 64 : G, GROUPS = TOKENS / G, THREADS = 2 * TOKENS;
};

struct PagesParams {
    PagePool pool;
    const int *slots;
    int n_groups;
    int first;                          // 0: keys and (blockIdx.z = 1) values, 1: values only
    const void *x[2];                   // keys, values
    long long xt[2], xh[2];
    void *y[2];                         // rows that are read back
    unsigned *status;
};

// A group's grid as it is stored, and what decides by it.
template <int BITS, bool M16>
__device__ __forceinline__ void grid_of(float m, float Mx, float &zero, float &delta)
{
    constexpr float invL = 1.0f / float((1 << BITS) - 1);
    delta = __fmul_rn(__fsub_rn(Mx, m), invL);
    zero = m;
    if (M16) {
        delta = __half2float(__float2half_rn(delta));
        zero = __half2float(__float2half_rn(m));
    }
}
struct Ends {
    float ra, rb;                       // reciprocal of the scale, a little more and a little less
    bool ok, fast;
};
__device__ __forceinline__ Ends ends_of(float delta)
{
    Ends e;
    e.ok = delta > 0.0f && delta < __int_as_float(0x7f800000);
    e.fast = delta > 0x1p-100f && delta < 0x1p100f;
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(delta));
    e.ra = __fmul_rn(r, 1.0f + 0x1p-20f);
    e.rb = __fmul_rn(r, 1.0f - 0x1p-20f);
    return e;
}

// A code that the bracket leaves open: `hi`, its upper end, or one less.  The border is k = hi - 1/2, and the sign of (x - z) - k Delta,
// one fma, says on which side x lies; zero is a tie and goes to the even code.  Where x - z is no float32 number (keys), the
// remainder too small for the quotient's own rounding (values) or the scale beyond the bracket's range (slow): the division.
template <int BITS, bool KEY>
__device__ __forceinline__ unsigned decide(float x, float z, float d, unsigned hi, bool slow)
{
    constexpr float L = float((1 << BITS) - 1);
    const float dl = __fsub_rn(x, z), k = (float)hi - 0.5f, r = __fmaf_rn(-k, d, dl), back = __fsub_rn(x, dl);
    const bool sure = KEY ? __fadd_rn(__fsub_rn(x, __fadd_rn(dl, back)), __fsub_rn(back, z)) == 0.0f : r == 0.0f || fabsf(r) > k * d * 0x1p-21f;
    if (sure && !slow) return r > 0.0f || (r == 0.0f && (hi & 1u) == 0) ? hi : hi - 1u;
    if (KEY) return (unsigned)(int)fmin(fmax(rint(__ddiv_rn((double)x - (double)z, (double)d)), 0.0), (double)L);
    return (unsigned)(int)fminf(fmaxf(rintf(__fdiv_rn(dl, d)), 0.0f), L);
}
template <bool BF16>
__device__ __forceinline__ float element(const void *src, long long at)
{
    return BF16 ? __uint_as_float((unsigned)__ldg(static_cast<const unsigned short *>(src) + at) << 16) : __ldg(static_cast<const float *>(src) + at);
}
// A word of a token's values, one bit of `open` for each open code; out of line, and from memory again (it is in L1), so that the
// streaming code stays small.
template <int BITS, bool BF16>
__device__ __noinline__ unsigned patch_values(unsigned word, unsigned open, const void *src, long long at, float zero, float delta, bool slow)
{
    constexpr unsigned FIELD = (1u << BITS) - 1u;
    while (open) {
        const int pos = __ffs(open) - 1;
        open &= open - 1;
        word = (word & ~(FIELD << pos)) | decide<BITS, false>(element<BF16>(src, at + pos / BITS), zero, delta, word >> pos & FIELD, slow) << pos;
    }
    return word;
}

// Both ends of N codes (N * BITS <= 32, N even), packed low bits first.  zero2, ra2, rb2: pairs of neighbouring elements', STEP pairs apart
template <int BITS, int N, int STEP, bool M16>
__device__ __forceinline__ void pack_ends(const u64 *x2, const u64 *zero2, const u64 *ra2, const u64 *rb2, unsigned &a, unsigned &b)
{
    constexpr float L = float((1 << BITS) - 1);
    constexpr unsigned K = [] { unsigned k = 0; for (int i = 0; i < N; ++i) k += 0x4B400000u << (BITS * i); return k; }();
    const u64 magic2 = pack2(kMagic, kMagic);
    a = b = 0u - K;                     // what the constant upper bits add up to
#pragma unroll
    for (int i = 0; i < N / 2; ++i) {
        const u64 dl = fsub2(x2[i], zero2[i * STEP]);
        float a0, a1, b0, b1;
        unpack2(ffma2(dl, ra2[i * STEP], magic2), a0, a1);
        unpack2(ffma2(dl, rb2[i * STEP], magic2), b0, b1);
        if (M16) {                      // a rounded zero-point may lie above the minimum
            a0 = fminf(fmaxf(a0, kMagic), kMagic + L); b0 = fminf(fmaxf(b0, kMagic), kMagic + L);
            a1 = fminf(fmaxf(a1, kMagic), kMagic + L); b1 = fminf(fmaxf(b1, kMagic), kMagic + L);
        }
        a += __float_as_uint(a0) << (BITS * 2 * i);
        a += __float_as_uint(a1) << (BITS * (2 * i + 1));
        b += __float_as_uint(b0) << (BITS * 2 * i);
        b += __float_as_uint(b1) << (BITS * (2 * i + 1));
    }
}
template <int BITS, int N>
constexpr unsigned LOW_BITS = [] { unsigned m = 0; for (int i = 0; i < N; ++i) m |= 1u << (BITS * i); return m; }();

// Eight channels of a row as they were loaded; widened where they are used.
template <bool BF16>
struct Row8;
template <>
struct Row8<true> {
    uint4 r;
    __device__ __forceinline__ void load(const void *p, long long at) { r = ldg128(static_cast<const __nv_bfloat16 *>(p) + at); }
    __device__ __forceinline__ u64 pair(int i) const
    {
        const uint32_t w = i == 0 ? r.x : i == 1 ? r.y : i == 2 ? r.z : r.w;
        return pack2(bf16lo_to_f32(w), bf16hi_to_f32(w));
    }
    __device__ __forceinline__ void blank(int i, bool lo, bool hi)            // channels of pair i become zero
    {
        uint32_t &w = i == 0 ? r.x : i == 1 ? r.y : i == 2 ? r.z : r.w;
        w &= (lo ? 0u : 0xffffu) | (hi ? 0u : 0xffff0000u);
    }
};
template <>
struct Row8<false> {
    float4 a, b;
    __device__ __forceinline__ void load(const void *p, long long at)
    {
        const float4 *s = reinterpret_cast<const float4 *>(static_cast<const float *>(p) + at);
        a = __ldg(s);
        b = __ldg(s + 1);
    }
    __device__ __forceinline__ u64 pair(int i) const { return i == 0 ? pack2(a.x, a.y) : i == 1 ? pack2(a.z, a.w) : i == 2 ? pack2(b.x, b.y) : pack2(b.z, b.w); }
    __device__ __forceinline__ void blank(int i, bool lo, bool hi)
    {
        float4 &v = i < 2 ? a : b;
        float &x = i % 2 ? v.z : v.x, &y = i % 2 ? v.w : v.y;
        x = lo ? 0.0f : x;
        y = hi ? 0.0f : y;
    }
};
// Minimum and maximum of pairs of channels: packed bf16, or two floats.
template <bool BF16>
struct MinMax2;
template <>
struct MinMax2<true> {
    unsigned lo, hi;
    __device__ __forceinline__ void start(const Row8<true> &r, int i) { lo = hi = i == 0 ? r.r.x : i == 1 ? r.r.y : i == 2 ? r.r.z : r.r.w; }
    __device__ __forceinline__ void join(const MinMax2 &o) { lo = hmin2_nan_bits(lo, o.lo); hi = hmax2_nan_bits(hi, o.hi); }
    __device__ __forceinline__ MinMax2 other(int lanes) const { return {__shfl_xor_sync(0xffffffffu, lo, lanes), __shfl_xor_sync(0xffffffffu, hi, lanes)}; }
    __device__ __forceinline__ float2 min2() const { return make_float2(bf16lo_to_f32(lo), bf16hi_to_f32(lo)); }
    __device__ __forceinline__ float2 max2() const { return make_float2(bf16lo_to_f32(hi), bf16hi_to_f32(hi)); }
};
template <>
struct MinMax2<false> {
    float2 lo, hi;
    __device__ __forceinline__ void start(const Row8<false> &r, int i)
    {
        float x, y;
        unpack2(r.pair(i), x, y);
        lo = hi = make_float2(x, y);
    }
    __device__ __forceinline__ void join(const MinMax2 &o)
    {
        lo = make_float2(min_nan(lo.x, o.lo.x), min_nan(lo.y, o.lo.y));
        hi = make_float2(max_nan(hi.x, o.hi.x), max_nan(hi.y, o.hi.y));
    }
    __device__ __forceinline__ MinMax2 other(int lanes) const
    {
        return {make_float2(__shfl_xor_sync(0xffffffffu, lo.x, lanes), __shfl_xor_sync(0xffffffffu, lo.y, lanes)),
                make_float2(__shfl_xor_sync(0xffffffffu, hi.x, lanes), __shfl_xor_sync(0xffffffffu, hi.y, lanes))};
    }
    __device__ __forceinline__ float2 min2() const { return lo; }
    __device__ __forceinline__ float2 max2() const { return hi; }
};

template <bool M16>
__device__ __forceinline__ void store_meta(void *p, long long i, float v)
{
    if (M16) static_cast<__half *>(p)[i] = __float2half_rn(v);          // exact: already a binary16 value
    else static_cast<float *>(p)[i] = v;
}
template <bool M16>
__device__ __forceinline__ float load_meta(const void *p, long long i)
{
    return M16 ? __half2float(__ldg(static_cast<const __half *>(p) + i)) : __ldg(static_cast<const float *>(p) + i);
}

// A group's first token in the pool, or -1: padding or (flagged) a slot that is none.
template <int G>
__device__ __forceinline__ long long group_token(const PagesParams &p, const int *slots, int group, int h)
{
    const int slot = __ldg(slots + group);
    if (slot < 0) return -1;
    if (slot % G != 0 || slot / p.pool.page_tokens >= p.pool.n_pages) {
        atomicOr(p.status, SQUAT_FLAG_PAGES);
        return -1;
    }
    return token_at_slot(p.pool, slot, h);
}

// The threads of one of a CTA's groups.  (Barriers by constant numbers: a number in a register reserves all sixteen, and CTAs with
// sixteen each are few to an SM.)
template <int GROUPS, int N>
__device__ __forceinline__ void sync_group(int group)
{
    if (GROUPS == 1) __syncthreads();
    else if (group == 0) asm volatile("bar.sync 1, %0;" ::"n"(N) : "memory");
    else asm volatile("bar.sync 2, %0;" ::"n"(N) : "memory");
}

template <int G, int BITS, bool BF16, bool M16>
__device__ __forceinline__ void write_keys(const PagesParams &p, const void *src, const int *slots)
{
    using C = Cta<G>;
    constexpr int WARPS = G / 16, LANES = G / ROWS;          // of a group; threads of a group that share a channel
    using word_t = typename std::conditional<BITS == 2, unsigned short, unsigned>::type;         // eight codes
    __shared__ MinMax2<BF16> ends_sm[C::GROUPS][WARPS][D / 2];
    __shared__ __align__(16) word_t words_sm[C::TOKENS][16];
    __shared__ word_t open_sm[ROWS][C::THREADS];
    __shared__ __align__(16) float2 zero_sm[C::GROUPS][D / 2], delta_sm[C::GROUPS][D / 2];
    const int h = blockIdx.y, tid = threadIdx.x, c8 = tid & 15, r0 = (tid >> 4) % LANES, mine = tid / (16 * LANES), group = blockIdx.x * C::GROUPS + mine;
    const long long tok = group < p.n_groups ? group_token<G>(p, slots, group, h) : -1;
    const long long at = ((long long)group * G + r0) * p.xt[0] + (long long)h * p.xh[0] + 8 * c8;
    Row8<BF16> x[ROWS];
    if (tok >= 0) {
#pragma unroll
        for (int i = 0; i < ROWS; ++i) x[i].load(src, at + (long long)(LANES * i) * p.xt[0]);
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            MinMax2<BF16> e, o;
            e.start(x[0], c);
#pragma unroll
            for (int i = 1; i < ROWS; ++i) {
                o.start(x[i], c);
                e.join(o);
            }
            e.join(e.other(16));                             // (a warp's rows belong to one group)
            if ((tid & 16) == 0) ends_sm[mine][(tid >> 5) % WARPS][4 * c8 + c] = e;
        }
    }
    __syncthreads();
    const int pr = tid % (16 * LANES);                       // a pair of channels' grids
    if (tok >= 0 && pr < D / 2) {
        MinMax2<BF16> e = ends_sm[mine][0][pr];
#pragma unroll
        for (int w = 1; w < WARPS; ++w) e.join(ends_sm[mine][w][pr]);
        const float2 lo = e.min2(), hi = e.max2();
        float2 z, d;
        grid_of<BITS, M16>(lo.x, hi.x, z.x, d.x);
        grid_of<BITS, M16>(lo.y, hi.y, z.y, d.y);
        zero_sm[mine][pr] = z;
        delta_sm[mine][pr] = d;
        const long long to = tok / G * (D / 2) + pr;
        if (M16) {
            static_cast<__half2 *>(p.pool.ks)[to] = __floats2half2_rn(d.x, d.y);
            static_cast<__half2 *>(p.pool.kz)[to] = __floats2half2_rn(z.x, z.y);
        } else {
            static_cast<float2 *>(p.pool.ks)[to] = d;
            static_cast<float2 *>(p.pool.kz)[to] = z;
        }
        const bool none = d.x == 0.0f || d.y == 0.0f, odd = !(d.x < INFINITY && d.y < INFINITY);
        if (none || odd) atomicOr(p.status, (none ? SQUAT_FLAG_ZERO_RANGE : 0u) | (odd ? SQUAT_FLAG_NONFINITE : 0u));
    }
    __syncthreads();
    if (tok < 0) return;
    u64 zero2[4], ra2[4], rb2[4];
    unsigned keep = 0, slow = 0;                             // fields of channels with a grid; bits of those the bracket is not good for
#pragma unroll
    for (int c = 0; c < 4; ++c) {
        const float2 z = zero_sm[mine][4 * c8 + c], d = delta_sm[mine][4 * c8 + c];
        const Ends a = ends_of(d.x), b = ends_of(d.y);
        zero2[c] = pack2(z.x, z.y);
        ra2[c] = pack2(a.ra, b.ra);
        rb2[c] = pack2(a.rb, b.rb);
        keep |= (a.ok ? ((1u << BITS) - 1u) << (BITS * 2 * c) : 0u) | (b.ok ? ((1u << BITS) - 1u) << (BITS * (2 * c + 1)) : 0u);
        slow |= (a.fast ? 0u : 1u << (BITS * 2 * c)) | (b.fast ? 0u : 1u << (BITS * (2 * c + 1)));
        // Channels without a grid, or with one beyond the bracket's range: their ends are no codes (0 times infinity, as a rule), and in the
        // sum of a word they would spill into the fields above.  They enter it as zeros; those with a grid are decided by the division
        // below.  (Ends that are clamped spill nothing.)
        if (!M16 && !(a.ok && a.fast && b.ok && b.fast)) {
            const bool lo = !(a.ok && a.fast), hi = !(b.ok && b.fast);
            zero2[c] = pack2(lo ? 0.0f : z.x, hi ? 0.0f : z.y);
            ra2[c] = pack2(lo ? 0.0f : a.ra, hi ? 0.0f : b.ra);
            rb2[c] = pack2(lo ? 0.0f : a.rb, hi ? 0.0f : b.rb);
#pragma unroll
            for (int i = 0; i < ROWS; ++i) x[i].blank(c, lo, hi);
        }
    }
    // words first; the open ones of all rows then in one loop, so that a warp's lanes take theirs at the same time
    unsigned rows = 0;
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        u64 x2[4];
#pragma unroll
        for (int c = 0; c < 4; ++c) x2[c] = x[i].pair(c);
        unsigned word, low;
        pack_ends<BITS, 8, 1, M16>(x2, zero2, ra2, rb2, word, low);
        const unsigned open = ((word - low) | slow) & keep & LOW_BITS<BITS, 8>;
        words_sm[r0 + LANES * i + G * mine][c8] = (word_t)(word & keep);
        if (open) {
            rows |= 1u << i;
            open_sm[i][tid] = (word_t)open;
        }
    }
    if (rows) {
        unsigned open = 0;
        int i = 0;
        while (rows | open) {
            if (open == 0) {
                i = __ffs(rows) - 1;
                rows &= rows - 1;
                open = open_sm[i][tid];
            }
            constexpr unsigned FIELD = (1u << BITS) - 1u;
            const int pos = __ffs(open) - 1, c = pos / BITS;
            open &= open - 1;
            word_t &to = words_sm[r0 + LANES * i + G * mine][c8];
            const unsigned word = to;
            to = (word_t)((word & ~(FIELD << pos)) | decide<BITS, true>(element<BF16>(src, at + (long long)(LANES * i) * p.xt[0] + c), (&zero_sm[mine][4 * c8].x)[c], (&delta_sm[mine][4 * c8].x)[c],
                                                                       word >> pos & FIELD, slow >> pos & 1u) << pos);
        }
    }
    // a warp's rows of step i are two neighbouring tokens; the codes of the group are one span
    sync_group<C::GROUPS, 16 * LANES>(mine);
    uint4 *to = reinterpret_cast<uint4 *>(p.pool.kc + tok * (D * BITS / 8));
#pragma unroll
    for (int i = 0; i < G * BITS / (16 * LANES); ++i) to[pr + 16 * LANES * i] = reinterpret_cast<const uint4 *>(&words_sm[G * mine][0])[pr + 16 * LANES * i];
}

// Four lanes a token, two tokens a thread
template <int G, int BITS, bool BF16, bool M16>
__device__ __forceinline__ void write_values(const PagesParams &p, const void *src, const int *slots)
{
    using C = Cta<G>;
    constexpr int LANES = G / 32, PER_WORD = 32 / BITS, WORDS = BITS;        // lanes of a group; words of a thread's codes
    const int h = blockIdx.y, tid = threadIdx.x, span = tid & 3;
    Row8<BF16> x[2][4];
    long long tok[2], at[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int t = (tid >> 2) + C::TOKENS / 2 * j;                        // token of the CTA
        const int group = blockIdx.x * C::GROUPS + t / G;
        tok[j] = group < p.n_groups ? group_token<G>(p, slots, group, h) : -1;
        if (tok[j] < 0) continue;
        tok[j] += t % G;
        at[j] = ((long long)blockIdx.x * C::TOKENS + t) * p.xt[1] + (long long)h * p.xh[1] + 32 * span;
#pragma unroll
        for (int i = 0; i < 4; ++i) x[j][i].load(src, at[j] + 8 * i);
    }
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        if (tok[j] < 0) continue;                            // (all lanes of a warp hold tokens of one group, or of one and a missing one)
        MinMax2<BF16> e, o;
        e.start(x[j][0], 0);
#pragma unroll
        for (int i = 1; i < 16; ++i) {
            o.start(x[j][i / 4], i % 4);
            e.join(o);
        }
#pragma unroll
        for (int l = 1; l < LANES; l <<= 1) e.join(e.other(l));
        const float2 lo = e.min2(), hi = e.max2();
        float zero, delta;
        grid_of<BITS, M16>(min_nan(lo.x, lo.y), max_nan(hi.x, hi.y), zero, delta);
        const Ends r = ends_of(delta);
        const u64 zero2 = pack2(zero, zero), ra2 = pack2(r.ra, r.ra), rb2 = pack2(r.rb, r.rb);
        unsigned words[WORDS];
#pragma unroll
        for (int w = 0; w < WORDS; ++w) {
            u64 x2[PER_WORD / 2];
#pragma unroll
            for (int i = 0; i < PER_WORD / 2; ++i) x2[i] = x[j][(w * PER_WORD / 2 + i) / 4].pair((w * PER_WORD / 2 + i) % 4);
            unsigned word, low;
            pack_ends<BITS, PER_WORD, 0, M16>(x2, &zero2, &ra2, &rb2, word, low);
            unsigned open = r.fast ? word - low : LOW_BITS<BITS, PER_WORD>;
            if (open && r.ok) word = patch_values<BITS, BF16>(word, open, src, at[j] + w * PER_WORD, zero, delta, !r.fast);
            words[w] = r.ok ? word : 0u;
        }
        unsigned char *to = p.pool.vc + tok[j] * (D * BITS / 8) + span * (4 * BITS);
        if (BITS == 2) *reinterpret_cast<uint2 *>(to) = make_uint2(words[0], words[1]);
        else *reinterpret_cast<uint4 *>(to) = make_uint4(words[0], words[1], words[BITS - 2], words[BITS - 1]);
        if (span % LANES == 0) {
            const long long m = tok[j] * (D / G) + span / LANES;
            store_meta<M16>(p.pool.vs, m, delta);
            store_meta<M16>(p.pool.vz, m, zero);
            if (!r.ok) atomicOr(p.status, delta == 0.0f ? SQUAT_FLAG_ZERO_RANGE : SQUAT_FLAG_NONFINITE);
        }
    }
}

// grid (CTAs' tokens, heads, keys / values)
template <int G, int BITS, bool BF16, bool M16>
__global__ void __launch_bounds__(Cta<G>::THREADS, (BF16 ? 6 : 4) * 128 / Cta<G>::THREADS) pages_write_kernel(PagesParams p)
{
    const int part = p.first + blockIdx.z;
    const void *src = p.x[part];
    const int *slots = p.slots;
    grid_wait(src, slots);
    if (part == 0) write_keys<G, BITS, BF16, M16>(p, src, slots);
    else write_values<G, BITS, BF16, M16>(p, src, slots);
}

// Keys that squat_quantize_keys has left in the workspace, [heads, tokens]: codes x[0], metadata x[1] (scales, then zero-points
// y[0]); a group's codes are one span on either side.
template <int G, int BITS, bool M16>
__global__ void __launch_bounds__(128) pages_place_kernel(PagesParams p)
{
    const int h = blockIdx.y, tid = threadIdx.x;
    const unsigned char *codes = static_cast<const unsigned char *>(p.x[0]);
    const void *scales = p.x[1], *zeros = p.y[0];
    const int *slots = p.slots;
    grid_wait(codes, scales, zeros, slots);
    const long long tok = group_token<G>(p, slots, blockIdx.x, h);
    if (tok < 0) return;
    const long long from = (long long)h * p.n_groups + blockIdx.x;
    constexpr int CODES16 = G * BITS, META16 = D * (M16 ? 2 : 4) / 16;       // 16-byte pieces
    const uint4 *src = reinterpret_cast<const uint4 *>(codes) + from * CODES16;
    uint4 *dst = reinterpret_cast<uint4 *>(p.pool.kc + tok * (D * BITS / 8));
    for (int i = tid; i < CODES16; i += 128) dst[i] = __ldg(src + i);
    if (tid < 2 * META16) {
        const bool zero = tid >= META16;
        const int i = tid - (zero ? META16 : 0);
        const uint4 v = __ldg(static_cast<const uint4 *>(zero ? zeros : scales) + from * META16 + i);
        (static_cast<uint4 *>(zero ? p.pool.kz : p.pool.ks) + tok / G * META16)[i] = v;
    }
}

// Channels 2 I, 2 I + 1 of a thread's eight codes as two exact floats: a code, masked where it stands at bit s, under the exponent of
// 2^(23 - s) makes 2^(23 - s) + code, and the subtraction of the bias leaves the code.  4-bit codes 4 .. 7 are taken from word >> 16.
template <int BITS, int I>
__device__ __forceinline__ u64 codes_as_floats(unsigned word)
{
    constexpr int S0 = (BITS * 2 * I) % 16, S1 = (BITS * (2 * I + 1)) % 16;
    constexpr unsigned FIELD = (1u << BITS) - 1u, B0 = (unsigned)(150 - S0) << 23, B1 = (unsigned)(150 - S1) << 23;
    const unsigned w = BITS == 4 && I >= 2 ? word >> 16 : word;
    return fsub2(pack2(__uint_as_float((w & FIELD << S0) | B0), __uint_as_float((w & FIELD << S1) | B1)), pack2(__uint_as_float(B0), __uint_as_float(B1)));
}

// grid (runs of tokens, heads, keys / values): a thread takes eight channels of eight consecutive tokens, which lie in one
// group, so the eight scales and zero-points of a key group are read once for all of them.  A half-warp's stores are whole rows: channels
// 8 c .. of a bf16 row, 4 c .. and 64 + 4 c .. of a float32 row.
template <int G, int BITS, bool BF16, bool M16>
__global__ void __launch_bounds__(READ_THREADS, 4) pages_read_kernel(PagesParams p)
{
    constexpr int TOK = 8, APART = BF16 ? 4 : D / 2;             // from the thread's first four channels to its others
    constexpr int VG = !BF16 && G <= D / 2 ? 2 : 1;              // value groups of a token that its channels lie in
    const int part = p.first + blockIdx.z, h = blockIdx.y, c8 = threadIdx.x & 15, c0 = c8 * (BF16 ? 8 : 4);
    const long long run = (long long)blockIdx.x * (READ_THREADS / 16) + (threadIdx.x >> 4);
    const int group = (int)(run / (G / TOK)), in_group = (int)(run % (G / TOK)) * TOK;
    const unsigned char *codes = part == 0 ? p.pool.kc : p.pool.vc;
    const void *scales = part == 0 ? p.pool.ks : p.pool.vs, *zeros = part == 0 ? p.pool.kz : p.pool.vz;
    const int *slots = p.slots;
    grid_wait(codes, scales, zeros, slots);
    if (group >= p.n_groups) return;
    long long tok = group_token<G>(p, slots, group, h);
    if (tok < 0) return;
    tok += in_group;
    unsigned words[TOK];                         // eight codes
    const unsigned char *from = codes + tok * (D * BITS / 8) + c0 * BITS / 8;
#pragma unroll
    for (int i = 0; i < TOK; ++i) {
        const unsigned char *f = from + i * (D * BITS / 8);
        if (BF16) words[i] = BITS == 2 ? (unsigned)__ldg(reinterpret_cast<const unsigned short *>(f)) : __ldg(reinterpret_cast<const unsigned *>(f));
        else if (BITS == 2) words[i] = (unsigned)__ldg(f) | (unsigned)__ldg(f + D / 2 * BITS / 8) << 8;
        else words[i] = (unsigned)__ldg(reinterpret_cast<const unsigned short *>(f)) | (unsigned)__ldg(reinterpret_cast<const unsigned short *>(f + D / 2 * BITS / 8)) << 16;
    }
    u64 s2[4], z2[4];                            // of the channels (keys)
    float sv[TOK][VG], zv[TOK][VG];              // of the tokens (values)
    if (part == 0) {
        const long long at = tok / G * D + c0;
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            if (M16) {
                const uint2 a = __ldg(reinterpret_cast<const uint2 *>(static_cast<const __half *>(scales) + at + APART * c)), b = __ldg(reinterpret_cast<const uint2 *>(static_cast<const __half *>(zeros) + at + APART * c));
                const uint32_t aw[2] = {a.x, a.y}, bw[2] = {b.x, b.y};
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const float2 u = __half22float2(*reinterpret_cast<const __half2 *>(&aw[k])), v = __half22float2(*reinterpret_cast<const __half2 *>(&bw[k]));
                    s2[2 * c + k] = pack2(u.x, u.y);
                    z2[2 * c + k] = pack2(v.x, v.y);
                }
            } else {
                const float4 u = __ldg(reinterpret_cast<const float4 *>(static_cast<const float *>(scales) + at + APART * c)), v = __ldg(reinterpret_cast<const float4 *>(static_cast<const float *>(zeros) + at + APART * c));
                s2[2 * c] = pack2(u.x, u.y); s2[2 * c + 1] = pack2(u.z, u.w);
                z2[2 * c] = pack2(v.x, v.y); z2[2 * c + 1] = pack2(v.z, v.w);
            }
        }
    } else {
        const long long at = tok * (D / G) + c0 / G;
#pragma unroll
        for (int i = 0; i < TOK; ++i)
#pragma unroll
            for (int k = 0; k < VG; ++k) {
                sv[i][k] = load_meta<M16>(scales, at + i * (D / G) + APART / G * k);
                zv[i][k] = load_meta<M16>(zeros, at + i * (D / G) + APART / G * k);
            }
    }
    const long long at = ((long long)group * G + in_group) * p.xt[part] + (long long)h * p.xh[part] + c0;
#pragma unroll
    for (int i = 0; i < TOK; ++i) {
        const u64 code2[4] = {codes_as_floats<BITS, 0>(words[i]), codes_as_floats<BITS, 1>(words[i]), codes_as_floats<BITS, 2>(words[i]), codes_as_floats<BITS, 3>(words[i])};
        float y[8];
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            const float s = sv[i][c / 2 % VG], z = zv[i][c / 2 % VG];
            unpack2(part == 0 ? ffma2(code2[c], s2[c], z2[c]) : ffma2(code2[c], pack2(s, s), pack2(z, z)), y[2 * c], y[2 * c + 1]);
        }
        const long long to = at + i * p.xt[part];
        if (BF16) {
            uint32_t w[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const __nv_bfloat162 v = __floats2bfloat162_rn(y[2 * k], y[2 * k + 1]);
                w[k] = *reinterpret_cast<const uint32_t *>(&v);
            }
            *reinterpret_cast<uint4 *>(static_cast<__nv_bfloat16 *>(p.y[part]) + to) = make_uint4(w[0], w[1], w[2], w[3]);
        } else {
            float *f = static_cast<float *>(p.y[part]) + to;
            *reinterpret_cast<float4 *>(f) = make_float4(y[0], y[1], y[2], y[3]);
            *reinterpret_cast<float4 *>(f + APART) = make_float4(y[4], y[5], y[6], y[7]);
        }
    }
}

template <int G, int BITS>
int launch_inst(const PagesParams &p, bool write, dim3 grid, int dtype, int meta16, cudaStream_t st)
{
    const bool bf = dtype == SQUAT_BF16;
    grid.x = write ? (unsigned)((p.n_groups + Cta<G>::GROUPS - 1) / Cta<G>::GROUPS) : (unsigned)(((long long)p.n_groups * (G / 8) + READ_THREADS / 16 - 1) / (READ_THREADS / 16));
#define SQ_P(K, T, BF, MM) return squat_launch(K<G, BITS, BF, MM>, grid, T, 0, st, p)
    if (write) {
        if (bf) { if (meta16) SQ_P(pages_write_kernel, Cta<G>::THREADS, true, true); else SQ_P(pages_write_kernel, Cta<G>::THREADS, true, false); }
        else { if (meta16) SQ_P(pages_write_kernel, Cta<G>::THREADS, false, true); else SQ_P(pages_write_kernel, Cta<G>::THREADS, false, false); }
    } else {
        if (bf) { if (meta16) SQ_P(pages_read_kernel, READ_THREADS, true, true); else SQ_P(pages_read_kernel, READ_THREADS, true, false); }
        else { if (meta16) SQ_P(pages_read_kernel, READ_THREADS, false, true); else SQ_P(pages_read_kernel, READ_THREADS, false, false); }
    }
#undef SQ_P
}

int launch_sized(const PagesParams &p, bool write, dim3 grid, const squat_page_pool *pool, int dtype, cudaStream_t st)
{
#define SQ_P(GG, BB) return launch_inst<GG, BB>(p, write, grid, dtype, pool->meta16, st)
    if (pool->bits == 2) { if (pool->group_size == 32) SQ_P(32, 2); if (pool->group_size == 64) SQ_P(64, 2); SQ_P(128, 2); }
    if (pool->group_size == 32) SQ_P(32, 4);
    if (pool->group_size == 64) SQ_P(64, 4);
    SQ_P(128, 4);
#undef SQ_P
}

}  // namespace

int squat_launch_pages(bool write, const squat_page_pool *pool, const int *slots, int n_groups, int dtype,
                       const void *const (&x)[2], void *const (&y)[2], const long long (&strides)[2][2], unsigned *status, cudaStream_t st)
{
    PagesParams p;
    p.pool = page_pool_of(pool);
    p.slots = slots;
    p.n_groups = n_groups;
    p.status = status;
    int parts = 0;
    p.first = 1;
    for (int i = 0; i < 2; ++i) {
        p.x[i] = x[i];
        p.y[i] = y[i];
        p.xt[i] = strides[i][0];
        p.xh[i] = strides[i][1];
        if (!x[i] && !y[i]) continue;
        ++parts;
        if (i == 0) p.first = 0;
    }
    if (parts == 0) return SQUAT_OK;
    return launch_sized(p, write, dim3(1, (unsigned)pool->n_kv_heads, (unsigned)parts), pool, dtype, st);
}

int squat_launch_pages_place(const squat_page_pool *pool, const int *slots, int n_groups, const void *codes, const void *scales,
                             const void *zeros, unsigned *status, cudaStream_t st)
{
    PagesParams p;
    p.pool = page_pool_of(pool);
    p.slots = slots;
    p.n_groups = n_groups;
    p.status = status;
    p.first = 0;
    p.x[0] = codes;
    p.x[1] = scales;
    p.y[0] = const_cast<void *>(zeros);
    const dim3 grid((unsigned)n_groups, (unsigned)pool->n_kv_heads);
#define SQ_P(GG, BB) return pool->meta16 ? squat_launch(pages_place_kernel<GG, BB, true>, grid, 128, 0, st, p) : squat_launch(pages_place_kernel<GG, BB, false>, grid, 128, 0, st, p)
    if (pool->bits == 2) { if (pool->group_size == 32) SQ_P(32, 2); if (pool->group_size == 64) SQ_P(64, 2); SQ_P(128, 2); }
    if (pool->group_size == 32) SQ_P(32, 4);
    if (pool->group_size == 64) SQ_P(64, 4);
    SQ_P(128, 4);
#undef SQ_P
}
