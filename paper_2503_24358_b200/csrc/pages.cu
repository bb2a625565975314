// Groups of keys and values quantized into the pages of a paged cache, and read back (squat_pages_write, squat_pages_read).
//
//   Delta = (M - m) RN(1 / L),   c = clamp(rint((x - z) / Delta), 0, L),   x' = z + Delta c     (z = m; or both rounded to binary16)
//
// Delta is a product of binary32 numbers: its last bit may differ from the rounded quotient that the quantizers of contiguous
// caches store.  Codes are decided by the stored grid, so this is no error of theirs.
// over G tokens per channel (keys) or G channels per token (values).  A CTA takes one group of tokens of one head: G tokens
// are G rows of 256 or 512 contiguous bytes, and 16 threads hold a row, eight channels each, four rows to a thread.  So both
// reductions are short: keys over the rows (a thread's four, the two halves of a warp, the warps), values over neighbouring lanes.
//
// Decisions.  t is bracketed by (x - z) r (1 +- 2^-20), r the hardware reciprocal of Delta (1 ulp); adding 1.5 * 2^23 rounds both
// ends to integers, ties to even, and where they agree that integer is the code.  Where they do not (structural with bf16
// data), values take the IEEE binary32 sequence that defines them, keys the sign of (x - z) - (k + 1/2) Delta in float64: what
// real arithmetic on the stored grid decides.
//
// Bound: HBM (x is read once, codes and metadata are written once; a group's codes are one contiguous span of its page).
#include "pages.cuh"

namespace {

constexpr int D = SQUAT_D;
constexpr float kMagic = 12582912.0f;   // 1.5 * 2^23
constexpr int ROWS = 4;                 // rows of a group per thread

struct PagesParams {
    PagePool pool;
    const int *slots;
    int first;                          // 0: keys and (blockIdx.z = 1) values, 1: values only
    const void *x[2];                   // keys, values
    long long xt[2], xh[2];
    void *y[2];                         // rows that are read back
    unsigned *status;
};

// A group's grid as it is stored, and what decides by it.
struct Grid {
    float zero, delta, ra, rb;
    bool ok, fast;
};
template <int BITS, bool M16>
__device__ __forceinline__ Grid grid_of(float m, float Mx)
{
    Grid g;
    constexpr float invL = 1.0f / float((1 << BITS) - 1);
    g.delta = __fmul_rn(__fsub_rn(Mx, m), invL);
    g.zero = m;
    if (M16) {
        g.delta = __half2float(__float2half_rn(g.delta));
        g.zero = __half2float(__float2half_rn(m));
    }
    return g;
}
__device__ __forceinline__ void decide_by(Grid &g)
{
    g.ok = g.delta > 0.0f && g.delta < __int_as_float(0x7f800000);
    g.fast = g.delta > 0x1p-100f && g.delta < 0x1p100f;
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(g.delta));
    g.ra = __fmul_rn(r, 1.0f + 0x1p-20f);
    g.rb = __fmul_rn(r, 1.0f - 0x1p-20f);
}

// The code where the bracket leaves it open.
template <int BITS, bool KEY>
__device__ __noinline__ unsigned exact_code(float x, float zero, float delta)
{
    constexpr float L = float((1 << BITS) - 1);
    if (!KEY) return (unsigned)(int)fminf(fmaxf(rintf(__fdiv_rn(__fsub_rn(x, zero), delta)), 0.0f), L);
    const double dl = (double)x - (double)zero;
    return (unsigned)(int)fmin(fmax(rint(__ddiv_rn(dl, (double)delta)), 0.0), (double)L);
}

// Eight codes, packed low bits first.
template <int BITS, bool KEY, bool M16>
__device__ __forceinline__ unsigned codes_of(const float (&x)[8], const Grid *g, int g_step)
{
    constexpr float L = float((1 << BITS) - 1);
    unsigned word = 0, open = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const Grid &gr = g[i * g_step];
        const float dl = __fsub_rn(x[i], gr.zero);
        float ya = __fmaf_rn(dl, gr.ra, kMagic), yb = __fmaf_rn(dl, gr.rb, kMagic);
        if (M16) {                                  // a rounded zero-point may lie above the minimum
            ya = fminf(fmaxf(ya, kMagic), kMagic + L);
            yb = fminf(fmaxf(yb, kMagic), kMagic + L);
        }
        if (!gr.fast || ya != yb) open |= 1u << i;
        word |= gr.ok ? (__float_as_uint(ya) & ((1u << BITS) - 1u)) << (BITS * i) : 0u;
    }
    if (open) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const Grid &gr = g[i * g_step];
            if (!(open >> i & 1) || !gr.ok) continue;
            word = (word & ~(((1u << BITS) - 1u) << (BITS * i))) | exact_code<BITS, KEY>(x[i], gr.zero, gr.delta) << (BITS * i);
        }
    }
    return word;
}

template <bool BF16>
__device__ __forceinline__ void load_row(const void *p, long long at, float (&x)[8])
{
    if (BF16) {
        const uint4 r = ldg128(static_cast<const __nv_bfloat16 *>(p) + at);
        const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) { x[2 * i] = bf16lo_to_f32(w[i]); x[2 * i + 1] = bf16hi_to_f32(w[i]); }
    } else {
        const float4 *s = reinterpret_cast<const float4 *>(static_cast<const float *>(p) + at);
        const float4 a = __ldg(s), b = __ldg(s + 1);
        x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
    }
}

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

// The group's first token in the pool, or -1: padding or (flagged) a slot that is none.
template <int G>
__device__ __forceinline__ long long group_token(const PagesParams &p, const int *slots, int h)
{
    const int slot = __ldg(slots + blockIdx.x);
    if (slot < 0) return -1;
    if (slot % G != 0 || slot / p.pool.page_tokens >= p.pool.n_pages) {
        if (threadIdx.x == 0) atomicOr(p.status, SQUAT_FLAG_PAGES);
        return -1;
    }
    return token_at_slot(p.pool, slot, h);
}

// grid (groups, heads, keys / values); 4 G threads: thread t holds channels 8 (t mod 16) .. + 7 of rows t / 16 + (G / 4) i
template <int G, int BITS, bool BF16, bool M16>
__global__ void __launch_bounds__(4 * G) pages_write_kernel(PagesParams p)
{
    constexpr int WARPS = G / 8, STEP = G / ROWS;
    __shared__ __align__(16) float lo_sm[WARPS][D], hi_sm[WARPS][D];
    const int part = p.first + blockIdx.z, h = blockIdx.y, tid = threadIdx.x, c8 = tid & 15, r0 = tid >> 4;
    const void *src = p.x[part];
    const int *slots = p.slots;
    grid_wait(src, slots);
    const long long tok = group_token<G>(p, slots, h);
    if (tok < 0) return;
    float x[ROWS][8];
#pragma unroll
    for (int i = 0; i < ROWS; ++i)
        load_row<BF16>(src, ((long long)blockIdx.x * G + r0 + STEP * i) * p.xt[part] + (long long)h * p.xh[part] + 8 * c8, x[i]);
    unsigned char *codes = (part == 0 ? p.pool.kc : p.pool.vc) + (tok + r0) * (D * BITS / 8) + c8 * BITS;
    unsigned words[ROWS], flags = 0;
    if (part == 0) {
#pragma unroll
        for (int c = 0; c < 8; ++c) {
            float m = min_nan(min_nan(x[0][c], x[1][c]), min_nan(x[2][c], x[3][c])), Mx = max_nan(max_nan(x[0][c], x[1][c]), max_nan(x[2][c], x[3][c]));
            m = min_nan(m, __shfl_xor_sync(0xffffffffu, m, 16));
            Mx = max_nan(Mx, __shfl_xor_sync(0xffffffffu, Mx, 16));
            if ((tid & 16) == 0) {
                lo_sm[tid >> 5][8 * c8 + c] = m;
                hi_sm[tid >> 5][8 * c8 + c] = Mx;
            }
        }
        __syncthreads();
        if (tid < D) {                                   // a channel's grid
            float m = lo_sm[0][tid], Mx = hi_sm[0][tid];
#pragma unroll
            for (int w = 1; w < WARPS; ++w) {
                m = min_nan(m, lo_sm[w][tid]);
                Mx = max_nan(Mx, hi_sm[w][tid]);
            }
            const Grid g = grid_of<BITS, M16>(m, Mx);
            lo_sm[0][tid] = g.zero;
            hi_sm[0][tid] = g.delta;
            const long long at = tok / G * D + tid;
            store_meta<M16>(p.pool.ks, at, g.delta);
            store_meta<M16>(p.pool.kz, at, g.zero);
            if (!(g.delta > 0.0f && g.delta < __int_as_float(0x7f800000))) flags = g.delta == 0.0f ? SQUAT_FLAG_ZERO_RANGE : SQUAT_FLAG_NONFINITE;
        }
        __syncthreads();
        Grid g[8];
#pragma unroll
        for (int c = 0; c < 8; ++c) {
            g[c].zero = lo_sm[0][8 * c8 + c];
            g[c].delta = hi_sm[0][8 * c8 + c];
            decide_by(g[c]);
        }
#pragma unroll
        for (int i = 0; i < ROWS; ++i) words[i] = codes_of<BITS, true, M16>(x[i], g, 1);
    } else {
        constexpr int LANES = G / 8;                     // of a group
#pragma unroll
        for (int i = 0; i < ROWS; ++i) {
            float m = x[i][0], Mx = x[i][0];
#pragma unroll
            for (int c = 1; c < 8; ++c) { m = min_nan(m, x[i][c]); Mx = max_nan(Mx, x[i][c]); }
#pragma unroll
            for (int o = 1; o < LANES; o <<= 1) {
                m = min_nan(m, __shfl_xor_sync(0xffffffffu, m, o));
                Mx = max_nan(Mx, __shfl_xor_sync(0xffffffffu, Mx, o));
            }
            Grid g = grid_of<BITS, M16>(m, Mx);
            decide_by(g);
            words[i] = codes_of<BITS, false, M16>(x[i], &g, 0);
            if (c8 % LANES == 0) {
                const long long at = (tok + r0 + STEP * i) * (D / G) + c8 / LANES;
                store_meta<M16>(p.pool.vs, at, g.delta);
                store_meta<M16>(p.pool.vz, at, g.zero);
                if (!g.ok) flags |= g.delta == 0.0f ? SQUAT_FLAG_ZERO_RANGE : SQUAT_FLAG_NONFINITE;
            }
        }
    }
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        unsigned char *to = codes + STEP * i * (D * BITS / 8);
        if (BITS == 2) *reinterpret_cast<unsigned short *>(to) = (unsigned short)words[i];
        else *reinterpret_cast<unsigned *>(to) = words[i];
    }
    if (flags) atomicOr(p.status, flags);
}

// Keys that squat_quantize_keys has left in the workspace, [heads, tokens]: codes x[0], metadata x[1] (scales, then zero-points
// y[0]); a group's codes are one span on either side.
template <int G, int BITS, bool M16>
__global__ void __launch_bounds__(128) pages_place_kernel(PagesParams p, int n_groups)
{
    const int h = blockIdx.y, tid = threadIdx.x;
    const unsigned char *codes = static_cast<const unsigned char *>(p.x[0]);
    const void *scales = p.x[1], *zeros = p.y[0];
    const int *slots = p.slots;
    grid_wait(codes, scales, zeros, slots);
    const long long tok = group_token<G>(p, slots, h);
    if (tok < 0) return;
    const long long from = (long long)h * n_groups + blockIdx.x;
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

// grid (groups, heads, keys / values); threads as for the write
template <int G, int BITS, bool BF16, bool M16>
__global__ void __launch_bounds__(4 * G) pages_read_kernel(PagesParams p)
{
    constexpr int STEP = G / ROWS;
    const int part = p.first + blockIdx.z, h = blockIdx.y, tid = threadIdx.x, c8 = tid & 15, r0 = tid >> 4;
    const unsigned char *codes = part == 0 ? p.pool.kc : p.pool.vc;
    const void *scales = part == 0 ? p.pool.ks : p.pool.vs, *zeros = part == 0 ? p.pool.kz : p.pool.vz;
    const int *slots = p.slots;
    grid_wait(codes, scales, zeros, slots);
    const long long tok = group_token<G>(p, slots, h);
    if (tok < 0) return;
    unsigned words[ROWS];
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        const unsigned char *from = codes + (tok + r0 + STEP * i) * (D * BITS / 8) + c8 * BITS;
        words[i] = BITS == 2 ? (unsigned)__ldg(reinterpret_cast<const unsigned short *>(from)) : __ldg(reinterpret_cast<const unsigned *>(from));
    }
    float s[8], z[8];
    if (part == 0) {
#pragma unroll
        for (int c = 0; c < 8; ++c) {
            s[c] = load_meta<M16>(scales, tok / G * D + 8 * c8 + c);
            z[c] = load_meta<M16>(zeros, tok / G * D + 8 * c8 + c);
        }
    }
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        if (part == 1) {
            const long long at = (tok + r0 + STEP * i) * (D / G) + c8 / (G / 8);
            s[0] = load_meta<M16>(scales, at);
            z[0] = load_meta<M16>(zeros, at);
        }
        float y[8];
#pragma unroll
        for (int c = 0; c < 8; ++c)
            y[c] = __fmaf_rn((float)(words[i] >> (BITS * c) & ((1u << BITS) - 1u)), part == 0 ? s[c] : s[0], part == 0 ? z[c] : z[0]);
        const long long at = ((long long)blockIdx.x * G + r0 + STEP * i) * p.xt[part] + (long long)h * p.xh[part] + 8 * c8;
        if (BF16) {
            uint32_t w[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const __nv_bfloat162 v = __floats2bfloat162_rn(y[2 * k], y[2 * k + 1]);
                w[k] = *reinterpret_cast<const uint32_t *>(&v);
            }
            *reinterpret_cast<uint4 *>(static_cast<__nv_bfloat16 *>(p.y[part]) + at) = make_uint4(w[0], w[1], w[2], w[3]);
        } else {
            float4 *to = reinterpret_cast<float4 *>(static_cast<float *>(p.y[part]) + at);
            to[0] = make_float4(y[0], y[1], y[2], y[3]);
            to[1] = make_float4(y[4], y[5], y[6], y[7]);
        }
    }
}

template <int G, int BITS>
int launch_inst(const PagesParams &p, bool write, dim3 grid, int dtype, int meta16, cudaStream_t st)
{
#define SQ_P(K, BF, MM) return squat_launch(K<G, BITS, BF, MM>, grid, 4 * G, 0, st, p)
    const bool bf = dtype == SQUAT_BF16;
    if (write) {
        if (bf) { if (meta16) SQ_P(pages_write_kernel, true, true); else SQ_P(pages_write_kernel, true, false); }
        else { if (meta16) SQ_P(pages_write_kernel, false, true); else SQ_P(pages_write_kernel, false, false); }
    } else {
        if (bf) { if (meta16) SQ_P(pages_read_kernel, true, true); else SQ_P(pages_read_kernel, true, false); }
        else { if (meta16) SQ_P(pages_read_kernel, false, true); else SQ_P(pages_read_kernel, false, false); }
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
    return launch_sized(p, write, dim3((unsigned)n_groups, (unsigned)pool->n_kv_heads, (unsigned)parts), pool, dtype, st);
}

int squat_launch_pages_place(const squat_page_pool *pool, const int *slots, int n_groups, const void *codes, const void *scales,
                             const void *zeros, unsigned *status, cudaStream_t st)
{
    PagesParams p;
    p.pool = page_pool_of(pool);
    p.slots = slots;
    p.status = status;
    p.first = 0;
    p.x[0] = codes;
    p.x[1] = scales;
    p.y[0] = const_cast<void *>(zeros);
    const dim3 grid((unsigned)n_groups, (unsigned)pool->n_kv_heads);
#define SQ_P(GG, BB) return pool->meta16 ? squat_launch(pages_place_kernel<GG, BB, true>, grid, 128, 0, st, p, n_groups) : squat_launch(pages_place_kernel<GG, BB, false>, grid, 128, 0, st, p, n_groups)
    if (pool->bits == 2) { if (pool->group_size == 32) SQ_P(32, 2); if (pool->group_size == 64) SQ_P(64, 2); SQ_P(128, 2); }
    if (pool->group_size == 32) SQ_P(32, 4);
    if (pool->group_size == 64) SQ_P(64, 4);
    SQ_P(128, 4);
#undef SQ_P
}
