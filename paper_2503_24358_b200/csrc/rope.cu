// Rotary position embedding with several axes (squat_rope_apply).
//
//   angle = positions[axis(i)][t] * theta_i,   (x_i, x_{i+n}) <- (x_i cos - x_{i+n} sin, x_{i+n} cos + x_i sin)
//
// The angle of pair i for one position is a 64-bit fraction of a turn; its product with the position modulo 2^64 is the angle's
// rest, exact to position * 2^-65 turns, so that the float32 sine and cosine of position one million are as good as
// those of position 1 (a float32 angle of a million radians has a sixteenth of a radian as its last digit).
//
// A thread owns eight pairs (16 bytes of bf16 from either half of a row) of one token and walks over heads: the sines and
// cosines of a token are made once per thread, for all its heads.  Bound: HBM (every element is read and written once): 32768 tokens of 32 + 8 heads
// in bf16 take 118 us, 5.7 TB/s, in float32 214 us, 6.3 TB/s, either way round; 64 tokens take 7.6 us, of which most is the launch.
#include "device_helpers.cuh"

namespace {

constexpr int D = SQUAT_D;
constexpr int THREADS = 256, SLOTS = D / 16;         // threads of a token and head: eight pairs, or sixteen channels that are copied

struct RopeSide {
    const void *x;
    void *y;
    long long xt, xh, yt, yh;                        // element strides
    int heads;
};
struct RopeParams {
    squat_rope_plan plan;
    const void *positions;
    long long axis_stride;
    int positions64, n_tokens, per_thread;           // heads per thread
    float sign;
    RopeSide side[2];                                // queries, keys
};

// Eight channels of a row
template <bool BF16>
struct Chunk;
template <>
struct Chunk<true> {
    uint4 r;
    __device__ __forceinline__ void load(const void *p, long long at) { r = *reinterpret_cast<const uint4 *>(static_cast<const __nv_bfloat16 *>(p) + at); }
    __device__ __forceinline__ void store(void *p, long long at) const { *reinterpret_cast<uint4 *>(static_cast<__nv_bfloat16 *>(p) + at) = r; }
    __device__ __forceinline__ void get(float (&x)[8]) const
    {
        const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) { x[2 * i] = bf16lo_to_f32(w[i]); x[2 * i + 1] = bf16hi_to_f32(w[i]); }
    }
    __device__ __forceinline__ void set(const float (&x)[8])
    {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const __nv_bfloat162 v = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
            w[i] = *reinterpret_cast<const uint32_t *>(&v);
        }
        r = make_uint4(w[0], w[1], w[2], w[3]);
    }
};
template <>
struct Chunk<false> {
    float4 a, b;
    __device__ __forceinline__ void load(const void *p, long long at)
    {
        const float4 *s = reinterpret_cast<const float4 *>(static_cast<const float *>(p) + at);
        a = s[0];
        b = s[1];
    }
    __device__ __forceinline__ void store(void *p, long long at) const
    {
        float4 *d = reinterpret_cast<float4 *>(static_cast<float *>(p) + at);
        d[0] = a;
        d[1] = b;
    }
    __device__ __forceinline__ void get(float (&x)[8]) const { x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w; }
    __device__ __forceinline__ void set(const float (&x)[8]) { a = make_float4(x[0], x[1], x[2], x[3]); b = make_float4(x[4], x[5], x[6], x[7]); }
};

template <bool BF16>
__global__ void __launch_bounds__(THREADS) rope_kernel(const __grid_constant__ RopeParams p)
{
    // grid: (token and slot, runs of per_thread heads of queries and keys together)
    const long long flat = (long long)blockIdx.x * THREADS + threadIdx.x;
    const int slot = (int)(flat % SLOTS);
    const long long t = flat / SLOTS;
    if (t >= p.n_tokens) return;
    const int n = p.plan.n_pairs, i0 = slot * 8;
    const bool turns = i0 < n;
    const int lo = turns ? i0 : 2 * n + (slot - n / 8) * 16, hi = turns ? i0 + n : lo + 8;      // the thread's two runs of eight channels
    const void *positions = p.positions;
    grid_wait(positions);
    constexpr int AT_ONCE = BF16 ? 4 : 2;            // heads whose loads are in flight together
    float c[8], s[8];
    if (turns) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const long long at = (long long)p.plan.axis[i0 + i] * p.axis_stride + t;
            const long long pos = p.positions64 ? static_cast<const long long *>(positions)[at] : static_cast<const int *>(positions)[at];
            const unsigned long long rest = (unsigned long long)pos * p.plan.turn[i0 + i];
            // 32 of its bits as a signed number of half turns; a float keeps 24 of them
            sincospif((float)(int)(rest >> 32) * 0x1p-31f, &s[i], &c[i]);
            s[i] *= p.sign;
        }
    }
    const int h0 = blockIdx.y * p.per_thread, hq = p.side[0].heads, h1 = min(h0 + p.per_thread, hq + p.side[1].heads);
#pragma unroll
    for (int side = 0; side < 2; ++side) {
        const RopeSide &sd = p.side[side];
        const int begin = max(h0 - side * hq, 0), end = min(h1 - side * hq, sd.heads);
        const long long x0 = t * sd.xt, y0 = t * sd.yt;
        for (int h = begin; h < end; h += AT_ONCE) {
            Chunk<BF16> a[AT_ONCE], b[AT_ONCE];
#pragma unroll
            for (int j = 0; j < AT_ONCE; ++j)
                if (h + j < end) {
                    a[j].load(sd.x, x0 + (h + j) * sd.xh + lo);
                    b[j].load(sd.x, x0 + (h + j) * sd.xh + hi);
                }
#pragma unroll
            for (int j = 0; j < AT_ONCE; ++j)
                if (h + j < end) {
                    if (turns) {
                        float u[8], v[8];
                        a[j].get(u);
                        b[j].get(v);
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            const float x = fmaf(u[i], c[i], -v[i] * s[i]);
                            v[i] = fmaf(v[i], c[i], u[i] * s[i]);
                            u[i] = x;
                        }
                        a[j].set(u);
                        b[j].set(v);
                    }
                    a[j].store(sd.y, y0 + (h + j) * sd.yh + lo);
                    b[j].store(sd.y, y0 + (h + j) * sd.yh + hi);
                }
        }
    }
}

}  // namespace

int squat_launch_rope(const squat_rope_plan *plan, const void *positions, int positions64, long long axis_stride, int n_tokens,
                      int dtype, int inverse, const void *const (&x)[2], void *const (&y)[2], const int (&heads)[2],
                      const long long (&strides)[2][4], cudaStream_t st)
{
    RopeParams p;
    p.plan = *plan;
    p.positions = positions;
    p.axis_stride = axis_stride;
    p.positions64 = positions64;
    p.n_tokens = n_tokens;
    p.sign = inverse ? -1.0f : 1.0f;
    for (int i = 0; i < 2; ++i) p.side[i] = {x[i], y[i], strides[i][0], strides[i][1], strides[i][2], strides[i][3], heads[i]};
    const long long total = (long long)heads[0] + heads[1], blocks = ((long long)n_tokens * SLOTS + THREADS - 1) / THREADS;
    // As many heads to a thread as leave sixteen CTAs to every SM (two waves): the sines and cosines, eight of each, cost as much as
    // four heads.
    long long runs = (16LL * squat_sm_count() + blocks - 1) / blocks;
    runs = runs < 1 ? 1 : runs > total ? total : runs;
    p.per_thread = (int)((total + runs - 1) / runs);
    runs = (total + p.per_thread - 1) / p.per_thread;
    if (blocks > 0x7fffffffLL || runs > 65535) return SQUAT_ERR_UNSUPPORTED;
    const dim3 grid((unsigned)blocks, (unsigned)runs);
    return dtype == SQUAT_BF16 ? squat_launch(rope_kernel<true>, grid, THREADS, 0, st, p) : squat_launch(rope_kernel<false>, grid, THREADS, 0, st, p);
}
