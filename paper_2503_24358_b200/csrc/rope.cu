// Rotary position embedding with several axes (squat_rope_apply).
//
//   angle = positions[axis(i)][t] * theta_i,   (x_i, x_{i+n}) <- (x_i cos - x_{i+n} sin, x_{i+n} cos + x_i sin)
//
// The angle of pair i for one position is a 64-bit fraction of a turn; its product with the position modulo 2^64 is the angle's
// rest, exact to position * 2^-65 turns, so that the float32 sine and cosine of position one million are as good as
// those of position 1 (a float32 angle of a million radians has a sixteenth of a radian as its last digit).
//
// A thread owns eight pairs (16 bytes of bf16 from either half of a row) of one token and walks over heads: the sines and
// cosines of a token are made once per thread, for all its heads.  Bound: HBM (every element is read and written once).
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

template <bool BF16>
__device__ __forceinline__ void load8(const void *p, long long at, float (&x)[8])
{
    if (BF16) {
        const uint4 r = *reinterpret_cast<const uint4 *>(static_cast<const __nv_bfloat16 *>(p) + at);
        const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) { x[2 * i] = bf16lo_to_f32(w[i]); x[2 * i + 1] = bf16hi_to_f32(w[i]); }
    } else {
        const float4 *s = reinterpret_cast<const float4 *>(static_cast<const float *>(p) + at);
        const float4 a = s[0], b = s[1];
        x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
    }
}
template <bool BF16>
__device__ __forceinline__ void store8(void *p, long long at, const float (&x)[8])
{
    if (BF16) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const __nv_bfloat162 v = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
            w[i] = *reinterpret_cast<const uint32_t *>(&v);
        }
        *reinterpret_cast<uint4 *>(static_cast<__nv_bfloat16 *>(p) + at) = make_uint4(w[0], w[1], w[2], w[3]);
    } else {
        float4 *d = reinterpret_cast<float4 *>(static_cast<float *>(p) + at);
        d[0] = make_float4(x[0], x[1], x[2], x[3]);
        d[1] = make_float4(x[4], x[5], x[6], x[7]);
    }
}

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
    const int h0 = blockIdx.y * p.per_thread, h1 = min(h0 + p.per_thread, p.side[0].heads + p.side[1].heads);
    for (int h = h0; h < h1; ++h) {
        const bool key = h >= p.side[0].heads;
        const RopeSide &sd = p.side[key ? 1 : 0];
        const int hh = key ? h - p.side[0].heads : h;
        const long long x0 = t * sd.xt + hh * sd.xh, y0 = t * sd.yt + hh * sd.yh;
        float a[8], b[8];
        load8<BF16>(sd.x, x0 + lo, a);
        load8<BF16>(sd.x, x0 + hi, b);
        if (turns) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float u = fmaf(a[i], c[i], -b[i] * s[i]), v = fmaf(b[i], c[i], a[i] * s[i]);
                a[i] = u;
                b[i] = v;
            }
        }
        store8<BF16>(sd.y, y0 + lo, a);
        store8<BF16>(sd.y, y0 + hi, b);
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
    p.per_thread = 1;
    const long long runs = (total + p.per_thread - 1) / p.per_thread;
    if (blocks > 0x7fffffffLL || runs > 65535) return SQUAT_ERR_UNSUPPORTED;
    const dim3 grid((unsigned)blocks, (unsigned)runs);
    return dtype == SQUAT_BF16 ? squat_launch(rope_kernel<true>, grid, THREADS, 0, st, p) : squat_launch(rope_kernel<false>, grid, THREADS, 0, st, p);
}
