// Products in the microscaled 4-bit format, rows read straight into registers.
//
//   y[m][n] = alpha[n] * sum_k a[m][k] w[n][k] + bias[n]
//
// A matrix instruction takes 16 rows by 128 inputs of either operand; lane l holds inputs 32 (l / 16) .. + 31 (one scale
// block, 16 bytes) of row l % 16, so that a wave reads 64 consecutive bytes of every row.  The sum runs in steps of 512
// inputs: four instructions and 16 scale bytes a row, of which a lane keeps four in one word, byte j for instruction j.
// Weights are the first operand, so a lane gets four consecutive outputs.
#include "mx4_product.h"

namespace mbu {

struct Mx4Frag {
    v4i c[4];
    uint32_t s;
};

// 512 inputs of one held row for the lane's group; zeros where the row has ended
__device__ __forceinline__ void load_held(Mx4Frag &f, const uint8_t *codes, const uint8_t *scales, long long row,
                                          int kp, int step, int g)
{
    const uint4 *p = reinterpret_cast<const uint4 *>(codes + row * (kp >> 1) + step * 256 + g * 16);
    const uint32_t *q = reinterpret_cast<const uint32_t *>(scales + row * (kp >> 5) + step * 16);
    v4i s = {0, 0, 0, 0};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        uint4 v = {0, 0, 0, 0};
        if (step * 512 + j * 128 < kp) {
            v = p[4 * j];
            s[j] = (int)q[j];
        }
        f.c[j] = (v4i){(int)v.x, (int)v.y, (int)v.z, (int)v.w};
    }
    f.s = mx4_scales_of(s, g);
}

// the same from a blob of masked-binary weights (every scale 2^0)
__device__ __forceinline__ void load_masked(Mx4Frag &f, const uint4 *blob, long long tile, int steps, int step, int lane)
{
    const uint4 *p = blob + (tile * steps + step) * 128 + lane;
    const uint4 a = p[0], b = p[64];
    f.c[0] = expand_masked(a.x, a.y);
    f.c[1] = expand_masked(a.z, a.w);
    f.c[2] = expand_masked(b.x, b.y);
    f.c[3] = expand_masked(b.z, b.w);
    f.s = 0x7f7f7f7fu;
}

// the same from a row of floats, quantised here: a lane owns whole blocks, so nothing crosses lanes
template <typename T>
__device__ __forceinline__ void load_float(Mx4Frag &f, const T *row, int K, int step, int g)
{
    constexpr int C = Mx4In<T>::CHUNK;
    f.s = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int k0 = step * 512 + j * 128 + g * 32;
        Mx4In<T> in[4];
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
#pragma unroll
            for (int c = 0; c < 8 / C; ++c) {
                const int k = k0 + 8 * i + c * C;
                uint4 v = {0, 0, 0, 0};
                if (k < K) v = *reinterpret_cast<const uint4 *>(row + k);
                in[i].set_chunk(c, v);
            }
            top = max(top, in[i].top());
        }
        const uint32_t s = mx4_scale_byte(top);
        const float scale = mx4_scale_float(s);
        f.c[j] = (v4i){(int)in[0].codes(scale), (int)in[1].codes(scale), (int)in[2].codes(scale),
                       (int)in[3].codes(scale)};
        f.s |= s << (8 * j);
    }
}

// Block: blockDim / 64 waves, which share the steps of MT x 16 rows by NT x 16 outputs and add their sums up in LDS in
// the waves' order.  XT: type of the activations (uint8_t: held).
template <typename XT, Mx4Weights WK, int MT, int NT, typename OT>
__global__ __launch_bounds__(1024) void mx4_direct_kernel(const Mx4Args p)
{
    extern __shared__ v4f part[];                          // [wave][MT * NT][64 lanes]
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
    const int r = lane & 15, g = lane >> 4;
    const int tm = blockIdx.x / p.tiles_n, tn = blockIdx.x - tm * p.tiles_n;
    const long long m0 = (long long)tm * (16 * MT), n0 = (long long)tn * (16 * NT);
    v4f acc[MT][NT];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) acc[i][j] = (v4f){0, 0, 0, 0};
    for (int step = wave; step < p.steps; step += waves) {
        Mx4Frag w[NT], x[MT];
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            if (WK == W_HELD)
                load_held(w[j], (const uint8_t *)p.w, p.ws, min(n0 + 16 * j + r, (long long)p.N - 1), p.kp, step, g);
            else
                load_masked(w[j], (const uint4 *)p.w, min(n0 / 16 + j, (long long)(p.N - 1) / 16), p.steps, step, lane);
        }
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            const long long m = min(m0 + 16 * i + r, (long long)p.M - 1);
            if constexpr (sizeof(XT) == 1) load_held(x[i], (const uint8_t *)p.x, p.xs, m, p.kp, step, g);
            else load_float(x[i], (const XT *)p.x + m * p.ldx, p.K, step, g);
        }
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                acc[i][j] = mx4_mfma<0>(w[j].c[0], w[j].s, x[i].c[0], x[i].s, acc[i][j]);
                acc[i][j] = mx4_mfma<1>(w[j].c[1], w[j].s, x[i].c[1], x[i].s, acc[i][j]);
                acc[i][j] = mx4_mfma<2>(w[j].c[2], w[j].s, x[i].c[2], x[i].s, acc[i][j]);
                acc[i][j] = mx4_mfma<3>(w[j].c[3], w[j].s, x[i].c[3], x[i].s, acc[i][j]);
            }
    }
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) part[(wave * (MT * NT) + i * NT + j) * 64 + lane] = acc[i][j];
    __syncthreads();
    for (int t = wave; t < MT * NT; t += waves) {
        v4f v = part[t * 64 + lane];
        for (int s = 1; s < waves; ++s) v += part[(s * (MT * NT) + t) * 64 + lane];
        const long long m = m0 + t / NT * 16 + r, n = n0 + t % NT * 16 + 4 * g;
        if (m >= p.M || n >= p.N) continue;
        const int left = (int)min(4ll, p.N - n);
#pragma unroll
        for (int q = 0; q < 4; ++q)
            if (q < left) {
                if (p.alpha) v[q] *= p.alpha[n + q];
                if (p.bias) v[q] += p.bias[n + q];
            }
        OT *dst = (OT *)p.out + m * p.N + n;
        if ((p.N & 3) == 0) mx4_store4(dst, v);
        else
#pragma unroll
            for (int q = 0; q < 4; ++q)
                if (q < left) mx4_store(dst + q, v[q]);
    }
}

template <typename XT, Mx4Weights WK, int MT, int NT, typename OT>
static int launch_direct(const char *fn, Mx4Args p, int waves, hipStream_t s)
{
    p.tiles_n = ceil_div(p.N, 16 * NT);
    const long long blocks = (long long)ceil_div(p.M, 16 * MT) * p.tiles_n;
    if (blocks > 0x7fffffffLL) return fail(MBU_ERR_SHAPE, "%s: product too large", fn);
    MBU_LAUNCH((mx4_direct_kernel<XT, WK, MT, NT, OT>), dim3((unsigned)blocks), dim3(64 * waves),
               (size_t)waves * MT * NT * 1024, s, p);
    return check_launch(fn);
}

template <typename XT, Mx4Weights WK, typename OT>
static int choose_shape(const char *fn, const Mx4Args &p, hipStream_t s)
{
    const int waves = min(8, p.steps);
    if (p.M <= 16) return launch_direct<XT, WK, 1, 1, OT>(fn, p, waves, s);
    return launch_direct<XT, WK, 4, 2, OT>(fn, p, min(4, waves), s);
}

template <typename XT, typename OT>
static int choose_weights(const char *fn, const Mx4Args &p, bool masked, hipStream_t s)
{
    return masked ? choose_shape<XT, W_MASKED, OT>(fn, p, s) : choose_shape<XT, W_HELD, OT>(fn, p, s);
}

int launch_mx4_matmul(const char *fn, const uint8_t *a, const uint8_t *as, int M, bool masked, const void *w,
                      const uint8_t *ws, int N, int K, const float *alpha, const float *bias, void *out, int dtype,
                      hipStream_t s)
{
    const int kp = mx4_padded(K);
    const Mx4Args p = {a, as, w, ws, alpha, bias, out, 0, M, N, K, kp, ceil_div(kp, 512), 0};
    if (M > 64) return launch_mx4_tile(fn, p, masked, dtype, s);
    if (dtype == MBU_FLOAT32) return choose_weights<uint8_t, float>(fn, p, masked, s);
    if (dtype == MBU_FLOAT16) return choose_weights<uint8_t, _Float16>(fn, p, masked, s);
    return choose_weights<uint8_t, __bf16>(fn, p, masked, s);
}

}  // namespace mbu
