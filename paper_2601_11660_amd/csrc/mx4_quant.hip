// Microscaled 4-bit format: quantisation, dequantisation, packing of masked-binary weights.
#include "mx4_common.h"

namespace mbu {

// Rows with consecutive values.  Eight values a thread, so four threads share a block's scale (two lane exchanges
// inside a quad); `tpr` threads (a power of two) walk along a row, UNROLL groups of eight each with all loads in flight.
// Rows are read 16 bytes at a time wherever they start; WHOLE: K is a multiple of eight.
constexpr int QUANT_UNROLL = 4;

template <int TYPE, bool WHOLE>
__global__ __launch_bounds__(256) void mx4_quantize_kernel(const void *__restrict__ values, long long stride, int rows, int K,
                                                           int kp, int tpr_log, int segs, uint8_t *__restrict__ codes,
                                                           uint8_t *__restrict__ scales)
{
    const int tpr = 1 << tpr_log;
    const int group = blockIdx.x / segs, seg = blockIdx.x - group * segs;
    const long long row = (long long)group * (256 >> tpr_log) + (threadIdx.x >> tpr_log);
    if (row >= rows) return;                       // whole quads: tpr is a multiple of 16
    const int first = seg * tpr * QUANT_UNROLL + (threadIdx.x & (tpr - 1));
    using T = typename Mx4Type<TYPE>::T;
    const T *src = (const T *)values + row * stride;
    Mx4In<T> in[QUANT_UNROLL];
#pragma unroll
    for (int u = 0; u < QUANT_UNROLL; ++u) {
        const int k = (first + u * tpr) * 8;
        in[u] = zero_eight<T>();
        if (k + 8 <= K) in[u] = load_eight(src + k);
        else if (!WHOLE && k < K) in[u] = load_some(src + k, K - k);
    }
#pragma unroll
    for (int u = 0; u < QUANT_UNROLL; ++u) {
        const int k = (first + u * tpr) * 8;
        uint32_t top = in[u].top();
        top = max(top, (uint32_t)__builtin_amdgcn_mov_dpp((int)top, 0xb1, 0xf, 0xf, true));    // lanes 1 0 3 2
        top = max(top, (uint32_t)__builtin_amdgcn_mov_dpp((int)top, 0x4e, 0xf, 0xf, true));    // lanes 2 3 0 1
        const uint32_t s = mx4_scale_byte(top);
        const uint32_t q = s == 255u ? 0u : in[u].codes(mx4_scale_float(s));
        if (k < kp) {
            *reinterpret_cast<uint32_t *>(codes + row * (kp >> 1) + (k >> 1)) = q;
            if ((threadIdx.x & 3) == 0) scales[row * (kp >> 5) + (k >> 5)] = (uint8_t)s;
        }
    }
}

// Rows whose values lie `stride` apart, neighbouring rows next to each other: a lane takes one block of its row, 64
// consecutive rows per wave.
template <int TYPE>
__global__ __launch_bounds__(256) void mx4_quantize_across_kernel(const void *__restrict__ values, long long stride, int rows,
                                                                  int K, int kp, int kgroups,
                                                                  uint8_t *__restrict__ codes,
                                                                  uint8_t *__restrict__ scales)
{
    const int tile = blockIdx.x / kgroups, kg = blockIdx.x - tile * kgroups;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const long long row = (long long)tile * 64 + lane;
    if (row >= rows) return;
    const int k0 = kg * 128 + wave * 32;
    using T = typename Mx4Type<TYPE>::T;
    const T *const x = (const T *)values;
    Mx4In<T> in[4];
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int k = k0 + 8 * j + i;
            in[j].set(i, k < K ? x[k * stride + row] : (T)0.0f);
        }
    uint32_t top = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) top = max(top, in[j].top());
    const uint32_t s = mx4_scale_byte(top);
    uint32_t q[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) q[j] = s == 255u ? 0u : in[j].codes(mx4_scale_float(s));
    *reinterpret_cast<uint4 *>(codes + row * (kp >> 1) + (k0 >> 1)) = make_uint4(q[0], q[1], q[2], q[3]);
    scales[row * (kp >> 5) + (k0 >> 5)] = (uint8_t)s;
}

// number of codes [8 i, 8 i + 8) -> values; every product of a code and a scale is exact in float32
__device__ __forceinline__ void mx4_values(uint32_t q, uint32_t s, float v[8])
{
    const float scale = mx4_scale_float(s);
    v2f p[4] = {__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, scale, 0), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, scale, 1),
                __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, scale, 2), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, scale, 3)};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = s == 255u ? __uint_as_float(0x7fc00000u) : p[i].x;
        v[2 * i + 1] = s == 255u ? __uint_as_float(0x7fc00000u) : p[i].y;
    }
}

template <int TYPE, bool VEC>
__global__ __launch_bounds__(256) void mx4_dequantize_kernel(const uint8_t *__restrict__ codes,
                                                             const uint8_t *__restrict__ scales, int rows, int K, int kp,
                                                             int tpr_log, int segs, void *__restrict__ out)
{
    const int tpr = 1 << tpr_log;
    const int group = blockIdx.x / segs, seg = blockIdx.x - group * segs;
    const long long row = (long long)group * (256 >> tpr_log) + (threadIdx.x >> tpr_log);
    if (row >= rows) return;
    const int first = seg * tpr * QUANT_UNROLL + (threadIdx.x & (tpr - 1));
#pragma unroll
    for (int u = 0; u < QUANT_UNROLL; ++u) {
        const int k = (first + u * tpr) * 8;
        if (k >= K) break;
        const uint32_t q = *reinterpret_cast<const uint32_t *>(codes + row * (kp >> 1) + (k >> 1));
        const uint32_t s = scales[row * (kp >> 5) + (k >> 5)];
        float v[8];
        mx4_values(q, s, v);
        using T = typename Mx4Type<TYPE>::T;
        T *dst = (T *)out + row * K + k;
        if (VEC) {
            mx4_store4(dst, (v4f){v[0], v[1], v[2], v[3]});
            mx4_store4(dst + 4, (v4f){v[4], v[5], v[6], v[7]});
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (k + i < K) mx4_store(dst + i, v[i]);
        }
    }
}

// One thread: 64 weights of one output, as the lane that multiplies them reads them (layout: Mx4MaskedLayout).
__global__ __launch_bounds__(256) void mx4_pack_masked_kernel(const int8_t *__restrict__ w, int N, int K,
                                                              int steps, long long units, uint4 *__restrict__ dst)
{
    const long long u = (long long)blockIdx.x * 256 + threadIdx.x;
    if (u >= units) return;
    const int lane = (int)(u & 63), half = (int)(u >> 6) & 1;
    const long long t = u >> 7;                     // 16 outputs x 512 inputs
    const int step = (int)(t % steps);
    const long long n = t / steps * 16 + (lane & 15);
    const long long k0 = (long long)step * 512 + half * 256 + (lane >> 4) * 32;
    uint32_t word[4] = {0, 0, 0, 0};
    if (n < N) {
        const int8_t *src = w + n * K;
#pragma unroll
        for (int i = 0; i < 64; ++i) {
            const long long k = k0 + (i & 31) + (i >> 5) * 128;
            const int v = k < K ? src[k] : 0;
            const uint32_t b = (v != 0 ? 2u : 0u) | (v < 0 ? 8u : 0u);
            word[i >> 4] |= ((i & 8) ? b >> 1 : b) << (4 * (i & 7));
        }
    }
    dst[u] = make_uint4(word[0], word[1], word[2], word[3]);
}

static int quant_geometry(int rows, int per_row, int *tpr_log, int *segs, long long *blocks)
{
    int lg = 4;
    while (lg < 8 && (1 << lg) < per_row) ++lg;
    *tpr_log = lg;
    *segs = ceil_div(per_row, (1 << lg) * QUANT_UNROLL);
    *blocks = ((long long)rows + (256 >> lg) - 1) / (256 >> lg) * *segs;
    return *blocks <= 0x7fffffffLL ? MBU_OK : fail(MBU_ERR_SHAPE, "mbu_mx4: tensor too large");
}

template <int TYPE>
static int quantize(const void *x, int rows, int K, long long stride, bool across, uint8_t *codes, uint8_t *scales,
                    hipStream_t s)
{
    const int kp = mx4_padded(K);
    if (across) {
        const int kg = kp / 128;
        const long long blocks = ((long long)rows + 63) / 64 * kg;
        if (blocks > 0x7fffffffLL) return fail(MBU_ERR_SHAPE, "mbu_mx4_quantize: tensor too large");
        MBU_LAUNCH((mx4_quantize_across_kernel<TYPE>), dim3((unsigned)blocks), dim3(256), 0, s, x, stride, rows, K, kp, kg,
                   codes, scales);
        return check_launch("mbu_mx4_quantize");
    }
    int lg, segs;
    long long blocks;
    const int rc = quant_geometry(rows, kp / 8, &lg, &segs, &blocks);
    if (rc) return rc;
    const dim3 grid((unsigned)blocks), block(256);
    if (K % 8 == 0)
        MBU_LAUNCH((mx4_quantize_kernel<TYPE, true>), grid, block, 0, s, x, stride, rows, K, kp, lg, segs, codes, scales);
    else
        MBU_LAUNCH((mx4_quantize_kernel<TYPE, false>), grid, block, 0, s, x, stride, rows, K, kp, lg, segs, codes, scales);
    return check_launch("mbu_mx4_quantize");
}

int launch_mx4_quantize(const void *x, int dtype, int rows, int K, long long stride, bool across, uint8_t *codes,
                        uint8_t *scales, hipStream_t s)
{
    if (dtype == MBU_FLOAT32) return quantize<MBU_FLOAT32>(x, rows, K, stride, across, codes, scales, s);
    if (dtype == MBU_FLOAT16) return quantize<MBU_FLOAT16>(x, rows, K, stride, across, codes, scales, s);
    return quantize<MBU_BFLOAT16>(x, rows, K, stride, across, codes, scales, s);
}

template <int TYPE>
static int dequantize(const uint8_t *codes, const uint8_t *scales, int rows, int K, void *out, hipStream_t s)
{
    const int kp = mx4_padded(K);
    int lg, segs;
    long long blocks;
    const int rc = quant_geometry(rows, ceil_div(K, 8), &lg, &segs, &blocks);
    if (rc) return rc;
    const dim3 grid((unsigned)blocks), block(256);
    if (K % 8 == 0)
        MBU_LAUNCH((mx4_dequantize_kernel<TYPE, true>), grid, block, 0, s, codes, scales, rows, K, kp, lg, segs, out);
    else
        MBU_LAUNCH((mx4_dequantize_kernel<TYPE, false>), grid, block, 0, s, codes, scales, rows, K, kp, lg, segs, out);
    return check_launch("mbu_mx4_dequantize");
}

int launch_mx4_dequantize(const uint8_t *codes, const uint8_t *scales, int rows, int K, void *out, int dtype,
                          hipStream_t s)
{
    if (dtype == MBU_FLOAT32) return dequantize<MBU_FLOAT32>(codes, scales, rows, K, out, s);
    if (dtype == MBU_FLOAT16) return dequantize<MBU_FLOAT16>(codes, scales, rows, K, out, s);
    return dequantize<MBU_BFLOAT16>(codes, scales, rows, K, out, s);
}

int launch_mx4_pack_masked(const int8_t *w, int N, int K, void *packed, hipStream_t s)
{
    const Mx4MaskedLayout L = mx4_masked_layout(N, K);
    const long long units = (long long)L.tiles * L.steps * 128, blocks = (units + 255) / 256;
    if (blocks > 0x7fffffffLL) return fail(MBU_ERR_SHAPE, "mbu_mx4_pack_masked_binary: tensor too large");
    MBU_LAUNCH((mx4_pack_masked_kernel), dim3((unsigned)blocks), dim3(256), 0, s, w, N, K, L.steps, units,
               (uint4 *)packed);
    return check_launch("mbu_mx4_pack_masked_binary");
}

}  // namespace mbu
