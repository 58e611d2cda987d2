// Products in the microscaled 4-bit format for few rows (tokens): bound by reading the weights, each of which is read once.
//
// A block's waves share the steps of 512 inputs and take the same 16 outputs, so that even one token on a small layer
// keeps every compute unit busy; they add their sums up in LDS, in the waves' order, and go on to the next 16 outputs
// while the weights of those are on their way already.  The rows stay in registers as fragments, quantised there where
// they come as floats: a lane owns whole blocks of 32, so nothing crosses lanes.
#include "mx4_product.h"

namespace mbu {

constexpr int FEW_WAVES = 16;

struct Mx4Frag {
    v4i c[4];
    uint32_t s;
};

// 512 inputs of one held row for the lane's group; zeros where the row has ended
__device__ __forceinline__ void load_held(Mx4Frag &f, __amdgpu_buffer_rsrc_t codes, __amdgpu_buffer_rsrc_t scales, int row,
                                          int pitch, int spitch, int step, int g)
{
#pragma unroll
    for (int j = 0; j < 4; ++j)
        f.c[j] = load16(codes, step * 256 + j * 64 < pitch ? row * pitch + g * 16 : OUT_OF_RANGE, step * 256 + j * 64);
    const v4i s = load16(scales, step * 16 < spitch ? row * spitch : OUT_OF_RANGE, step * 16);
    f.s = mx4_scales_of(mx4_row_end(s, spitch - step * 16), g);
}

// Rows of K floats (aligned to their type only), quantised by the whole block into LDS: a thread takes 32 consecutive
// values, so that every value is read and quantised once.  Rows lie an odd number of 16 bytes apart: sixteen rows read at
// one place are in different banks.
__host__ __device__ inline int few_code_pitch(int steps) { return steps * 256 + 16; }
__host__ __device__ inline int few_scale_pitch(int steps) { return steps * 16 + 16; }

template <typename T> struct FewItem {
    Mx4In<T> in[4];
    int code_at, scale_at;
    __device__ __forceinline__ void fetch(const T *x, long long ldx, int K, int steps, int item, int items)
    {
        const int blocks = steps * 16, row = item / blocks, b = item - row * blocks, k = b * 32, whole = K & ~7;
        const bool any = item < items;
        const T *const src = x + row * ldx;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            in[i] = zero_eight<T>();
            if (any && k + 8 * i < whole) in[i] = load_eight(src + k + 8 * i);
        }
        if (any && whole < K && whole >> 5 == b) {               // the group that the row ends in
            const Mx4In<T> rest = load_some(src + whole, K - whole);
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (i == (whole >> 3 & 3)) in[i] = rest;
        }
        code_at = any ? row * few_code_pitch(steps) + b * 16 : -1;
        scale_at = row * few_scale_pitch(steps) + b;
    }
    __device__ __forceinline__ void quantize(uint8_t *codes, uint8_t *scales) const
    {
        const uint32_t top = max(max(in[0].top(), in[1].top()), max(in[2].top(), in[3].top()));
        const uint32_t s = mx4_scale_byte(top);
        const float scale = mx4_scale_float(s);
        if (code_at < 0) return;
        *reinterpret_cast<v4i *>(codes + code_at) = (v4i){(int)in[0].codes(scale), (int)in[1].codes(scale),
                                                          (int)in[2].codes(scale), (int)in[3].codes(scale)};
        scales[scale_at] = (uint8_t)s;
    }
};

// weights as they lie in memory: expanded (masked) or their scales put in order (held) when they are used
template <bool MASKED> struct FewWeights;
template <> struct FewWeights<false> {
    v4i c[4], s;
    __device__ __forceinline__ void load(const Mx4Args &p, int tile, int step, int lane)
    {
        const int pitch = p.kp >> 1, spitch = p.kp >> 5, r = lane & 15, g = lane >> 4;
        const __amdgpu_buffer_rsrc_t wr = rows_of(p.w, (uint32_t)tile * 16, p.N, 16, pitch);
        const __amdgpu_buffer_rsrc_t wsr = rows_of(p.ws, (uint32_t)tile * 16, p.N, 16, spitch);
#pragma unroll
        for (int j = 0; j < 4; ++j)
            c[j] = load16(wr, step * 256 + j * 64 < pitch ? r * pitch + g * 16 : OUT_OF_RANGE, step * 256 + j * 64);
        s = load16(wsr, step * 16 < spitch ? r * spitch : OUT_OF_RANGE, step * 16);
    }
    __device__ __forceinline__ v4i codes(int j) const { return c[j]; }
    __device__ __forceinline__ uint32_t scales(const Mx4Args &p, int step, int g) const
    {
        return mx4_scales_of(mx4_row_end(s, (p.kp >> 5) - step * 16), g);
    }
};
template <> struct FewWeights<true> {
    v4i c[2];
    __device__ __forceinline__ void load(const Mx4Args &p, int tile, int step, int lane)
    {
        const __amdgpu_buffer_rsrc_t wr = rows_of(p.w, tile, ((uint32_t)p.N + 15) / 16, 1, p.steps * 2048);
#pragma unroll
        for (int h = 0; h < 2; ++h)
            c[h] = load16(wr, step < p.steps ? lane * 16 : OUT_OF_RANGE, step * 2048 + h * 1024);
    }
    __device__ __forceinline__ v4i codes(int j) const
    {
        const v4i v = c[j >> 1];
        return (j & 1) ? expand_masked((uint32_t)v.z, (uint32_t)v.w) : expand_masked((uint32_t)v.x, (uint32_t)v.y);
    }
    __device__ __forceinline__ uint32_t scales(const Mx4Args &, int, int) const { return 0x7f7f7f7fu; }
};

// X: type of the rows, HELD or that of floats.  MT: 16 rows each.  SW: steps of a wave at most, with the rows' fragments kept in
// registers; 0: any number, the rows read again for every 16 outputs.
template <int X, bool MASKED, int MT, int SW>
__global__ __launch_bounds__(64 * FEW_WAVES) void mx4_few_kernel(const Mx4Args p)
{
    // first the quantised rows, then the waves' sums [2][wave][MT][64 lanes]
    extern __shared__ v4i shared[];
    v4f *const part = reinterpret_cast<v4f *>(shared);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
    const int r = lane & 15, g = lane >> 4, pitch = p.kp >> 1, spitch = p.kp >> 5, tiles = p.tiles_n;
    constexpr int KEPT = SW ? SW : 1;

    using XT = typename Mx4Type<X>::T;
    FewWeights<MASKED> w[KEPT];
    Mx4Frag x[MT][KEPT];
    auto load_weights = [&](int k, int tile) { w[k].load(p, tile, wave + k * waves, lane); };
    auto load_rows = [&](int k, int step) {
#pragma unroll
        for (int i = 0; i < MT; ++i)
            load_held(x[i][k], rows_of(p.x, 0, p.M, 16 * MT, pitch), rows_of(p.xs, 0, p.M, 16 * MT, spitch),
                      min(16 * i + r, p.M - 1), pitch, spitch, step, g);
    };

    int tile = blockIdx.x;
    // the rows before the weights: they come from the cache, and loads return in order
    if constexpr (X == HELD && SW) {
#pragma unroll
        for (int k = 0; k < KEPT; ++k) {
            load_rows(k, wave + k * waves);
            load_weights(k, tile);
        }
    }
    if constexpr (X != HELD) {
        uint8_t *const codes = reinterpret_cast<uint8_t *>(shared), *const scales = codes + p.M * few_code_pitch(p.steps);
        const int items = p.M * p.steps * 16;
        constexpr int TOGETHER = sizeof(XT) == 4 ? 1 : 2;
        FewItem<XT> item[TOGETHER];
        auto fetch = [&](int at) {
#pragma unroll
            for (int t = 0; t < TOGETHER; ++t) item[t].fetch((const XT *)p.x, p.ldx, p.K, p.steps, at + t * blockDim.x, items);
        };
        auto quantize = [&] {
#pragma unroll
            for (int t = 0; t < TOGETHER; ++t) item[t].quantize(codes, scales);
        };
        fetch(threadIdx.x);
#pragma unroll
        for (int k = 0; k < KEPT; ++k) load_weights(k, tile);
        quantize();
        for (int at = threadIdx.x + TOGETHER * blockDim.x; at < items; at += TOGETHER * blockDim.x) {
            fetch(at);
            quantize();
        }
        __syncthreads();
        const int row = min(r, p.M - 1);
#pragma unroll
        for (int k = 0; k < KEPT; ++k) {
            const int step = min(wave + k * waves, p.steps - 1);
            const v4i *const c = reinterpret_cast<const v4i *>(codes + row * few_code_pitch(p.steps) + step * 256);
#pragma unroll
            for (int j = 0; j < 4; ++j) x[0][k].c[j] = c[j * 4 + g];
            x[0][k].s = mx4_scales_of(*reinterpret_cast<const v4i *>(scales + row * few_scale_pitch(p.steps) + step * 16), g);
        }
        __syncthreads();
    }
    for (int turn = 0; tile < tiles; ++turn) {
        const int next = tile + gridDim.x;
        v4f acc[MT];
#pragma unroll
        for (int i = 0; i < MT; ++i) acc[i] = (v4f){0, 0, 0, 0};
        auto multiply = [&](int k, int step) {
            const uint32_t s = w[k].scales(p, step, g);
            repeat<4>([&](auto number) {
                constexpr int j = decltype(number)::value;
                const v4i c = w[k].codes(j);
#pragma unroll
                for (int i = 0; i < MT; ++i) acc[i] = mx4_mfma<j>(c, s, x[i][k].c[j], x[i][k].s, acc[i]);
            });
        };
        if (SW) {
#pragma unroll
            for (int k = 0; k < KEPT; ++k) {
                multiply(k, wave + k * waves);
                load_weights(k, next);
            }
        } else {
            for (int step = wave; step < p.steps; step += waves) {
                w[0].load(p, tile, step, lane);
                load_rows(0, step);
                multiply(0, step);
            }
        }
#pragma unroll
        for (int i = 0; i < MT; ++i) part[(((turn & 1) * waves + wave) * MT + i) * 64 + lane] = acc[i];
        __syncthreads();
        // the waves take turns at adding up
#pragma unroll
        for (int i = 0; i < MT; ++i)
            if ((turn * MT + i) % waves == wave) {
                const v4f *const sums = part + (((turn & 1) * waves) * MT + i) * 64 + lane;
                v4f v[1][1] = {{sums[0]}};
                for (int s = 1; s < waves; ++s) v[0][0] += sums[s * MT * 64];
                store_tile<1, 1>(p, v, 16 * i + r, (uint32_t)tile * 16 + 4 * g);
            }
        tile = next;
    }
}

template <int X, bool MASKED, int MT, int SW> static int launch_few(const char *fn, Mx4Args p, hipStream_t s)
{
    p.tiles_n = ceil_div(p.N, 16);
    const int waves = min(FEW_WAVES, p.steps);
    const int blocks = min(p.tiles_n, 256 * FEW_WAVES / waves);
    size_t lds = (size_t)2 * waves * MT * 1024;
    if (X != HELD) lds = max(lds, (size_t)p.M * (few_code_pitch(p.steps) + few_scale_pitch(p.steps)));
    MBU_LAUNCH((mx4_few_kernel<X, MASKED, MT, SW>), dim3((unsigned)blocks), dim3(64 * waves), lds, s, p);
    return check_launch(fn);
}

template <int X, bool MASKED> static int choose_few(const char *fn, const Mx4Args &p, hipStream_t s)
{
    const int each = ceil_div(p.steps, FEW_WAVES);                 // steps of a wave
    if (p.M <= 16) {
        if (each <= 1) return launch_few<X, MASKED, 1, 1>(fn, p, s);
        if (each <= 2) return launch_few<X, MASKED, 1, 2>(fn, p, s);
        if constexpr (X == HELD) return launch_few<X, MASKED, 1, 0>(fn, p, s);
    }
    if constexpr (X == HELD) {
        if (p.M <= 32) return each <= 1 ? launch_few<X, MASKED, 2, 1>(fn, p, s) : launch_few<X, MASKED, 2, 0>(fn, p, s);
        return each <= 1 ? launch_few<X, MASKED, 4, 1>(fn, p, s) : launch_few<X, MASKED, 4, 0>(fn, p, s);
    }
    return fail(MBU_ERR_SHAPE, "%s: no kernel", fn);
}

// Rows of floats that a product quantises on the way: every block quantises all of them, which beyond 2^17 values takes
// longer than a launch that quantises them once (8 x 14336 by 4096 outputs: 12.8 against 9.9 us and a launch of 2.5;
// 16 x 16384: 18.9 against 10.5 and 3).  The fragments of all inputs have to fit into registers.
bool mx4_few_floats(int M, int K)
{
    const int steps = ceil_div(mx4_padded(K), 512);
    return M <= 16 && steps <= 2 * FEW_WAVES && M * steps <= 256;
}

template <int X> static int choose_weights(const char *fn, const Mx4Args &p, bool masked, hipStream_t s)
{
    return masked ? choose_few<X, true>(fn, p, s) : choose_few<X, false>(fn, p, s);
}

int launch_mx4_few_floats(const char *fn, const void *x, int x_dtype, int M, long long stride, bool masked, const void *w,
                          const uint8_t *ws, int N, int K, const float *alpha, const float *bias, void *out, int dtype,
                          hipStream_t s)
{
    const int kp = mx4_padded(K);
    const Mx4Args p = {x, nullptr, w, ws, alpha, bias, out, stride, M, N, K, kp, ceil_div(kp, 512), 0, dtype};
    if (x_dtype == MBU_FLOAT32) return choose_weights<MBU_FLOAT32>(fn, p, masked, s);
    if (x_dtype == MBU_FLOAT16) return choose_weights<MBU_FLOAT16>(fn, p, masked, s);
    return choose_weights<MBU_BFLOAT16>(fn, p, masked, s);
}

int launch_mx4_matmul(const char *fn, const uint8_t *a, const uint8_t *as, int M, bool masked, const void *w,
                      const uint8_t *ws, int N, int K, const float *alpha, const float *bias, void *out, int dtype,
                      hipStream_t s)
{
    const int kp = mx4_padded(K);
    const Mx4Args p = {a, as, w, ws, alpha, bias, out, 0, M, N, K, kp, ceil_div(kp, 512), 0, dtype};
    if (M <= 64) return choose_weights<HELD>(fn, p, masked, s);
    return masked ? launch_mx4_tile_masked(fn, p, s) : launch_mx4_tile_held(fn, p, s);
}

}  // namespace mbu
