// Products in the microscaled 4-bit format for few rows (tokens): bound by reading the weights, each of which is read once.
//
// A block's waves share the steps of 512 inputs and take the same 16 outputs, so that even one token on a small layer
// keeps every compute unit busy; they add their sums up in LDS, in the waves' order, and go on to the next 16 outputs
// while the weights of those are on their way already.  The rows stay in registers as fragments, quantised there where
// they come as floats: a lane owns whole blocks of 32, so nothing crosses lanes.
#include "mx4_product.h"

namespace mbu {

constexpr int FEW_WAVES = 8;

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

// the same from a row of K floats (aligned to their type only), quantised here
template <typename T>
__device__ __forceinline__ void load_float(Mx4Frag &f, const T *row, int K, int step, int g)
{
    Mx4In<T> in[4][4];
    const int whole = K & ~7;                                    // values in whole groups of eight
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int k = step * 512 + j * 128 + g * 32 + 8 * i;
            in[j][i] = zero_eight<T>();
            if (k < whole) in[j][i] = load_eight(row + k);
        }
    if (whole < K && whole >> 9 == step) {                       // the group that the row ends in
        const Mx4In<T> rest = load_some(row + whole, K - whole);
        const int at = whole >> 7 & 3, part = whole >> 3 & 3;
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (j == at && i == part && g == (whole >> 5 & 3)) in[j][i] = rest;
    }
    f.s = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const uint32_t top = max(max(in[j][0].top(), in[j][1].top()), max(in[j][2].top(), in[j][3].top()));
        const uint32_t s = mx4_scale_byte(top);
        const float scale = mx4_scale_float(s);
        f.c[j] = (v4i){(int)in[j][0].codes(scale), (int)in[j][1].codes(scale), (int)in[j][2].codes(scale),
                       (int)in[j][3].codes(scale)};
        f.s |= s << (8 * j);
    }
    // the codes are made here, not where they are first used: the floats of one step at a time in registers
#pragma unroll
    for (int j = 0; j < 4; ++j) asm volatile("" : "+v"(f.c[j]));
}

// weights as they lie in memory: expanded (masked) or their scales put in order (held) when they are used
template <Mx4Weights WK> struct FewWeights;
template <> struct FewWeights<W_HELD> {
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
template <> struct FewWeights<W_MASKED> {
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

// XT: type of the rows (uint8_t: held).  MT: 16 rows each.  SW: steps of a wave at most, with the rows' fragments kept in
// registers; 0: any number, the rows read again for every 16 outputs.
template <typename XT, Mx4Weights WK, int MT, int SW>
__global__ __launch_bounds__(64 * FEW_WAVES) void mx4_few_kernel(const Mx4Args p)
{
    __shared__ v4f part[2][FEW_WAVES][MT][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
    const int r = lane & 15, g = lane >> 4, pitch = p.kp >> 1, spitch = p.kp >> 5, tiles = p.tiles_n;
    constexpr int KEPT = SW ? SW : 1;

    FewWeights<WK> w[KEPT];
    Mx4Frag x[MT][KEPT];
    auto load_weights = [&](int tile) {
#pragma unroll
        for (int k = 0; k < KEPT; ++k) w[k].load(p, tile, wave + k * waves, lane);
    };
    auto load_rows = [&](int k, int step) {
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            const int m = min(16 * i + r, p.M - 1);
            if constexpr (sizeof(XT) == 1)
                load_held(x[i][k], rows_of(p.x, 0, p.M, 16 * MT, pitch), rows_of(p.xs, 0, p.M, 16 * MT, spitch), m, pitch,
                          spitch, step, g);
            else load_float(x[i][k], (const XT *)p.x + m * p.ldx, p.K, step, g);
        }
    };

    int tile = blockIdx.x;
    if (SW) {
        load_weights(tile);
#pragma unroll
        for (int k = 0; k < KEPT; ++k) load_rows(k, wave + k * waves);
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
            for (int k = 0; k < KEPT; ++k) multiply(k, wave + k * waves);
            load_weights(next);
        } else {
            for (int step = wave; step < p.steps; step += waves) {
                w[0].load(p, tile, step, lane);
                load_rows(0, step);
                multiply(0, step);
            }
        }
#pragma unroll
        for (int i = 0; i < MT; ++i) part[turn & 1][wave][i][lane] = acc[i];
        __syncthreads();
        // the waves take turns at adding up
#pragma unroll
        for (int i = 0; i < MT; ++i)
            if ((turn * MT + i) % waves == wave) {
                v4f v[1][1] = {{part[turn & 1][0][i][lane]}};
                for (int s = 1; s < waves; ++s) v[0][0] += part[turn & 1][s][i][lane];
                store_tile<1, 1>(p, v, 16 * i + r, (uint32_t)tile * 16 + 4 * g);
            }
        tile = next;
    }
}

template <typename XT, Mx4Weights WK, int MT, int SW> static int launch_few(const char *fn, Mx4Args p, hipStream_t s)
{
    p.tiles_n = ceil_div(p.N, 16);
    const int waves = min(FEW_WAVES, p.steps);
    const int blocks = min(p.tiles_n, 512 * FEW_WAVES / waves);
    MBU_LAUNCH((mx4_few_kernel<XT, WK, MT, SW>), dim3((unsigned)blocks), dim3(64 * waves), 0, s, p);
    return check_launch(fn);
}

template <typename XT, Mx4Weights WK> static int choose_few(const char *fn, const Mx4Args &p, hipStream_t s)
{
    const int each = ceil_div(p.steps, FEW_WAVES);                 // steps of a wave
    if (p.M <= 16) {
        if (each <= 1) return launch_few<XT, WK, 1, 1>(fn, p, s);
        if (each <= 2) return launch_few<XT, WK, 1, 2>(fn, p, s);
        if (each <= 4) return launch_few<XT, WK, 1, 4>(fn, p, s);
        if constexpr (sizeof(XT) == 1) return launch_few<XT, WK, 1, 0>(fn, p, s);
    }
    if constexpr (sizeof(XT) == 1) {
        if (p.M <= 32) return each <= 1 ? launch_few<XT, WK, 2, 1>(fn, p, s) : launch_few<XT, WK, 2, 0>(fn, p, s);
        return each <= 1 ? launch_few<XT, WK, 4, 1>(fn, p, s) : launch_few<XT, WK, 4, 0>(fn, p, s);
    }
    return fail(MBU_ERR_SHAPE, "%s: no kernel", fn);
}

// rows of floats that a product quantises on the way: up to 16, with the fragments of all inputs in registers
bool mx4_few_floats(int M, int K) { return M <= 16 && ceil_div(mx4_padded(K), 512) <= 4 * FEW_WAVES; }

template <typename XT> static int choose_weights(const char *fn, const Mx4Args &p, bool masked, hipStream_t s)
{
    return masked ? choose_few<XT, W_MASKED>(fn, p, s) : choose_few<XT, W_HELD>(fn, p, s);
}

int launch_mx4_few_floats(const char *fn, const void *x, int x_dtype, int M, long long stride, bool masked, const void *w,
                          const uint8_t *ws, int N, int K, const float *alpha, const float *bias, void *out, int dtype,
                          hipStream_t s)
{
    const int kp = mx4_padded(K);
    const Mx4Args p = {x, nullptr, w, ws, alpha, bias, out, stride, M, N, K, kp, ceil_div(kp, 512), 0, dtype};
    if (x_dtype == MBU_FLOAT32) return choose_weights<float>(fn, p, masked, s);
    if (x_dtype == MBU_FLOAT16) return choose_weights<_Float16>(fn, p, masked, s);
    return choose_weights<__bf16>(fn, p, masked, s);
}

int launch_mx4_matmul(const char *fn, const uint8_t *a, const uint8_t *as, int M, bool masked, const void *w,
                      const uint8_t *ws, int N, int K, const float *alpha, const float *bias, void *out, int dtype,
                      hipStream_t s)
{
    const int kp = mx4_padded(K);
    const Mx4Args p = {a, as, w, ws, alpha, bias, out, 0, M, N, K, kp, ceil_div(kp, 512), 0, dtype};
    if (M <= 64) return choose_weights<uint8_t>(fn, p, masked, s);
    return masked ? launch_mx4_tile_masked(fn, p, s) : launch_mx4_tile_held(fn, p, s);
}

}  // namespace mbu
