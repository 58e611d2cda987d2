// Products in the microscaled 4-bit format for many rows: activations through LDS, weights straight into registers.
//
// A block takes 16 MT rows by 4 x 16 NT outputs: each of its four waves all rows by 16 NT outputs of its own.  The sum
// runs in steps of 512 inputs (mx4_matmul.hip has the assignment of inputs to lanes).  Every wave needs all activations of a
// step and only its own weights, so the activations (256 bytes of a row per step) go through a double-buffered LDS
// window, and the weights, which nobody shares, from global memory into the registers of the lane that multiplies them.
#include "mx4_product.h"

namespace mbu {

// unit of 16 bytes `chunk` of a row of the window; the exclusive or spreads the 16 rows that a quarter of a wave reads
// over all banks
__device__ __forceinline__ int window_unit(int row, int chunk) { return row * 16 + (chunk ^ (row & 15)); }

// Weights of a wave: SLOTS of 16 bytes per lane and 16 outputs, a slot for one instruction (held) or for two (masked).
template <Mx4Weights WK, int NT, int SLOTS> struct TileWeights {
    v4i c[SLOTS][NT];
    __device__ __forceinline__ v4i get(int j, int n) const
    {
        if (WK == W_HELD) return c[j % SLOTS][n];
        const v4i v = c[(j >> 1) % SLOTS][n];
        return (j & 1) ? expand_masked((uint32_t)v.z, (uint32_t)v.w) : expand_masked((uint32_t)v.x, (uint32_t)v.y);
    }
};

template <Mx4Weights WK, int MW, int MT, int NT, int SLOTS, typename OT>
__global__ __launch_bounds__(256 * MW, 2) void mx4_tile_kernel(const Mx4Args p)
{
    constexpr int BM = 16 * MT * MW, BN = 64 * NT, THREADS = 256 * MW;
    __shared__ v4i window[2][BM * 16];
    __shared__ v4i window_scales[2][THREADS];                    // rows behind BM: zeros, never read
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int r = lane & 15, g = lane >> 4, wn = wave & 3, wm = wave >> 2;

    const TileAt at_tile = tile_of_block(p.tiles_n, (int)(((uint32_t)p.M + BM - 1) / BM));
    const int tm = at_tile.m, tn = at_tile.n;
    const uint32_t m0 = (uint32_t)tm * BM, n0 = (uint32_t)tn * BN + wn * 16 * NT;

    const int pitch = p.kp >> 1, spitch = p.kp >> 5, steps = p.steps;
    const __amdgpu_buffer_rsrc_t xr = rows_of(p.x, m0, p.M, BM, pitch), xsr = rows_of(p.xs, m0, p.M, BM, spitch);
    const uint32_t nw = min(n0, (uint32_t)p.N - 1);              // a wave behind the last output: nothing is stored
    const uint32_t tiles_w = ((uint32_t)p.N + 15) / 16;
    const __amdgpu_buffer_rsrc_t wr = WK == W_HELD ? rows_of(p.w, nw, p.N, 16 * NT, pitch)
                                                   : rows_of(p.w, nw / 16, tiles_w, NT, steps * 2048);
    const __amdgpu_buffer_rsrc_t wsr = rows_of(WK == W_HELD ? p.ws : p.xs, WK == W_HELD ? nw : 0, WK == W_HELD ? p.N : 1, 16 * NT, spitch);

    const int srow = tid >> 4, schunk = tid & 15;                // what the thread stages: rows srow + 16 MW q
    const int x_lane = srow * pitch + schunk * 16, xs_lane = tid < BM ? tid * spitch : OUT_OF_RANGE;
    const int w_lane = WK == W_HELD ? r * pitch + g * 16 : lane * 16, ws_lane = r * spitch;
    const int write_unit = window_unit(srow, schunk);
    const int read_row = wm * 16 * MT + r;
    int read_unit[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) read_unit[j] = window_unit(read_row, 4 * j + g);

    v4f acc[MT][NT];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int n = 0; n < NT; ++n) acc[i][n] = (v4f){0, 0, 0, 0};

    TileWeights<WK, NT, SLOTS> w;
    uint32_t ws[NT];
    constexpr int PER_STEP = WK == W_HELD ? 4 : 2;               // slots that a step goes through
    // slot number `at` of a step, counted on into the next one
    auto load_weights = [&](int at, int step) {
        step += at / PER_STEP;
        const int slot = at % PER_STEP;
        const int off = (WK == W_HELD ? step * 256 + slot * 64 < pitch : step < steps) ? w_lane : OUT_OF_RANGE;
#pragma unroll
        for (int n = 0; n < NT; ++n)
            w.c[at % SLOTS][n] = WK == W_HELD ? load16(wr, off + 64 * slot, n * 16 * pitch + step * 256)
                                              : load16(wr, off + 1024 * slot, (n * steps + step) * 2048);
    };
    auto load_weight_scales = [&](int step, v4i (&to)[NT]) {
#pragma unroll
        for (int n = 0; n < NT; ++n)
            if (WK == W_HELD) to[n] = load16(wsr, ws_lane, n * 16 * spitch + step * 16);
    };
    auto take_weight_scales = [&](int step, const v4i (&from)[NT]) {
#pragma unroll
        for (int n = 0; n < NT; ++n)
            ws[n] = WK == W_HELD ? mx4_scales_of(mx4_row_end(from[n], spitch - step * 16), g) : 0x7f7f7f7fu;
    };
    auto stage = [&](int q, int step) {
        const int off = step * 256 + schunk * 16 < pitch ? x_lane : OUT_OF_RANGE;
        return load16(xr, off, q * 16 * MW * pitch + step * 256);
    };
    // the scales of one row, in the order in which the lanes take them: word g of a row for lane group g
    auto stage_scales = [&](int step) { return load16(xsr, xs_lane, step * 16); };
    auto in_lane_order = [&](v4i s, int step) {
        s = mx4_row_end(s, spitch - step * 16);
        return (v4i){(int)mx4_scales_of(s, 0), (int)mx4_scales_of(s, 1), (int)mx4_scales_of(s, 2), (int)mx4_scales_of(s, 3)};
    };

    {
        v4i st[MT];
#pragma unroll
        for (int q = 0; q < MT; ++q) st[q] = stage(q, 0);
        const v4i ss = stage_scales(0);
#pragma unroll
        for (int j = 0; j < SLOTS; ++j) load_weights(j, 0);
        v4i ws0[NT];
        load_weight_scales(0, ws0);
        take_weight_scales(0, ws0);
#pragma unroll
        for (int q = 0; q < MT; ++q) window[0][write_unit + q * 256 * MW] = st[q];
        window_scales[0][tid] = in_lane_order(ss, 0);
    }
    __syncthreads();

    for (int step = 0; step < steps; ++step) {
        const v4i *cur = window[step & 1];
        const uint32_t *cur_scales = reinterpret_cast<const uint32_t *>(window_scales[step & 1]) + read_row * 4 + g;
        v4i *nxt = window[(step & 1) ^ 1];
        uint32_t xs[MT];
        v4i st[MT], f[4], ss, ws2[NT];
        constexpr int GROUPS = 4 * MT, EVERY = MT >= 8 ? 3 : 2, BEHIND = GROUPS - EVERY * MT;
        xs[0] = cur_scales[0];
        if (MT > 1) xs[1] = cur_scales[64];
        repeat<3>([&](auto group) {
            constexpr int G = decltype(group)::value;
            f[G] = cur[read_unit[G / MT] + (G % MT) * 256];
        });
        repeat<GROUPS>([&](auto group) {
            constexpr int G = decltype(group)::value, j = G / MT, i = G % MT;
            if constexpr (G + 3 < GROUPS) f[(G + 3) & 3] = cur[read_unit[(G + 3) / MT] + ((G + 3) % MT) * 256];
            if constexpr (G + 2 < MT) xs[G + 2] = cur_scales[(G + 2) * 64];
            if constexpr (G % EVERY == 0 && G / EVERY < MT) st[G / EVERY] = stage(G / EVERY, step + 1);
            if constexpr (G == MT) ss = stage_scales(step + 1);
            if constexpr (G == 3 * MT) load_weight_scales(step + 1, ws2);
            if constexpr (G >= BEHIND && (G - BEHIND) % EVERY == 0 && (G - BEHIND) / EVERY < MT)
                nxt[write_unit + (G - BEHIND) / EVERY * 256 * MW] = st[(G - BEHIND) / EVERY];
            if constexpr (G == GROUPS - 1) window_scales[(step & 1) ^ 1][tid] = in_lane_order(ss, step + 1);
#pragma unroll
            for (int n = 0; n < NT; ++n)
                acc[i][n] = mx4_mfma<j>(w.get(j, n), ws[n], f[G & 3], xs[i], acc[i][n]);
            __builtin_amdgcn_sched_barrier(0);
            if constexpr (i == MT - 1) {
                if constexpr (WK == W_HELD) load_weights(j + SLOTS, step);
                else if constexpr (j & 1) load_weights((j >> 1) + SLOTS, step);
            }
        });
        take_weight_scales(step + 1, ws2);
        __syncthreads();
    }

    store_tile<MT, NT, OT>(p, acc, m0 + wm * 16 * MT + r, n0 + 4 * g);
}

template <Mx4Weights WK, int MW, int MT, int NT, typename OT>
static int launch_tile(const char *fn, Mx4Args p, hipStream_t s)
{
    constexpr int SLOTS = WK == W_MASKED || NT > 2 ? 2 : 4;
    p.tiles_n = ceil_div(p.N, 64 * NT);
    const long long blocks = (long long)ceil_div(p.M, 16 * MT * MW) * p.tiles_n;
    if (blocks > 0x7fffffffLL) return fail(MBU_ERR_SHAPE, "%s: product too large", fn);
    MBU_LAUNCH((mx4_tile_kernel<WK, MW, MT, NT, SLOTS, OT>), dim3((unsigned)blocks), dim3(256 * MW), 0, s, p);
    return check_launch(fn);
}

template <Mx4Weights WK, typename OT> static int choose_tile(const char *fn, const Mx4Args &p, hipStream_t s)
{
    if (WK == W_HELD) return launch_mx4_tile_held(fn, p, OutType<OT>(), s);
    if ((long long)ceil_div(p.M, 256) * ceil_div(p.N, 256) >= 192) return launch_tile<WK, 2, 8, 4, OT>(fn, p, s);
    if ((long long)ceil_div(p.M, 128) * ceil_div(p.N, 128) >= 192) return launch_tile<WK, 1, 8, 2, OT>(fn, p, s);
    return launch_tile<WK, 1, 4, 1, OT>(fn, p, s);
}

int launch_mx4_tile(const char *fn, const Mx4Args &p, bool masked, int dtype, hipStream_t s)
{
    if (dtype == MBU_FLOAT32) return masked ? choose_tile<W_MASKED, float>(fn, p, s) : choose_tile<W_HELD, float>(fn, p, s);
    if (dtype == MBU_FLOAT16) return masked ? choose_tile<W_MASKED, _Float16>(fn, p, s) : choose_tile<W_HELD, _Float16>(fn, p, s);
    return masked ? choose_tile<W_MASKED, __bf16>(fn, p, s) : choose_tile<W_HELD, __bf16>(fn, p, s);
}

}  // namespace mbu
