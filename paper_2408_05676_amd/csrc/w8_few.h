// Products of few rows in 8-bit codes with 8-bit weights (see eight_bit.h): the waves of a workgroup share the inputs of its outputs.
//
// out[r][n] = s_x[r] s_w[n] sum of c_x c_w. A wave takes its share of the inputs of 16 NT outputs and 16 MT rows, weights a kilobyte a load straight into registers; the
// waves' sums meet in LDS. Every workgroup reads its rows whole, from L2: with few outputs (one layer's 4096) that is as much as the weights from some 30 rows on.
//
// Bound: the weights' way from memory (in a graph of twenty launches, six matrices in turn: one row gated 4096 -> 2 x 11008 90 MB in 20.2 us, 4.5 TB/s where a long read reaches 5.5; nine rows
// 4096 -> 12288 13.7 us, 11008 -> 4096 10.6; with three matrices in turn, which the last-level cache holds in part, 16.0 us for the first), with more rows theirs through LDS too (72 rows 11008 -> 4096 16.6 us, 2048 -> 6144 7.6 us: start 0.7, stages 3.9, sums 1, launch 2).
#pragma once

#include "w8_tile.h"

namespace laser {

// MT: fragments of 16 rows; 0: up to four rows, whose codes come straight into registers (their lanes share lines of memory anyway). NT: fragments of 16
// outputs. WK: waves, each with a share of the inputs, its own ring of rows in LDS and no barrier before its sums are complete.
struct W8Few { int mt, nt, wk; };
constexpr int w8_few_stages(W8Few f) { return f.mt * f.wk * 2048 * 4 <= 81920 ? 4 : f.mt * f.wk * 2048 * 3 <= 163840 ? 3 : 2; }
constexpr int w8_few_lds(W8Few f) {
    const int ring = f.mt * f.wk * 2048 * w8_few_stages(f), sums = (f.mt ? f.mt : 1) * f.nt * f.wk * 1024;
    return ring > sums ? ring : sums;
}

// sum s_w s_x. FAR: some weights' scales are not within 2^-126 .. 2^97, so that a sum times one may pass fp32 or lose bits below its normal numbers where the product with both
// scales does not; it goes through their mantissas. In between the bits are the same. Such matrices have kernels of their own at any number of rows (704 rows gated 4096 -> 2 x 11008 135 us of 60):
// in the tiles, whose epilogue is a seventh of a launch, mantissas took 256 rows of that product from 35.7 to 36.4 us, a branch past them 704 rows of 4096 -> 12288 from 40.1 to 41.6,
// and a branch here 72 rows of 2048 -> 6144 from 7.7 to 8.0.
template <bool FAR>
__device__ inline float w8_scaled(int sum, float sw, float sx) {
    if constexpr (!FAR) return (float)sum * sw * sx;
    else return __builtin_ldexpf((float)sum * __builtin_amdgcn_frexp_mantf(sw) * __builtin_amdgcn_frexp_mantf(sx), __builtin_amdgcn_frexp_expf(sw) + __builtin_amdgcn_frexp_expf(sx));
}

template <int MT_, int NT, int WK, bool GATED, bool FAR = false>
__global__ __launch_bounds__(64 * WK) void w8_few_kernel(W8Args a) {
    constexpr W8Few F{MT_, NT, WK};
    constexpr bool DIRECT = MT_ == 0;
    constexpr int MT = DIRECT ? 1 : MT_, NA = GATED ? 2 : 1, NS = w8_few_stages(F), WS = NT == 1 ? 4 : 3, STAGE = MT * 2048;
    static_assert(NT % NA == 0 && WS >= NS - 1 && w8_few_lds(F) <= 163840, "");
    __shared__ __attribute__((aligned(1024))) char lds[w8_few_lds(F)];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
    // an XCD takes an equal share of the units, row tiles of the same outputs one after the other: their weights come to its L2 once
    const int units = a.tiles_m * a.tiles_n, per = (units + 7) / 8, li = blockIdx.x / 8, unit = (blockIdx.x % 8) * per + li;
    if (li >= per || unit >= units) return;
    const int tiles = a.rows / 16, tile0 = unit / a.tiles_m * NT, row0 = unit % a.tiles_m * MT * 16;
    const int nst = a.Kp / 128, nx = (a.Kd + 127) / 128;             // stages of 128 inputs; nst is even, where nx is odd the last stage of weights is zeros
    const int k0 = (int)((long)nst * wave / WK), k1 = (int)((long)nst * (wave + 1) / WK);

    // The scales' lines are asked for now: behind the last product they would be a round trip to memory.
    const float touch_w = a.w_scales[min(tile0 * 16 + (int)threadIdx.x, a.rows - 1)], touch_x = a.x_scales[min(row0 + (int)threadIdx.x, a.M - 1)];
    int4_t acc[NT][MT];
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int i = 0; i < MT; ++i) acc[j][i] = int4_t{0, 0, 0, 0};
    if (k0 < k1) {
        // ---- rows: chunk c of row r sits at c ^ (r / 2 % 8)
        uint32_t voff[2 * MT];
#pragma unroll
        for (int p = 0; p < 2 * MT; ++p) {
            const int row = p * 8 + (lane >> 3);
            voff[p] = (uint32_t)min(row, a.M - 1 - row0) * (uint32_t)a.x_stride + (((lane & 7) ^ ((row >> 1) & 7)) * 16);
        }
        uint64_t xbase = (uint64_t)(uintptr_t)a.x + (uint64_t)row0 * a.x_stride + (uint64_t)min(k0, nx - 1) * 128;
        const uint32_t ring = lds_address(lds) + wave * NS * STAGE;
        const char* const mine = lds + wave * NS * STAGE;
        int kreq = k0, fill = 0, slot = 0;
        auto request_x = [&] {
#pragma unroll
            for (int p = 0; p < 2 * MT; ++p) load_to_lds(xbase, voff[p], ring + fill + p * 1024);
            ++kreq;
            xbase += kreq < nx ? 128 : 0;                            // (past the last stage it comes again; nobody reads it)
            fill = fill + STAGE < NS * STAGE ? fill + STAGE : 0;
        };
        const uint32_t xo = (uint32_t)min(r, a.M - 1 - row0) * (uint32_t)a.x_stride + 16 * g;
        // ---- weights (and rows, DIRECT), WS stages ahead
        uint32_t wo[NT];
#pragma unroll
        for (int j = 0; j < NT; ++j) wo[j] = (uint32_t)(min(tile0 + j, tiles - 1) - tile0) * 1024 + lane * 16;
        const uint64_t wstep = (uint64_t)tiles * 1024;
        const uint8_t* wbase = a.w + (size_t)tile0 * 1024 + (size_t)k0 * 2 * wstep;
        int wreq = k0;
        u32x4 wq[WS][2][NT], xq[DIRECT ? WS : 1][2];
        const int8_t* xd = a.x + (size_t)row0 * a.x_stride + (size_t)min(k0, nx - 1) * 128;
        auto request_w = [&](auto uc) {
            constexpr int u = decltype(uc)::value;
#pragma unroll
            for (int s = 0; s < 2; ++s) {
#pragma unroll
                for (int j = 0; j < NT; ++j) wq[u][s][j] = *reinterpret_cast<const u32x4*>(wbase + s * wstep + wo[j]);
                if constexpr (DIRECT) xq[u][s] = *reinterpret_cast<const u32x4*>(xd + xo + s * 64);
            }
            ++wreq;
            wbase += wreq < k1 ? 2 * wstep : 0;
            if constexpr (DIRECT) xd += wreq < min(k1, nx) ? 128 : 0;
        };
        if constexpr (!DIRECT)
#pragma unroll
            for (int s = 0; s < NS - 1; ++s) request_x();
        static_for<0, WS>([&](auto uc) { request_w(uc); __builtin_amdgcn_sched_barrier(0); });
        uint32_t ox[2];
#pragma unroll
        for (int s = 0; s < 2; ++s) ox[s] = r * 128 + (((s * 4 + g) ^ ((r >> 1) & 7)) * 16);
        for (int kt = k0; kt < k1; kt += WS)
            static_for<0, WS>([&](auto uc) {
                constexpr int u = decltype(uc)::value;
                if (kt + u < k1) {
                    if constexpr (!DIRECT) {
                        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");       // the slot's last reads
                        request_x();
                        // newer than the rows waited for: those of NS - 1 stages and as many stages' weights
                        asm volatile("s_waitcnt vmcnt(%0)" ::"n"((NS - 1) * (2 * MT + 2 * NT) < 63 ? (NS - 1) * (2 * MT + 2 * NT) : 63) : "memory");
                    }
#pragma unroll
                    for (int s = 0; s < 2; ++s) {
                        u32x4 fx[MT];
#pragma unroll
                        for (int i = 0; i < MT; ++i) {
                            if constexpr (DIRECT) fx[i] = xq[u][s];
                            else fx[i] = *reinterpret_cast<const u32x4*>(mine + slot + ox[s] + i * 2048);
                        }
#pragma unroll
                        for (int j = 0; j < NT; ++j)
#pragma unroll
                            for (int i = 0; i < MT; ++i) acc[j][i] = mfma_i8(wq[u][s][j], fx[i], acc[j][i]);
                    }
                    slot = slot + STAGE < NS * STAGE ? slot + STAGE : 0;
                    request_w(uc);
                }
            });
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");               // surplus rows must not land in what follows
    }

    asm volatile("" ::"v"(touch_w), "v"(touch_x));
    // ---- the waves' sums; a thread adds up, scales and stores four outputs of a row, threads side by side the next ones
    __syncthreads();
    int4_t* const sums = reinterpret_cast<int4_t*>(lds);             // [wave][output fragment][row][four outputs]
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int i = 0; i < MT; ++i) sums[((wave * NT + j) * MT + i) * 64 + r * 4 + g] = acc[j][i];
    __syncthreads();
    auto store = [&](auto dt) {
        constexpr int PER = NT / NA * 4;
        for (int idx = threadIdx.x; idx < MT * 16 * PER; idx += 64 * WK) {
            const int j = idx % PER / 4 * NA, rr = idx / PER, row = row0 + rr, n = (tile0 + j) * 16 + 4 * (idx & 3), at = rr * 4 + (idx & 3);
            if (row >= a.M || tile0 + j >= tiles) continue;
            float o[NA][4];
#pragma unroll
            for (int h = 0; h < NA; ++h) {
                int4_t v = sums[(j + h) * MT * 64 + at];
#pragma unroll
                for (int w = 1; w < WK; ++w) v += sums[(w * NT + j + h) * MT * 64 + at];
                const float4_t sw = *reinterpret_cast<const float4_t*>(a.w_scales + n + 16 * h);
#pragma unroll
                for (int e = 0; e < 4; ++e) o[h][e] = w8_scaled<FAR>(v[e], sw[e], a.x_scales[row]);
            }
            if constexpr (GATED)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[0][e] = silu_times(o[0][e], o[NA - 1][e]);
            w8_store<decltype(dt)::value>(a, row, GATED ? (tile0 + j) * 8 + 4 * (idx & 3) : n, o[0]);
        }
    };
    if (a.dtype == DT_F16) store(std::integral_constant<int, DT_F16>{});
    else if (a.dtype == DT_BF16) store(std::integral_constant<int, DT_BF16>{});
    else store(std::integral_constant<int, DT_F32>{});
}

constexpr W8Few kW8Few[] = {{0, 1, 8}, {0, 2, 4}, {1, 1, 8}, {1, 2, 4}, {2, 2, 4}, {2, 4, 4}, {3, 2, 4}, {3, 4, 4}, {4, 4, 4}};
constexpr int kW8FewN = (int)(sizeof(kW8Few) / sizeof(kW8Few[0]));

template <int V, bool GATED, bool FAR>
inline void go_w8_few(W8Args a, hipStream_t stream) {
    constexpr W8Few F = kW8Few[V];
    a.tiles_m = (a.M + (F.mt ? F.mt : 1) * 16 - 1) / ((F.mt ? F.mt : 1) * 16);
    a.tiles_n = (a.rows / 16 + F.nt - 1) / F.nt;
    launch(w8_few_kernel<F.mt, F.nt, F.wk, GATED, FAR>, dim3(8u * (unsigned)((a.tiles_m * a.tiles_n + 7) / 8)), dim3(64 * F.wk), stream, a);
}
inline void launch_w8_few(const W8Args& a, bool gated, int v, hipStream_t stream) {
    each<0, kW8FewN>([&](auto vc) {
        constexpr int V = decltype(vc)::value;
        if (V != v) return;
        if constexpr (kW8Few[V].nt % 2 == 0)
            if (gated) go_w8_few<V, true, false>(a, stream);
        if (!gated) go_w8_few<V, false, false>(a, stream);
    });
}
inline void launch_w8_far(const W8Args& a, bool gated, hipStream_t stream) {
    constexpr int ONE = 3, MANY = kW8FewN - 1;                       // {1, 2, 4}, {4, 4, 4}
    if (a.M <= 16) gated ? go_w8_few<ONE, true, true>(a, stream) : go_w8_few<ONE, false, true>(a, stream);
    else gated ? go_w8_few<MANY, true, true>(a, stream) : go_w8_few<MANY, false, true>(a, stream);
}

}  // namespace laser
