// Rows into 8-bit codes with one scale each, alone or behind the residual's addition and the root-mean-square norm, and back.
//
// h = x + res, u = h gain (u = x without the norm), m = max |u|: codes c = rint(127 u / m) and scale s = m / 127 / sqrt(mean h^2 + eps).
// The root is the same for a row's elements, so codes need the extremes of h gain only. h, u and 127 u are 64-bit numbers, of which a code is the formula's exactly, and
// squares of any fp32 rows have room.
// Bound: a launch and one round trip to memory up to some hundred rows (1 x 4096 2.4 us, with the norm 3.6; an empty launch 2.3), then both and the vector
// instructions of the codes: 704 x 11008 fp16 7.1 us (3.3 TB/s; a copy of as many bytes takes 4.6), the norm of 704 x 4096 with its residual in bf16 7.7 us (2.6 TB/s). Reading back 5.3 us
// (704 x 11008, 4.4 TB/s).
#include <algorithm>

#include "eight_bit.h"

namespace laser {

constexpr int kNoResidual = -1;

template <int DT>
__device__ inline float load_elem(const void* p, int64_t o) {
    if constexpr (DT == DT_F32) return ((const float*)p)[o];
    else if constexpr (DT == DT_BF16) return bf16_to_f32(((const uint16_t*)p)[o]);
    else return f16_to_f32(((const uint16_t*)p)[o]);
}
template <int DT>
__device__ inline void store_elem(void* p, int64_t o, float x) {
    if constexpr (DT == DT_F32) ((float*)p)[o] = x;
    else if constexpr (DT == DT_BF16) ((uint16_t*)p)[o] = f32_to_bf16(x);
    else ((uint16_t*)p)[o] = f32_to_f16(x);
}

// Eight elements of a row as they lie in memory
template <int DT>
struct Raw8 {
    uint32_t w[DT == DT_F32 ? 8 : 4];
    __device__ float get(int i) const {
        if constexpr (DT == DT_F32) return __uint_as_float(w[i]);
        else if constexpr (DT == DT_BF16) return __uint_as_float(i & 1 ? w[i / 2] & 0xFFFF0000u : w[i / 2] << 16);
        else return f16_to_f32((uint16_t)(w[i / 2] >> (16 * (i & 1))));
    }
    __device__ float pick(int i) const {                 // the same for an i that is known at run time only
        auto two = [&](uint32_t a, uint32_t b, int bit) { return i & bit ? b : a; };
        if constexpr (DT == DT_F32) return __uint_as_float(two(two(two(w[0], w[1], 1), two(w[2], w[3], 1), 2), two(two(w[4], w[5], 1), two(w[6], w[7], 1), 2), 4));
        else {
            const uint16_t h = (uint16_t)(two(two(w[0], w[1], 2), two(w[2], w[3], 2), 4) >> (16 * (i & 1)));
            return DT == DT_BF16 ? bf16_to_f32(h) : f16_to_f32(h);
        }
    }
};
template <int DT>
__device__ inline void load8(Raw8<DT>& r, const void* p, int64_t o) {
    if constexpr (DT == DT_F32) {
        const f32x4_a4 *q = reinterpret_cast<const f32x4_a4*>((const float*)p + o), a = q[0], b = q[1];
#pragma unroll
        for (int i = 0; i < 4; ++i) { r.w[i] = __float_as_uint(a[i]); r.w[4 + i] = __float_as_uint(b[i]); }
    } else {
        const u32x4_a2 a = *reinterpret_cast<const u32x4_a2*>((const uint16_t*)p + o);
#pragma unroll
        for (int i = 0; i < 4; ++i) r.w[i] = a[i];
    }
}
template <int DT>
__device__ inline void store8(void* p, int64_t o, int left, const float (&x)[8]) {
    if (left >= 8) { store_elems<DT, 8>(p, o, x); return; }
#pragma unroll
    for (int i = 0; i < 8; ++i) if (i < left) store_elem<DT>(p, o + i, x[i]);
}
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
typedef unsigned u32x2_a1 __attribute__((ext_vector_type(2), aligned(1)));

// rint(127 u / m) in the low byte; rcp is 1 / m to a few places, so that c is the code or its neighbour, and what is left of 127 u tells which: it is exact, as c m has fewer
// bits than the fused product keeps. Adding 1.5 2^52 rounds to nearest even and leaves the whole number in the low bits.
__device__ inline uint32_t q8_code(double u, double rcp, double m) {
    constexpr double kWhole = 0x1.8p52;
    const double p = 127.0 * u, n = fma(p, rcp, kWhole), e = fma(kWhole - n, m, p), twice = fabs(e) + fabs(e);
    const uint32_t c = (uint32_t)__builtin_bit_cast(uint64_t, n);
    return twice > m || (twice == m && (c & 1)) ? c + (e > 0 ? 1u : ~0u) : c;
}

// x of another lane of the same sixteen (dpp control CTRL)
template <int CTRL, class T>
__device__ inline T row_move(T x) {
    if constexpr (sizeof(T) == 4) return __builtin_bit_cast(T, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CTRL, 0xF, 0xF, true));
    else {
        const uint64_t u = __builtin_bit_cast(uint64_t, x);
        const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)u, CTRL, 0xF, 0xF, true), hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(u >> 32), CTRL, 0xF, 0xF, true);
        return __builtin_bit_cast(T, (uint64_t)hi << 32 | lo);
    }
}
// op(a, b) of the sixteens (HALVES: halves) of a wave that lie side by side, in both: swapping x's odd ones with the even ones of a copy leaves all the even ones in one
// register and all the odd ones in the other.
template <bool HALVES, class T, class F>
__device__ inline T fold_sides(T x, F op) {
    auto swap = [](uint32_t a, uint32_t& even, uint32_t& odd) {
        if constexpr (HALVES) { const auto r = __builtin_amdgcn_permlane32_swap(a, a, false, false); even = r[0]; odd = r[1]; }
        else { const auto r = __builtin_amdgcn_permlane16_swap(a, a, false, false); even = r[0]; odd = r[1]; }
    };
    if constexpr (sizeof(T) == 4) {
        uint32_t a, b;
        swap(__builtin_bit_cast(uint32_t, x), a, b);
        return op(__builtin_bit_cast(T, a), __builtin_bit_cast(T, b));
    } else {
        const uint64_t u = __builtin_bit_cast(uint64_t, x);
        uint32_t al, bl, ah, bh;
        swap((uint32_t)u, al, bl);
        swap((uint32_t)(u >> 32), ah, bh);
        return op(__builtin_bit_cast(T, (uint64_t)ah << 32 | al), __builtin_bit_cast(T, (uint64_t)bh << 32 | bl));
    }
}
// op over a wave, in every lane
template <class T, class F>
__device__ inline T wave_fold(T x, F op) {
    x = op(x, row_move<0xB1>(x));                    // lanes 1 0 3 2 of four
    x = op(x, row_move<0x4E>(x));                    // lanes 2 3 0 1
    x = op(x, row_move<0x141>(x));                   // eight lanes mirrored
    x = op(x, row_move<0x140>(x));                   // sixteen mirrored
    x = fold_sides<false>(x, op);
    return fold_sides<true>(x, op);
}
__device__ inline double wave_max(double x) { return wave_fold(x, [](double a, double b) { return fmax(a, b); }); }
__device__ inline uint32_t wave_max(uint32_t x) { return wave_fold(x, [](uint32_t a, uint32_t b) { return max(a, b); }); }
__device__ inline double wave_sum(double x) { return wave_fold(x, [](double a, double b) { return a + b; }); }

// A row's scale. m: its largest |u|.
template <bool NORM>
__device__ inline float row_scale(double m, double ss, bool bad, int N, float eps) {
    double d = 127.0;
    if (NORM && m > 0) d *= sqrt(ss / N + (double)eps);
    return bad ? __builtin_nanf("") : (float)(m / d);
}

// WPR waves a row (four rows a workgroup where that is one), NV times eight columns a thread: the row stays in registers between its statistics and its codes.
// Behind the end of a row there are no elements: a thread that would pass it takes the last eight, some of them a second time (results are stored behind the barrier, when
// all have been read; only the squares leave the others' out).
//
// Codes take 32-bit numbers wherever those decide. inv is 127 / m with one rounding, u has one of the sum and one of the product with the gain (neither without the norm),
// t = u inv is never rounded itself and its distance from a whole number by 2^-25 at most: together less than 127 2^-24 + 2^-25 < 1.0625 2^-17, with the norm
// 3 127 2^-24 + 2^-25 < 1.5625 2^-16. (Sums of two floats never lose a small part; a product that does is 2^-66 of m.) Elements closer than that to a half take 64 bits, one at a time.
// A launch of some hundred rows has such elements somewhere, and waits for them: what costs is the way through instructions that no other wave has fetched, so they are few. 704 rows of
// 11008: all eight of a thread's in 64 bits 11.4 us; one at a time, with two divisions in the way 8.1 (with limits of 2^-14 as of 2^-22), without 7.1, not at all 6.1.
template <int DT, int RT, bool NORM, int WPR, int NV>
__global__ __launch_bounds__(WPR == 1 ? 256 : WPR * 64) void q8_rows_kernel(Q8Args a) {
    __shared__ __attribute__((aligned(16))) double sm_m[WPR], sm_ss[WPR];
    __shared__ __attribute__((aligned(16))) uint32_t sm_top[WPR];
    const int wave = threadIdx.x >> 6, t = WPR == 1 ? threadIdx.x & 63 : threadIdx.x;
    const int64_t row = WPR == 1 ? (int64_t)blockIdx.x * 4 + wave : blockIdx.x;
    if (WPR == 1 && row >= a.M) return;
    constexpr bool RES = RT != kNoResidual;
    Raw8<DT> x[NV];
    Raw8<RES ? RT : DT_F16> r[RES ? NV : 1];
    Raw8<DT_F32> g[NORM ? NV : 1];
    // All loads go out together, without a branch: a row has eight elements at least.
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        const int c = min((v * WPR * 64 + t) * 8, a.N - 8);
        load8<DT>(x[v], a.x, row * a.x_stride + c);
        if constexpr (RES) load8<RT>(r[v], a.res, row * a.res_stride + c);
        if constexpr (NORM) load8<DT_F32>(g[v], a.gain, c);
    }
    asm volatile("" ::: "memory");
    double m = 0, ss = 0;
    float z = 0;                                         // NaN where the gain is not finite
    uint32_t top = 0;                                    // without the norm: the largest |x| as its bits, which are in the order of the numbers, past the infinity's if one is
    u16x2 top2 = {0, 0};                                 // not a number; 16-bit elements in pairs
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        const int left = a.N - (v * WPR * 64 + t) * 8;
        if (left <= 0) continue;
        if constexpr (DT == DT_F32 && NORM)
            for (int p = 1; p < a.n_part; ++p) {         // sums of reduction parts (of whole pieces: the library's own), added to the first in fp32
                Raw8<DT_F32> q;
                load8<DT_F32>(q, a.x, row * a.x_stride + a.N - left + p * a.part_stride);
#pragma unroll
                for (int i = 0; i < 8; ++i) x[v].w[i] = __float_as_uint(x[v].get(i) + q.get(i));
            }
        if constexpr (NORM) {
            auto sum = [&](int i) {
                double h = (double)x[v].get(i);
                if constexpr (RES) h += (double)r[v].get(i);
                return h;
            };
            const double before = ss;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const double h = sum(i);
                m = fmax(m, fabs(h * (double)g[v].get(i)));
                ss = fma(h, h, ss);
                z = fmaf(g[v].get(i), 0.f, z);
            }
            if (left < 8) {
                ss = before;
#pragma unroll
                for (int i = 1; i < 8; ++i) ss = i >= 8 - left ? fma(sum(i), sum(i), ss) : ss;
            }
        } else
#pragma unroll
            for (const uint32_t w : x[v].w) {
                if constexpr (DT == DT_F32) top = max(top, w & 0x7FFFFFFFu);
                else top2 = __builtin_elementwise_max(top2, __builtin_bit_cast(u16x2, w & 0x7FFF7FFFu));
            }
    }
    // An infinite m stands for a row that is not finite: products of two floats stay below it. Only the first thread needs the squares.
    if constexpr (NORM) {
        if (!(z == 0) || !(ss < INFINITY)) m = INFINITY;     // (squares of finite sums do not pass 64 bits)
        m = wave_max(m);
        ss = wave_sum(ss);
        if constexpr (WPR > 1) {
            if ((t & 63) == 0) { sm_m[wave] = m; sm_ss[wave] = ss; }
            __syncthreads();
#pragma unroll
            for (int w = 0; w < WPR; ++w) m = fmax(m, sm_m[w]);
            if (t == 0)
#pragma unroll
                for (int w = 1; w < WPR; ++w) ss += sm_ss[w];
        }
    } else {
        if constexpr (DT != DT_F32) top = max(top2[0], top2[1]);
        top = wave_max(top);
        if constexpr (WPR > 1) {
            if ((t & 63) == 0) sm_top[wave] = top;
            __syncthreads();
#pragma unroll
            for (int w = 0; w < WPR; ++w) top = max(top, sm_top[w]);
        }
        if (top >= (DT == DT_F32 ? 0x7F800000u : DT == DT_BF16 ? 0x7F80u : 0x7C00u)) m = INFINITY;
        else m = DT == DT_F32 ? (double)__uint_as_float(top) : DT == DT_BF16 ? (double)bf16_to_f32((uint16_t)top) : (double)f16_to_f32((uint16_t)top);
    }
    const uint32_t m_high = __builtin_amdgcn_readfirstlane((uint32_t)(__builtin_bit_cast(uint64_t, m) >> 32));     // (all lanes' is the same)
    const bool bad = m_high == 0x7FF00000u, some = m_high != 0 && !bad;      // (a product of two floats that is not 0 is 2^-298 at least)
    const bool usual = m_high - 0x3C300000u <= 0x43B00000u - 0x3C300000u;    // 2^-60 .. 2^60
    const float mh = (float)m, rcp = __builtin_amdgcn_rcpf(mh), inv0 = 127.f * rcp, rest = fmaf(-mh, inv0, 127.f);
    const float inv = fmaf(NORM ? fmaf(-(float)(m - (double)mh), inv0, rest) : rest, rcp, inv0);
    constexpr float kWhole = 0x1.8p23f, kFar = 0.5f - (NORM ? 0x1.9p-16f : 0x1.1p-17f);              // the first as in q8_code
    const float least_far = usual ? kFar : some ? -1.f : INFINITY;
    int8_t* const to = a.codes + row * a.codes_stride;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        const int c = (v * WPR * 64 + t) * 8, at = min(c, a.N - 8);
        if (c >= a.N) continue;
        uint32_t w[2] = {0, 0};
        float sum[8];
        if (some || RES) {
            float n[8], d[8], far = 0;                       // the largest distance from a whole number; not a number where one is
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                sum[i] = x[v].get(i);
                if constexpr (RES) sum[i] += r[v].get(i);
                const float u = NORM ? sum[i] * g[v].get(i) : sum[i];
                n[i] = fmaf(u, inv, kWhole);
                d[i] = fabsf(fmaf(u, inv, kWhole - n[i]));
                far = __builtin_elementwise_maximum(far, d[i]);
            }
            static_for<0, 2>([&](auto hc) {
                constexpr int h = decltype(hc)::value * 4;
                auto bits = [&](int i) { return __float_as_uint(n[h + i]); };
                w[h / 4] = __builtin_amdgcn_perm(bits(1), bits(0), 0x0C0C0400u) | __builtin_amdgcn_perm(bits(3), bits(2), 0x04000C0Cu);
            });
            if (!(far <= least_far)) {
                uint32_t close = 0;
#pragma unroll
                for (int i = 0; i < 8; ++i) close |= !(d[i] <= least_far) ? 1u << i : 0u;
                double mm = m;
                asm volatile("" : "+v"(mm));                 // (what follows from it is for these elements only)
                do {
                    const int i = __ffs(close) - 1, shift = 8 * (i & 3);
                    close &= close - 1;
                    double u = (double)x[v].pick(i);
                    if constexpr (RES) u += (double)r[v].pick(i);
                    if constexpr (NORM) u *= (double)g[v].pick(i);
                    const uint32_t code = (q8_code(u, __builtin_amdgcn_rcp(mm), mm) & 255u) << shift, keep = ~(255u << shift);
                    if (i < 4) w[0] = (w[0] & keep) | code;
                    else w[1] = (w[1] & keep) | code;
                } while (close);
            }
            if (!some) w[0] = w[1] = 0;
        }
        if constexpr (RES) store_elems<RT, 8>(a.res_out, row * a.res_out_stride + at, sum);
        *reinterpret_cast<u32x2_a1*>(to + at) = u32x2_a1{w[0], w[1]};
    }
    if (t == 0) a.scales[row] = row_scale<NORM>(m, ss, bad, a.N, a.eps);
}

// Rows of any length (a wave for those below eight elements): read twice, the sum written the second time (it may go where the residual came from).
template <int DT, int RT, bool NORM>
__global__ __launch_bounds__(1024) void q8_long_rows_kernel(Q8Args a) {
    __shared__ double sm_m[16], sm_ss[16];
    __shared__ int sm_bad[16];
    const int64_t row = blockIdx.x;
    const int t = threadIdx.x;
    double h = 0;
    auto value = [&](int i) {
        float x = load_elem<DT>(a.x, row * a.x_stride + i);
        if constexpr (DT == DT_F32)
            for (int p = 1; p < a.n_part; ++p) x += ((const float*)a.x)[row * a.x_stride + i + p * a.part_stride];
        h = (double)x;
        if constexpr (RT != kNoResidual) h += (double)load_elem<RT>(a.res, row * a.res_stride + i);
        return NORM ? h * (double)a.gain[i] : h;
    };
    double m = 0, ss = 0, z = 0;
    for (int i = t; i < a.N; i += (int)blockDim.x) {
        const double u = value(i);
        m = fmax(m, fabs(u));
        ss = fma(h, h, ss);
        z = fma(u, 0.0, fma(h, 0.0, z));
    }
    m = wave_max(m);
    ss = wave_sum(ss);
    bool bad = __any(!(z == 0));
    if ((t & 63) == 0) { sm_m[t >> 6] = m; sm_ss[t >> 6] = ss; sm_bad[t >> 6] = bad; }
    __syncthreads();
    m = sm_m[0]; ss = sm_ss[0]; bad = sm_bad[0];
    for (int w = 1; w < (int)blockDim.x / 64; ++w) { m = fmax(m, sm_m[w]); ss += sm_ss[w]; bad |= (bool)sm_bad[w]; }
    const double rcp = m > 0 && !bad ? __builtin_amdgcn_rcp(m) : 0.0;
    for (int i = t; i < a.N; i += (int)blockDim.x) {
        const double u = value(i);
        a.codes[row * a.codes_stride + i] = rcp > 0 ? (int8_t)q8_code(u, rcp, m) : (int8_t)0;
        if constexpr (RT != kNoResidual) store_elem<RT>(a.res_out, row * a.res_out_stride + i, (float)h);
    }
    if (t == 0) a.scales[row] = row_scale<NORM>(m, ss, bad, a.N, a.eps);
}

// Eight elements a thread.
template <int DT>
__global__ __launch_bounds__(256) void q8_read_kernel(const int8_t* codes, int64_t codes_stride, const float* scales, int N, void* out, int64_t out_stride) {
    const int64_t row = blockIdx.x;
    const float s = scales[row];
    for (int64_t c = ((int64_t)blockIdx.y * blockDim.x + threadIdx.x) * 8; c < N; c += (int64_t)gridDim.y * blockDim.x * 8) {
        const int8_t* from = codes + row * codes_stride + c;
        const int left = (int)(N - c);
        union { u32x2_a1 v; int8_t b[8]; } q{};
        if (left >= 8) q.v = *reinterpret_cast<const u32x2_a1*>(from);
        else
#pragma unroll
            for (int i = 0; i < 8; ++i) if (i < left) q.b[i] = from[i];
        float x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = s * (float)q.b[i];
        store8<DT>(out, row * out_stride + c, left, x);
    }
}

template <int DT, int RT, bool NORM>
static void launch_rows(const Q8Args& a, hipStream_t stream) {
    const long pieces = (a.N + 7l) / 8;
    auto go = [&](auto wprc, auto nvc) {
        constexpr int WPR = decltype(wprc)::value, NV = decltype(nvc)::value;
        launch(q8_rows_kernel<DT, RT, NORM, WPR, NV>, dim3(WPR == 1 ? (a.M + 3) / 4 : a.M), dim3(WPR == 1 ? 256 : WPR * 64), stream, a);
    };
    using C1 = std::integral_constant<int, 1>;
    using C2 = std::integral_constant<int, 2>;
    using C4 = std::integral_constant<int, 4>;
    using C8 = std::integral_constant<int, 8>;
    using C16 = std::integral_constant<int, 16>;
    if (a.N < 8) launch(q8_long_rows_kernel<DT, RT, NORM>, dim3(a.M), dim3(64), stream, a);
    else if (pieces <= 64) go(C1{}, C1{});
    else if (pieces <= 256) go(C4{}, C1{});
    else if (pieces <= 1024 && a.M <= 256) go(C16{}, C1{});
    else if (pieces <= 512) go(C8{}, C1{});              // 704 rows of 4096 with a residual 7.7 us; four waves 7.9, two 9.8
    else if (pieces <= 1024) go(C8{}, C2{});
    else if (!NORM && pieces <= 1536 && a.M > 256) go(C8{}, std::integral_constant<int, NORM ? 2 : 3>{});
    else if (pieces <= 2048) go(C16{}, C2{});
    else if (!NORM && pieces <= 4096) go(C16{}, std::integral_constant<int, NORM ? 2 : 4>{});       // (the norm's rows would not fit the registers)
    else launch(q8_long_rows_kernel<DT, RT, NORM>, dim3(a.M), dim3(1024), stream, a);
}

int launch_q8(const Q8Args& a, int dtype, int res_dtype, hipStream_t stream) {
    auto with = [&](auto dt) {
        constexpr int DT = decltype(dt)::value;
        if (!a.gain) launch_rows<DT, kNoResidual, false>(a, stream);
        else if (res_dtype == kNoResidual) launch_rows<DT, kNoResidual, true>(a, stream);
        else if (res_dtype == DT_F32) launch_rows<DT, DT_F32, true>(a, stream);
        else launch_rows<DT, DT, true>(a, stream);   // (of x's type)
    };
    if (dtype == DT_F32) with(std::integral_constant<int, DT_F32>{});
    else if (dtype == DT_BF16) with(std::integral_constant<int, DT_BF16>{});
    else with(std::integral_constant<int, DT_F16>{});
    LASER_HIP_CHECK(hipGetLastError());
    return LASER_OK;
}

bool rows_apart(const void* a, int64_t a_row, int64_t a_step, const void* b, int64_t b_row, int64_t b_step, int64_t M) {
    const int64_t p = (int64_t)(uintptr_t)a, q = (int64_t)(uintptr_t)b;
    if (p + (M - 1) * a_step + a_row <= q || q + (M - 1) * b_step + b_row <= p) return true;
    if (a_step != b_step || a_step <= 0) return false;
    const int64_t d = ((q - p) % a_step + a_step) % a_step;          // columns of one matrix
    return d >= a_row && d + b_row <= a_step;
}

}  // namespace laser

using namespace laser;

static bool is_dtype(int t) { return t == LASER_F16 || t == LASER_BF16 || t == LASER_F32; }

static int check_rows(const void* x, int64_t x_stride, int M, int N, int dtype, const int8_t* codes, int64_t codes_stride, const float* scales) {
    LASER_REQUIRE(is_dtype(dtype), LASER_E_INVALID_ARG, "dtype %d: LASER_F16, LASER_BF16 or LASER_F32", dtype);
    LASER_REQUIRE(M >= 0 && M <= kQ8MaxRows, LASER_E_INVALID_ARG, "M %d out of range", M);
    LASER_REQUIRE(N > 0 && N <= (1 << 30), LASER_E_INVALID_ARG, "N %d out of range", N);
    LASER_REQUIRE(x_stride >= 0 && x_stride < (1ll << 36), LASER_E_INVALID_ARG, "x_stride %lld out of range", (long long)x_stride);
    LASER_REQUIRE(codes_stride >= N && codes_stride < (1ll << 36), LASER_E_INVALID_ARG, "rows of codes overlap: stride %lld", (long long)codes_stride);
    if (M == 0) return LASER_OK;
    LASER_REQUIRE(x && codes && scales, LASER_E_INVALID_ARG, "NULL argument");
    LASER_REQUIRE((uintptr_t)x % dtype_bytes(dtype) == 0 && (uintptr_t)scales % 4 == 0, LASER_E_INVALID_ARG, "x or scales is not aligned to its elements");
    const int64_t e = (int64_t)dtype_bytes(dtype);
    LASER_REQUIRE(rows_apart(x, N * e, x_stride * e, codes, N, codes_stride, M), LASER_E_INVALID_ARG, "codes overlap x");
    LASER_REQUIRE(rows_apart(scales, 4, 4, codes, N, codes_stride, M) && rows_apart(scales, 4, 4, x, N * e, x_stride * e, M), LASER_E_INVALID_ARG, "scales overlap x or codes");
    return LASER_OK;
}

extern "C" int laser_q8_rows(const void* x, int64_t x_stride, int M, int N, int dtype, int8_t* codes, int64_t codes_stride, float* scales, void* stream) {
    if (const int rc = check_rows(x, x_stride, M, N, dtype, codes, codes_stride, scales)) return rc;
    if (M == 0) return LASER_OK;
    Q8Args a{};
    a.x = x; a.x_stride = x_stride; a.n_part = 1;
    a.codes = codes; a.codes_stride = codes_stride; a.scales = scales;
    a.M = M; a.N = N;
    return launch_q8(a, dtype, kNoResidual, (hipStream_t)stream);
}

extern "C" int laser_q8_norm(const void* x, int64_t x_stride, int dtype, const void* res, int64_t res_stride, void* res_out, int64_t res_out_stride, int res_dtype,
                             const float* gain, float eps, int M, int N, int8_t* codes, int64_t codes_stride, float* scales, void* stream) {
    if (const int rc = check_rows(x, x_stride, M, N, dtype, codes, codes_stride, scales)) return rc;
    LASER_REQUIRE(eps >= 0 && eps <= 1e30f, LASER_E_INVALID_ARG, "eps %g out of range", (double)eps);
    LASER_REQUIRE((res == nullptr) == (res_out == nullptr), LASER_E_INVALID_ARG, "res and res_out go together");
    if (res) {
        LASER_REQUIRE(res_dtype == dtype || res_dtype == LASER_F32, LASER_E_INVALID_ARG, "res_dtype %d: x's type or LASER_F32", res_dtype);
        LASER_REQUIRE(res_stride >= 0 && res_stride < (1ll << 36), LASER_E_INVALID_ARG, "res_stride %lld out of range", (long long)res_stride);
        LASER_REQUIRE(res_out_stride >= N && res_out_stride < (1ll << 36), LASER_E_INVALID_ARG, "rows of res_out overlap: stride %lld", (long long)res_out_stride);
    }
    if (M == 0) return LASER_OK;
    LASER_REQUIRE(gain != nullptr, LASER_E_INVALID_ARG, "gain is NULL");
    LASER_REQUIRE((uintptr_t)gain % 4 == 0, LASER_E_INVALID_ARG, "gain is not aligned to its elements");
    LASER_REQUIRE(rows_apart(gain, 4ll * N, 0, codes, N, codes_stride, M) && rows_apart(gain, 4ll * N, 0, scales, 4, 4, M), LASER_E_INVALID_ARG, "codes or scales overlap gain");
    if (res) {
        const int64_t e = (int64_t)dtype_bytes(dtype), f = (int64_t)dtype_bytes(res_dtype);
        LASER_REQUIRE((uintptr_t)res % f == 0 && (uintptr_t)res_out % f == 0, LASER_E_INVALID_ARG, "res or res_out is not aligned to its elements");
        auto away = [&](const void* p, int64_t row, int64_t step) { return rows_apart(res_out, N * f, res_out_stride * f, p, row, step, M); };
        LASER_REQUIRE((res == res_out && res_stride == res_out_stride) || away(res, N * f, res_stride * f), LASER_E_INVALID_ARG, "res_out overlaps res and is not res itself");
        LASER_REQUIRE((x == res_out && x_stride == res_out_stride && dtype == res_dtype) || away(x, N * e, x_stride * e), LASER_E_INVALID_ARG, "res_out overlaps x and is not x itself");
        LASER_REQUIRE(away(codes, N, codes_stride) && away(scales, 4, 4) && away(gain, 4ll * N, 0), LASER_E_INVALID_ARG, "res_out overlaps codes, scales or gain");
        LASER_REQUIRE(rows_apart(res, N * f, res_stride * f, codes, N, codes_stride, M) && rows_apart(res, N * f, res_stride * f, scales, 4, 4, M), LASER_E_INVALID_ARG,
                      "codes or scales overlap res");
    }
    Q8Args a{};
    a.x = x; a.x_stride = x_stride; a.n_part = 1;
    a.res = res; a.res_stride = res_stride; a.res_out = res_out; a.res_out_stride = res_out_stride;
    a.gain = gain; a.eps = eps;
    a.codes = codes; a.codes_stride = codes_stride; a.scales = scales;
    a.M = M; a.N = N;
    return launch_q8(a, dtype, res ? res_dtype : kNoResidual, (hipStream_t)stream);
}

extern "C" int laser_q8_read(const int8_t* codes, int64_t codes_stride, const float* scales, int M, int N, int dtype, void* out, int64_t out_stride, void* stream) {
    LASER_REQUIRE(is_dtype(dtype), LASER_E_INVALID_ARG, "dtype %d: LASER_F16, LASER_BF16 or LASER_F32", dtype);
    LASER_REQUIRE(M >= 0 && M <= kQ8MaxRows, LASER_E_INVALID_ARG, "M %d out of range", M);
    LASER_REQUIRE(N > 0 && N <= (1 << 30), LASER_E_INVALID_ARG, "N %d out of range", N);
    LASER_REQUIRE(codes_stride >= 0 && codes_stride < (1ll << 36), LASER_E_INVALID_ARG, "codes_stride %lld out of range", (long long)codes_stride);
    LASER_REQUIRE(out_stride >= N && out_stride < (1ll << 36), LASER_E_INVALID_ARG, "rows of out overlap: stride %lld", (long long)out_stride);
    if (M == 0) return LASER_OK;
    LASER_REQUIRE(codes && scales && out, LASER_E_INVALID_ARG, "NULL argument");
    const int64_t e = (int64_t)dtype_bytes(dtype);
    LASER_REQUIRE((uintptr_t)out % e == 0 && (uintptr_t)scales % 4 == 0, LASER_E_INVALID_ARG, "out or scales is not aligned to its elements");
    LASER_REQUIRE(rows_apart(out, N * e, out_stride * e, codes, N, codes_stride, M) && rows_apart(out, N * e, out_stride * e, scales, 4, 4, M), LASER_E_INVALID_ARG,
                  "out overlaps codes or scales");
    const long pieces = (N + 7l) / 8;
    const dim3 block(pieces <= 64 ? 64 : pieces <= 128 ? 128 : 256), grid(M, (unsigned)std::min((pieces + block.x - 1) / block.x, 1024l));
    const auto kernel = dtype == LASER_F32 ? q8_read_kernel<DT_F32> : dtype == LASER_BF16 ? q8_read_kernel<DT_BF16> : q8_read_kernel<DT_F16>;
    launch(kernel, grid, block, (hipStream_t)stream, codes, codes_stride, scales, N, out, out_stride);
    LASER_HIP_CHECK(hipGetLastError());
    return LASER_OK;
}
