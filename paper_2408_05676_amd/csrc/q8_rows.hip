// Rows into 8-bit codes with one scale each, alone or behind the residual's addition and the root-mean-square norm, and back.
//
// h = x + res, u = h gain (u = x without the norm), m = max |u|: codes c = rint(127 u / m) and scale s = m / 127 / sqrt(mean h^2 + eps).
// The root is the same for a row's elements, so codes need the extremes of h gain only. All in 64 bits, where x + res and the
// products are exact: a code is the formula's whatever the order of operations, and squares of any fp32 rows have room. t = u (127 / m) is
// off by some 2^-46; only where it is closer than 2^-30 to a half is the quotient itself taken.
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

struct RowStats { double m, ss, bad; };              // largest |u|, sum of h^2, not 0 (NaN) if some u is not finite

__device__ inline RowStats wave_stats(RowStats s) {
#pragma unroll
    for (int o = 1; o < 64; o *= 2) {
        s.m = fmax(s.m, __shfl_xor(s.m, o));
        s.ss += __shfl_xor(s.ss, o);
        s.bad += __shfl_xor(s.bad, o);
    }
    return s;
}

__device__ inline int q8_code(double u, double inv, double m) {
    const double t = u * inv;
    double c = rint(t);
    if (fabs(t - c) > 0.5 - 0x1p-30) c = rint(127.0 * u / m);
    return (int)c;
}

template <int DT, int RT>
__global__ __launch_bounds__(256) void q8_rows_kernel(Q8Args a) {
    __shared__ RowStats sm[4];
    const int64_t row = blockIdx.x;
    const int t = threadIdx.x;
    double h = 0;
    auto value = [&](int i) {                        // u of column i; h on the side
        h = (double)load_elem<DT>(a.x, row * a.x_stride + i);
        if constexpr (DT == DT_F32)
            for (int p = 1; p < a.n_part; ++p) h += (double)((const float*)a.x)[row * a.x_stride + i + p * a.part_stride];
        if constexpr (RT != kNoResidual) h += (double)load_elem<RT>(a.res, row * a.res_stride + i);
        return a.gain ? h * (double)a.gain[i] : h;
    };
    RowStats s{0, 0, 0};
    for (int i = t; i < a.N; i += 256) {
        const double u = value(i);
        s.m = fmax(s.m, fabs(u));
        s.ss = fma(h, h, s.ss);
        s.bad = fma(u, 0.0, s.bad);
    }
    s = wave_stats(s);
    if ((t & 63) == 0) sm[t >> 6] = s;
    __syncthreads();
    s = sm[0];
    for (int w = 1; w < 4; ++w) { s.m = fmax(s.m, sm[w].m); s.ss += sm[w].ss; s.bad += sm[w].bad; }
    const bool bad = !(s.bad == 0) || !__builtin_isfinite(s.ss);
    const double inv = s.m > 0 && !bad ? 127.0 / s.m : 0.0;
    for (int i = t; i < a.N; i += 256) {
        const double u = value(i);
        a.codes[row * a.codes_stride + i] = inv > 0 ? (int8_t)q8_code(u, inv, s.m) : (int8_t)0;
        if constexpr (RT != kNoResidual) store_elem<RT>(a.res_out, row * a.res_out_stride + i, (float)h);
    }
    if (t == 0) {
        double scale = s.m / 127.0;
        if (a.gain && s.m > 0) scale /= sqrt(s.ss / a.N + (double)a.eps);
        a.scales[row] = bad ? __builtin_nanf("") : (float)scale;
    }
}

template <int DT>
__global__ __launch_bounds__(256) void q8_read_kernel(const int8_t* codes, int64_t codes_stride, const float* scales, int N, void* out, int64_t out_stride) {
    const int64_t row = blockIdx.x;
    const float s = scales[row];
    for (int i = threadIdx.x; i < N; i += 256) store_elem<DT>(out, row * out_stride + i, s * (float)codes[row * codes_stride + i]);
}

int launch_q8(const Q8Args& a, int dtype, int res_dtype, hipStream_t stream) {
    auto go = [&](auto dt, auto rt) {
        hipLaunchKernelGGL((q8_rows_kernel<decltype(dt)::value, decltype(rt)::value>), dim3(a.M), dim3(256), 0, stream, a);
    };
    auto with = [&](auto dt) {
        using F32 = std::integral_constant<int, DT_F32>;
        if (res_dtype == kNoResidual) go(dt, std::integral_constant<int, kNoResidual>{});
        else if (res_dtype == DT_F32) go(dt, F32{});
        else go(dt, dt);                             // (of x's type)
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
    hipStream_t s = (hipStream_t)stream;
    if (dtype == LASER_F32) hipLaunchKernelGGL(q8_read_kernel<DT_F32>, dim3(M), dim3(256), 0, s, codes, codes_stride, scales, N, out, out_stride);
    else if (dtype == LASER_BF16) hipLaunchKernelGGL(q8_read_kernel<DT_BF16>, dim3(M), dim3(256), 0, s, codes, codes_stride, scales, N, out, out_stride);
    else hipLaunchKernelGGL(q8_read_kernel<DT_F16>, dim3(M), dim3(256), 0, s, codes, codes_stride, scales, N, out, out_stride);
    LASER_HIP_CHECK(hipGetLastError());
    return LASER_OK;
}
