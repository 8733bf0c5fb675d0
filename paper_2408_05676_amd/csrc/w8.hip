// Products of rows in 8-bit codes with 8-bit weights: out[M][outs] = s_x[row] s_w[output] sum c_x c_w, plain or gated (silu(gate) up).
#include <algorithm>
#include <cmath>
#include <memory>
#include <new>

#include "w8_few.h"

namespace laser {

// Row of the handle's layout -> output of the caller's matrix, or -1.
__device__ inline int w8_source(int row, int N, int gated) {
    if (!gated) return row < N ? row : -1;
    const int f = (row >> 5) * 16 + (row & 15), F = N / 2;
    return f < F ? f + (row & 16 ? F : 0) : -1;
}

// A thread per 16 bytes: an output and 16 of its inputs. Inputs beyond Kd and rows beyond N are zeros.
__global__ __launch_bounds__(256) void w8_layout_kernel(const int8_t* codes, const float* scales, int N, int Kd, int gated, int rows, int Kp, uint8_t* out, float* out_scales) {
    const size_t i = (size_t)blockIdx.x * 256 + threadIdx.x, frag = i >> 6;
    const int tiles = rows / 16, row = (int)(frag % tiles) * 16 + (int)(i & 15), k = (int)(frag / tiles) * 64 + 16 * (int)(i >> 4 & 3);
    if (k >= Kp) return;
    const int n = w8_source(row, N, gated);
    union { u32x4 v; int8_t b[16]; } t;
#pragma unroll
    for (int j = 0; j < 16; ++j) t.b[j] = n >= 0 && k + j < Kd ? codes[(size_t)n * Kd + k + j] : (int8_t)0;
    reinterpret_cast<u32x4*>(out)[i] = t.v;
    if (k == 0) out_scales[row] = n >= 0 ? scales[n] : 0.f;
}

// Which kernel a launch takes: 0 .. kW8FewN - 1 of w8_few.h, beyond of w8_tile.h.
//
// Up to 16 rows: one output fragment and eight waves where that is at most a workgroup for each of 256 compute units, else two and four (6144 outputs of 2048
// inputs, one row 5.0 us, the other way 5.9; 4096 x 4096 6.1 and 6.2; 4096 x 11008 10.3 and 12.5).
// More rows: the least of the microseconds below, which grow with the workgroups of a compute unit and their stages. Fitted by least squares to what every kernel within
// 1.25 of the fastest took, at 17 to 1000 rows of ten matrices (256 x 768 to 4096 x 2 x 11008) and of 400 random ones: 2600 measurements. What it takes is 0.5 % slower
// than the fastest on average at the ten, 0.8 % at the random ones, 21 % at worst (520 rows 3712 -> 238: 6.7 us of 5.5). Epilogues of tiles that leave a compute unit to one
// workgroup, by their registers, stand behind nothing else's products.
static int w8_pick(const W8Args& a, bool gated) {
    constexpr int cus = 256;
    const int frags = a.rows / 16;
    const double k = a.Kp / 1024.0, weights = 1e-6 * a.rows * a.Kp, results = 2e-6 * a.M * a.outs;
    auto up = [](long a, long b) { return (a + b - 1) / b; };
    if (a.M <= 16) return (a.M <= 4 ? 0 : 2) + (gated || frags > cus);
    int best = 0;
    double least = 1e300;
    for (int v = 0; v < kW8FewN; ++v) {
        const W8Few f = kW8Few[v];
        if (f.mt == 0 || (gated && f.nt % 2)) continue;
        const long units = up(frags, f.nt) * up(a.M, 16 * f.mt);
        if (units * 64 * f.wk >= (1l << 32)) continue;           // (a launch's threads)
        const double each = (double)up(units, cus);
        const double us = 3.07 + each * (k * (0.141 * f.nt + 0.169 * f.mt) + 0.052 + 0.0914 * f.nt * f.mt) + 0.0979 * weights + 0.568 * results;
        if (us < least) { least = us; best = v; }
    }
    for (int v = 0; v < kW8ShapeN; ++v) {
        const W8Shape s = kW8Shapes[v];
        const double each = (double)up(up(a.M, s.wm * 16) * up(a.rows, s.wn * 64), cus);
        const double end = s.wm * s.wn >= 32 ? (gated ? 0.103 : 0.0838) : gated ? 0.0616 : 0.0547;
        const double us = 3.3 + each * (k * (0.071 * s.wm * s.wn + 0.109 * s.wm + 0.352 * s.wn) + end * s.wm * s.wn) + 0.466 * k + 0.0877 * weights + 0.328 * results;
        if (us < least) { least = us; best = kW8FewN + v; }
    }
    return best;
}

int launch_w8(const W8* w, const int8_t* x, int64_t x_stride, const float* x_scales, int M, int dtype, void* out, int64_t out_stride, hipStream_t stream) {
    LASER_REQUIRE((long)(w->rows / 16) * ((M + 15) / 16) < (1l << 25), LASER_E_LIMIT, "%d rows times %d outputs are too many for a launch", M, w->rows);
    const W8Args a{w->codes, w->scales, x, x_scales, out, x_stride, out_stride, M, w->outs, w->rows, w->Kd, w->Kp, dtype, 0, 0};
    const int v = w->far ? -1 : w8_pick(a, w->gated);
    if (v < 0) launch_w8_far(a, w->gated, stream);
    else if (v < kW8FewN) launch_w8_few(a, w->gated, v, stream);
    else if (w->gated) launch_w8_tile_gated(a, v - kW8FewN, stream);
    else launch_w8_tile_plain(a, v - kW8FewN, stream);
    LASER_HIP_CHECK(hipGetLastError());
    return LASER_OK;
}

}  // namespace laser

using namespace laser;

static int check_w8(int N, int Kd) {
    LASER_REQUIRE(N > 0 && Kd > 0, LASER_E_INVALID_ARG, "N and Kd must be positive");
    LASER_REQUIRE(Kd <= kQ8MaxK, LASER_E_LIMIT, "Kd %d: sums of more than %d products may pass 32 bits", Kd, kQ8MaxK);
    LASER_REQUIRE(N <= (1 << 25) && ((long)N + 15) / 16 * (((long)Kd + 127) / 128) < (1l << 23), LASER_E_LIMIT, "matrix too large");   // (offsets of 32 bits; a launch has less than 2^32 threads)
    return LASER_OK;
}

extern "C" int laser_w8_create(const int8_t* codes, const float* scales, int N, int Kd, int gated, void* stream, laser_w8** out) {
    LASER_REQUIRE(codes && scales && out, LASER_E_INVALID_ARG, "NULL argument");
    if (const int rc = check_w8(N, Kd)) return rc;
    LASER_REQUIRE(gated == 0 || gated == 1, LASER_E_INVALID_ARG, "gated must be 0 or 1");
    LASER_REQUIRE(!gated || N % 2 == 0, LASER_E_SHAPE, "a gated matrix has as many up as gate outputs: N %d is odd", N);
    LASER_REQUIRE((uintptr_t)scales % 4 == 0, LASER_E_INVALID_ARG, "scales are not aligned to their elements");
    const int outs = gated ? N / 2 : N, rows = (outs + 15) / 16 * 16 * (gated ? 2 : 1), Kp = (Kd + 255) / 256 * 256;
    W8* w = new W8{N, Kd, gated, outs, rows, Kp, nullptr, nullptr, 0};
    const size_t bytes = (size_t)rows * Kp;
    auto fail = [&](hipError_t e, const char* what) {
        set_error("%s: %s", what, hipGetErrorString(e));
        laser_w8_destroy(reinterpret_cast<laser_w8*>(w));
        return LASER_E_HIP;
    };
    hipError_t e = hipMalloc((void**)&w->codes, bytes + (size_t)rows * 4);
    if (e != hipSuccess) return fail(e, "hipMalloc");
    w->scales = reinterpret_cast<float*>(w->codes + bytes);
    hipLaunchKernelGGL(w8_layout_kernel, dim3((unsigned)((bytes / 16 + 255) / 256)), dim3(256), 0, (hipStream_t)stream, codes, scales, N, Kd, gated, rows, Kp, w->codes, w->scales);
    if ((e = hipGetLastError()) != hipSuccess) return fail(e, "w8_layout_kernel");
    const std::unique_ptr<float[]> held(new (std::nothrow) float[rows]);
    if (!held) return fail(hipErrorOutOfMemory, "memory for the scales");
    if ((e = hipMemcpyAsync(held.get(), w->scales, (size_t)rows * 4, hipMemcpyDeviceToHost, (hipStream_t)stream)) != hipSuccess) return fail(e, "hipMemcpyAsync");
    if ((e = hipStreamSynchronize((hipStream_t)stream)) != hipSuccess) return fail(e, "hipStreamSynchronize");
    for (int i = 0; i < rows; ++i) {
        const float s = std::fabs(held[i]);
        w->far |= std::isfinite(s) && s != 0 && (s < 0x1p-126f || s >= 0x1p97f);
    }
    *out = reinterpret_cast<laser_w8*>(w);
    return LASER_OK;
}

extern "C" int laser_w8_destroy(laser_w8* h) {
    W8* w = reinterpret_cast<W8*>(h);
    if (!w) return LASER_OK;
    if (w->codes) (void)hipFree(w->codes);
    delete w;
    return LASER_OK;
}

extern "C" int laser_w8_quantize(const uint16_t* w, int N, int Kd, int8_t* codes, float* scales, void* stream) {
    LASER_REQUIRE(w && codes && scales, LASER_E_INVALID_ARG, "NULL argument");
    if (const int rc = check_w8(N, Kd)) return rc;
    for (int n = 0; n < N; n += kQ8MaxRows)          // (a launch's rows)
        if (const int rc = laser_q8_rows(w + (size_t)n * Kd, Kd, std::min(N - n, kQ8MaxRows), Kd, LASER_BF16, codes + (size_t)n * Kd, Kd, scales + n, stream)) return rc;
    return LASER_OK;
}

extern "C" int laser_w8_matmul(const laser_w8* h, const int8_t* x, int64_t x_stride, const float* x_scales, int M, int dtype, void* out, int64_t out_stride, void* stream) {
    const W8* w = reinterpret_cast<const W8*>(h);
    LASER_REQUIRE(w != nullptr, LASER_E_INVALID_ARG, "w is NULL");
    LASER_REQUIRE(dtype == LASER_F16 || dtype == LASER_BF16 || dtype == LASER_F32, LASER_E_INVALID_ARG, "dtype %d: LASER_F16, LASER_BF16 or LASER_F32", dtype);
    LASER_REQUIRE(M >= 0 && M <= kQ8MaxRows, LASER_E_INVALID_ARG, "M %d out of range", M);
    LASER_REQUIRE(x_stride % kQ8Pad == 0 && x_stride >= w->Kd && x_stride < (1ll << 22), LASER_E_INVALID_ARG, "x_stride %lld: a multiple of %d below 2^22, at least %d", (long long)x_stride, kQ8Pad, w->Kd);
    LASER_REQUIRE(out_stride >= w->outs && out_stride < (1ll << 32), LASER_E_INVALID_ARG, "rows of out overlap: stride %lld", (long long)out_stride);
    if (M == 0) return LASER_OK;
    LASER_REQUIRE(x && x_scales && out, LASER_E_INVALID_ARG, "NULL argument");
    const int64_t e = (int64_t)dtype_bytes(dtype);
    LASER_REQUIRE((uintptr_t)x % 16 == 0, LASER_E_INVALID_ARG, "x is not aligned to 16 bytes");
    LASER_REQUIRE((uintptr_t)out % e == 0 && (uintptr_t)x_scales % 4 == 0, LASER_E_INVALID_ARG, "out or x_scales is not aligned to its elements");
    LASER_REQUIRE(rows_apart(out, w->outs * e, out_stride * e, x, (w->Kd + kQ8Pad - 1) / kQ8Pad * kQ8Pad, x_stride, M) && rows_apart(out, w->outs * e, out_stride * e, x_scales, 4, 4, M), LASER_E_INVALID_ARG,
                  "out overlaps x or x_scales");
    return launch_w8(w, x, x_stride, x_scales, M, dtype, out, out_stride, (hipStream_t)stream);
}
