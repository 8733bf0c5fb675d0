// Products of rows with 4-bit weights: out[M][N] = x[M][Kd] W^T, W[n][i] = m + s c of its group (laser.h).
//
// A handle keeps, for every tile of 16 outputs, blocks of 128 inputs one after the other: 1 KB of codes as the 64 lanes of a wave
// hold a matrix operand (lane (r = lane % 16, g = lane / 16): output r, inputs 32 c + 8 g .. + 7 in word c) and the 16 x (128 / group)
// scales and offsets. A wave streams the blocks of its tiles over its share of the inputs; per group
//   D = sum c x (matrix instructions on the bare codes), X = sum x (one more, with ones), acc += s D + m X in fp32.
// Codes enter as 16-bit floats: for fp16 rows a code masked out of its word is the subnormal c 2^-20 (in bits 0..3, as c 2^-24, an activation 3000 times
// the others' cost their sum three times the error of fp32 sums: four_bit.h), for bf16 rows it is put under the exponent of 128
// and stands for 128 + c, which the offset m - 128 s takes back.
// Bound (calls one after the other in a captured graph, bf16, group 128): up to four rows the weights' way from memory (4096 -> 22016, one row: 48 MB in
// 12.0 us, 4.0 TB/s where a long read reaches 5.5); with more rows theirs as well, from L2 once a workgroup (9 rows 12.7 us, 11008 -> 4096 9.3 us); from 17
// rows on the matrix and vector instructions of the waves that fit (72 rows 2048 -> 6144 10.1 us, 4096 -> 22016 36 us, 0.36 PFLOP/s).
// Groups of 64 and 32 have two and four times the scales to apply: 72 rows 4096 -> 22016 41 and 48 us, 704 rows 256 and 339 (group 128 226).
// Staging a block's rows in LDS for four waves, behind a barrier a block, was slower at every size (72 rows 2048 -> 6144 17.8 us).
#include <algorithm>
#include <vector>

#include "four_bit.h"

namespace laser {

constexpr int block_bytes(int ng) { return 1024 + 64 * ng; }      // ng = groups of a block

// ------------------------------------------------------------------------------------------------
// A thread per word of codes, and the first 16 ng of a block for its scales and offsets. Outputs and inputs beyond the matrix are zeros.
__global__ __launch_bounds__(256) void w4_layout_kernel(const uint8_t* codes, const uint16_t* scales, const uint16_t* offsets, int N, int Kd, int group,
                                                        int nkb, uint8_t* blocks) {
    const size_t blk = blockIdx.x;
    const int tile = (int)(blk / nkb), kb = (int)(blk % nkb), ng = 128 / group, t = threadIdx.x;
    uint8_t* out = blocks + blk * block_bytes(ng);
    {
        const int lane = t >> 2, c = t & 3, n = tile * 16 + (lane & 15), i = kb * 128 + 32 * c + 8 * (lane >> 4);
        uint32_t w = 0;
        if (n < N && i < Kd)
#pragma unroll
            for (int j = 0; j < 8; ++j) {                         // element j: bits 4 (j / 2) of half j % 2
                const uint32_t byte = codes[((size_t)n * Kd + i + j) >> 1];
                w |= ((j & 1 ? byte >> 4 : byte) & 15u) << (4 * (j >> 1) + 16 * (j & 1));
            }
        reinterpret_cast<uint32_t*>(out)[t] = w;
    }
    if (t < 16 * ng) {
        const int n = tile * 16 + t / ng, gi = kb * ng + t % ng, per = Kd / group;
        uint32_t sm = 0;
        if (n < N && gi < per) sm = (uint32_t)scales[(size_t)n * per + gi] | ((uint32_t)offsets[(size_t)n * per + gi] << 16);
        reinterpret_cast<uint32_t*>(out + 1024)[t] = sm;
    }
}

// Eight threads per group of a bf16 matrix. A group with a weight that is not finite: offset NaN, scale and codes 0.
__global__ __launch_bounds__(256) void w4_quantize_kernel(const uint16_t* w, size_t groups, int group, uint8_t* codes, uint16_t* scales, uint16_t* offsets) {
    const size_t i = ((size_t)blockIdx.x * 256 + threadIdx.x) >> 3;
    const int lane = threadIdx.x & 7, per = group / 8;            // elements a thread takes: 4, 8 or 16
    if (i >= groups) return;                                      // (eight lanes together)
    const uint16_t* p = w + i * group + lane * per;
    float lo = INFINITY, hi = -INFINITY;
    int bad = 0;
    for (int j = 0; j < per; ++j) { const float x = bf16_to_f32(p[j]); lo = fminf(lo, x); hi = fmaxf(hi, x); bad |= !__builtin_isfinite(x); }
#pragma unroll
    for (int o = 1; o < 8; o *= 2) { lo = fminf(lo, __shfl_xor(lo, o)); hi = fmaxf(hi, __shfl_xor(hi, o)); bad |= __shfl_xor(bad, o); }
    if (bad) lo = hi = 0.f;
    const _Float16 s = f64_to_f16(fmin(((double)hi - (double)lo) / 15.0, 65504.0)), m = (_Float16)fminf(fmaxf(lo, -65504.f), 65504.f);
    auto code = [&](uint16_t h) {
        const double n = rint(((double)bf16_to_f32(h) - (double)(float)m) / (double)(float)s);
        return (float)s > 0.f && !bad ? (uint32_t)fmin(fmax(n, 0.0), 15.0) : 0u;
    };
    uint8_t* q = codes + (i * group + lane * per) / 2;
    for (int j = 0; j < per; j += 2) q[j / 2] = (uint8_t)(code(p[j]) | (code(p[j + 1]) << 4));
    if (lane == 0) { scales[i] = __builtin_bit_cast(uint16_t, s); offsets[i] = bad ? 0x7E00 : __builtin_bit_cast(uint16_t, m); }
}

// ------------------------------------------------------------------------------------------------
struct W4Args {
    const uint8_t* blocks;
    const uint16_t* x; void* out;
    int64_t x_stride, out_stride;
    int M, N, Kd, nkb, tiles;                                      // W4_SWIGLU: N and tiles of a half
    int epi, up_tile;                                              // the first tile of the up half, W4_SWIGLU only
};

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
template <bool BF>
__device__ inline float4_t mfma_x(const Frag8& a, const Frag8& b, float4_t c) {
    if constexpr (BF) return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a.v4), __builtin_bit_cast(bf16x8_t, b.v4), c, 0, 0, 0);
    else return mfma_16x16x32(a, b, c);
}

// BF: bf16 rows (else fp16). NG: groups of a block. SWAP: more than four rows. MT: 16-row tiles. NT: 16-output tiles of a wave. WK: waves that share the inputs.
// Weights are requested two blocks ahead, rows XD pieces of 32 inputs ahead, two pieces (whole lines of memory) together.
template <bool BF, int NG, bool SWAP, int MT, int NT, int WK>
__global__ __launch_bounds__(WK * 64) void w4_matmul_kernel(W4Args a) {
    constexpr int WD = 2;
    constexpr int XD = MT == 1 ? 8 : 4;
    constexpr int CPG = 4 / NG;                                    // pieces of a group
    extern __shared__ float lds[];                                 // [WK / 2][NT][MT][16 rows][16 outputs]
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
    // A wave's tiles side by side; W4_SWIGLU: half of them gate, the other half their up tiles (NT is even then).
    const bool swiglu = NT > 1 && a.epi == W4_SWIGLU;
    const int own = swiglu ? NT / 2 : NT, tile0 = blockIdx.x * own, row0 = blockIdx.y * (MT * 16);
    const int k0 = (int)((long)a.nkb * wave / WK), k1 = (int)((long)a.nkb * (wave + 1) / WK);
    const uint8_t* wp[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) wp[n] = a.blocks + (size_t)(n < own ? min(tile0 + n, a.tiles - 1) : a.up_tile + min(tile0 + n - own, a.tiles - 1)) * a.nkb * block_bytes(NG);
    const uint16_t* xp[MT];
#pragma unroll
    for (int m = 0; m < MT; ++m) xp[m] = a.x + (size_t)min(row0 + m * 16 + (SWAP ? lane >> 2 : r), a.M - 1) * a.x_stride + 8 * (SWAP ? lane & 3 : g);
    // lane r of a row of sixteen keeps the scale of output 4 g + r / NG, group r % NG
    const int sm_at = 1024 + 4 * (4 * g * NG + (lane & (4 * NG - 1)));

    // More than four rows are requested four lanes to a row, so that lanes side by side share lines of memory, and change places on their way to
    // the operand: lane (r, g) takes what lane 4 r + g loaded. Requested as operands, sixteen rows side by side, they took 68 clocks a request:
    // 72 rows x 11008 x 4096 49 us, so 28; 9 rows x 4096 x 22016 14.0 and 13.0. Up to four rows lanes share lines anyway, and changing places costs
    // more than it gains (one row x 11008 x 4096 8.0 us, so 9.3).
    const int from = 4 * (4 * r + g);
    u32x4 wq[WD][NT];
    uint32_t smq[WD][NT];
    Frag8 xq[XD][MT];
    auto load_w = [&](auto slot, int kb) {
        constexpr int s = decltype(slot)::value;
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const uint8_t* p = wp[n] + (size_t)min(kb, k1 - 1) * block_bytes(NG);
            wq[s][n] = *reinterpret_cast<const u32x4*>(p + lane * 16);
            smq[s][n] = *reinterpret_cast<const uint32_t*>(p + sm_at);
        }
    };
    const int last = min(k1 * 4, a.Kd / 32) - 1;                                // (past the last input, in a padded block: codes, scales and offsets are zero)
    auto load_x = [&](auto slot, int piece) {                      // pieces `piece`, `piece` + 1
        constexpr int s = decltype(slot)::value;
        const int i = min(piece, last) * 32, j = min(piece + 1, last) * 32;
#pragma unroll
        for (int m = 0; m < MT; ++m) {
            xq[s][m].v4 = *reinterpret_cast<const u32x4_a2*>(xp[m] + i);
            xq[s + 1][m].v4 = *reinterpret_cast<const u32x4_a2*>(xp[m] + j);
        }
    };
    Frag8 ones;
#pragma unroll
    for (int i = 0; i < 4; ++i) ones.w[i] = BF ? 0x3F803F80u : 0x3C003C00u;

    float4_t acc[NT][MT];
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int m = 0; m < MT; ++m) acc[n][m] = float4_t{0.f, 0.f, 0.f, 0.f};

    if (k0 < k1) {
        static_for<0, XD / 2>([&](auto s) { load_x(std::integral_constant<int, 2 * decltype(s)::value>{}, 4 * k0 + 2 * decltype(s)::value); });
        static_for<0, WD>([&](auto s) { load_w(s, k0 + decltype(s)::value); });
        for (int kb0 = k0; kb0 < k1; kb0 += WD)
            static_for<0, WD>([&](auto ws) {
                constexpr int s = decltype(ws)::value;
                const int kb = kb0 + s;
                if (kb < k1) {
                    float ss[NT], mm[NT];
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        const float sc = sm_scale(smq[s][n]);
                        ss[n] = BF ? sc : sc * (kCodeUnit / 16.f);
                        mm[n] = BF ? fmaf(-128.f, sc, sm_offset(smq[s][n])) : sm_offset(smq[s][n]);
                    }
                    static_for<0, NG>([&](auto gg) {
                        constexpr int gi = decltype(gg)::value;
                        float4_t X[MT], D[NT][MT];
#pragma unroll
                        for (int m = 0; m < MT; ++m) {
                            X[m] = float4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                            for (int n = 0; n < NT; ++n) D[n][m] = float4_t{0.f, 0.f, 0.f, 0.f};
                        }
                        static_for<0, CPG>([&](auto pc) {
                            constexpr int c = gi * CPG + decltype(pc)::value, xs = (s * 4 + c) % XD;
                            Frag8 xf[MT];
#pragma unroll
                            for (int m = 0; m < MT; ++m)
#pragma unroll
                                for (int j = 0; j < 4; ++j) xf[m].w[j] = SWAP ? __builtin_amdgcn_ds_bpermute(from, xq[xs][m].w[j]) : xq[xs][m].w[j];
#pragma unroll
                            for (int m = 0; m < MT; ++m) X[m] = mfma_x<BF>(ones, xf[m], X[m]);
#pragma unroll
                            for (int n = 0; n < NT; ++n) {
                                Frag8 wf;
#pragma unroll
                                for (int j = 0; j < 4; ++j)
                                    wf.w[j] = BF ? ((wq[s][n][c] >> (4 * j)) & kCodeLo) | 0x43004300u : (j ? wq[s][n][c] >> (4 * j - 4) : wq[s][n][c] << 4) & kCodeHi;
#pragma unroll
                                for (int m = 0; m < MT; ++m) D[n][m] = mfma_x<BF>(wf, xf[m], D[n][m]);
                            }
                            if constexpr (c % 2 == 1) load_x(std::integral_constant<int, xs - 1>{}, 4 * kb + c - 1 + XD);
                        });
#pragma unroll
                        for (int n = 0; n < NT; ++n)
                            static_for<0, 4>([&](auto ii) {
                                constexpr int i = decltype(ii)::value;
                                const float sc = row_lane<i * NG + gi>(ss[n]), of = row_lane<i * NG + gi>(mm[n]);
#pragma unroll
                                for (int m = 0; m < MT; ++m) acc[n][m][i] = fmaf(of, X[m][i], fmaf(sc, D[n][m][i], acc[n][m][i]));
                            });
                    });
                    load_w(ws, kb + WD);
                }
            });
    }

    // ---- the waves' sums: those of the upper half go to the lower half, whose are then added up in their order
    auto place = [&](int w, int n, int m) {                        // [row r][output 4 g + i]
        return reinterpret_cast<float4_t*>(lds + ((w * NT + n) * MT + m) * 256 + r * 16 + 4 * g);
    };
    if (wave >= WK / 2)
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int m = 0; m < MT; ++m) *place(wave - WK / 2, n, m) = acc[n][m];
    __syncthreads();
    if (wave < WK / 2)
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int m = 0; m < MT; ++m) *place(wave, n, m) = acc[n][m] + *place(wave, n, m);
    __syncthreads();
    auto sum = [&](int at) {
        float v = lds[at];
#pragma unroll
        for (int w = 1; w < WK / 2; ++w) v += lds[w * NT * MT * 256 + at];
        return v;
    };
    for (int idx = threadIdx.x; idx < own * MT * 256; idx += WK * 64) {
        const int o = idx & 15, n = idx >> 4 & (own - 1), row = idx / (16 * own);      // outputs of a row side by side
        const int at = (n * MT + (row >> 4)) * 256 + (row & 15) * 16 + o;
        const int gr = row0 + row, gn = (tile0 + n) * 16 + o;
        if (gr >= a.M || gn >= a.N) continue;
        const float v = sum(at);
        const size_t to = (size_t)gr * a.out_stride + gn;
        if (a.epi == W4_STORE) ((uint16_t*)a.out)[to] = BF ? f32_to_bf16(v) : f32_to_f16(v);
        else if (a.epi == W4_F32) ((float*)a.out)[to] = v;
        else if (a.epi == W4_ADD_F32) ((float*)a.out)[to] += v;
        else if (swiglu) ((uint16_t*)a.out)[to] = f32_to_f16(v / (1.f + __expf(-v)) * sum(at + own * MT * 256));
    }
}

template <bool BF, int NG, bool SWAP, int MT, int NT, int WK>
static void launch_kernel(const W4Args& a, hipStream_t stream) {
    const int own = a.epi == W4_SWIGLU ? NT / 2 : NT;
    const dim3 grid((unsigned)((a.tiles + own - 1) / own), (unsigned)((a.M + MT * 16 - 1) / (MT * 16)));
    hipLaunchKernelGGL((w4_matmul_kernel<BF, NG, SWAP, MT, NT, WK>), grid, dim3(WK * 64), WK / 2 * NT * MT * 1024, stream, a);
}

// All sizes that follow are those of 256 compute units, in the rule as well.
// Tiles of rows (MT) and outputs (NT) per wave, waves to a workgroup (WK). Up to 16 rows: two output tiles where there are tiles enough for
// every compute unit all the same (1 row 4096 -> 22016 one tile and eight waves 14.4 us, so 11.9; 9 rows 15.8, 13.0; 1 row 4096 -> 4096 4.3, with two 5.2).
// More rows: the smallest tile of a wave with which workgroups of eight waves are at most one for each of 256 compute units; a larger one leaves
// units idle, a smaller one gives some a second workgroup. us as taken / with the next smaller / the next larger tile, bf16, group 128:
//   1 x 2 (outputs x rows) 40 rows 2048 -> 2048 5.1 / - / 5.9;        2 x 2 40 rows 4096 -> 4096 8.4 / 10.2 / 10.7;
//   2 x 3 72 rows 11008 -> 4096 21.8 / 24.6 / 27.5;                   4 x 3 72 rows 4096 -> 8192 15.4 / 20.0 / 18.3 (4 x 3, four waves)
// Where no tile is large enough, four waves: 4 x 3, with at least two workgroups a unit unless the rows fill such tiles much better than pairs, and not if they fill
// them much worse (72 rows 4096 -> 22016 35.9, 2 x 2 40.8; 40 rows 25.0 and 28.8), else 2 x 2 (240 rows 4096 -> 4096 21.2, 4 x 3 24.9; 24 rows
// 4096 -> 22016 17.1 and 24.6; 112 rows, group 32, 73.2 and 84.8). Groups of 32 leave fewer registers: 2 x 5 and eight waves where the rows fill that better
// (72 rows 4096 -> 22016 47.9, 4 x 3 54.9).
template <bool BF, int NG>
static void launch_rows(const W4Args& a, hipStream_t stream) {
    const bool pairs = a.epi == W4_SWIGLU;                           // (gate and up tiles share a wave)
    const long tiles = pairs ? 2l * a.tiles : a.tiles, by2 = (a.M + 31) / 32, by3 = (a.M + 47) / 48, by5 = (a.M + 79) / 80, cus = 256;
    const bool threes = 3 * by3 * 8 < 2 * by2 * (tiles * by3 < 8 * cus ? 7 : 9);
    if (a.M <= 4) tiles >= 1024 || pairs ? launch_kernel<BF, NG, false, 1, 2, 4>(a, stream) : launch_kernel<BF, NG, false, 1, 1, 8>(a, stream);
    else if (a.M <= 16) tiles >= 1024 || pairs ? launch_kernel<BF, NG, true, 1, 2, 4>(a, stream) : launch_kernel<BF, NG, true, 1, 1, 8>(a, stream);
    else if (tiles * by2 <= cus && !pairs) launch_kernel<BF, NG, true, 2, 1, 8>(a, stream);
    else if (tiles * by2 <= 2 * cus) launch_kernel<BF, NG, true, 2, 2, 8>(a, stream);
    else if (tiles * by3 <= 2 * cus) launch_kernel<BF, NG, true, 3, 2, 8>(a, stream);
    else if (tiles * by2 <= 4 * cus) launch_kernel<BF, NG, true, 2, 4, 8>(a, stream);
    else if (tiles * by3 <= 4 * cus) launch_kernel<BF, NG, true, 3, 4, 8>(a, stream);
    else if (NG == 4 && 5 * by5 < std::min(3 * by3, 2 * by2)) launch_kernel<BF, NG, true, NG == 4 ? 5 : 3, NG == 4 ? 2 : 4, NG == 4 ? 8 : 4>(a, stream);
    else if (threes) launch_kernel<BF, NG, true, 3, 4, 4>(a, stream);
    else launch_kernel<BF, NG, true, 2, 2, 4>(a, stream);
}

int launch_w4(const W4* w, const void* x, int64_t x_stride, int M, int dtype, int epi, void* out, int64_t out_stride, hipStream_t stream) {
    const int N = epi == W4_SWIGLU ? w->N / 2 : w->N;
    const W4Args a{w->blocks, (const uint16_t*)x, out, x_stride, out_stride, M, N, w->Kd, w->nkb, (N + 15) / 16, epi, N / 16};
    auto go = [&](auto bf) {
        constexpr bool BF = decltype(bf)::value;
        if (w->group == 128) launch_rows<BF, 1>(a, stream);
        else if (w->group == 64) launch_rows<BF, 2>(a, stream);
        else launch_rows<BF, 4>(a, stream);
    };
    if (dtype == LASER_BF16) go(std::true_type{});
    else go(std::false_type{});
    LASER_HIP_CHECK(hipGetLastError());
    return LASER_OK;
}

}  // namespace laser

using namespace laser;

static int check_w4(int N, int Kd, int group) {
    LASER_REQUIRE(group == 32 || group == 64 || group == 128, LASER_E_SHAPE, "group %d: 32, 64 or 128", group);
    LASER_REQUIRE(N > 0 && Kd > 0, LASER_E_INVALID_ARG, "N and Kd must be positive");
    LASER_REQUIRE(Kd % group == 0, LASER_E_SHAPE, "Kd %d is not a multiple of the group, %d", Kd, group);
    LASER_REQUIRE(((long)N + 15) / 16 * (((long)Kd + 127) / 128) < (1l << 23), LASER_E_LIMIT, "matrix too large");       // (a launch has less than 2^32 threads)
    return LASER_OK;
}

extern "C" int laser_w4_create(const uint8_t* codes, const uint16_t* scales, const uint16_t* offsets, int N, int Kd, int group, void* stream, laser_w4** out) {
    LASER_REQUIRE(codes && scales && offsets && out, LASER_E_INVALID_ARG, "NULL argument");
    if (const int rc = check_w4(N, Kd, group)) return rc;
    LASER_REQUIRE((uintptr_t)scales % 2 == 0 && (uintptr_t)offsets % 2 == 0, LASER_E_INVALID_ARG, "scales or offsets are not aligned to their elements");
    W4* w = new W4{N, Kd, group, (Kd + 127) / 128, nullptr};
    const size_t n_blocks = (size_t)((N + 15) / 16) * w->nkb;
    auto fail = [&](hipError_t e, const char* what) {
        set_error("%s: %s", what, hipGetErrorString(e));
        laser_w4_destroy(reinterpret_cast<laser_w4*>(w));
        return LASER_E_HIP;
    };
    hipError_t e = hipMalloc((void**)&w->blocks, n_blocks * block_bytes(128 / group));
    if (e != hipSuccess) return fail(e, "hipMalloc");
    hipLaunchKernelGGL(w4_layout_kernel, dim3((unsigned)n_blocks), dim3(256), 0, (hipStream_t)stream, codes, scales, offsets, N, Kd, group, w->nkb, w->blocks);
    if ((e = hipGetLastError()) != hipSuccess) return fail(e, "w4_layout_kernel");
    if ((e = hipStreamSynchronize((hipStream_t)stream)) != hipSuccess) return fail(e, "hipStreamSynchronize");
    *out = reinterpret_cast<laser_w4*>(w);
    return LASER_OK;
}

extern "C" int laser_w4_destroy(laser_w4* h) {
    W4* w = reinterpret_cast<W4*>(h);
    if (!w) return LASER_OK;
    if (w->blocks) (void)hipFree(w->blocks);
    delete w;
    return LASER_OK;
}

extern "C" int laser_w4_quantize(const uint16_t* w, int N, int Kd, int group, uint8_t* codes, uint16_t* scales, uint16_t* offsets, void* stream) {
    LASER_REQUIRE(w && codes && scales && offsets, LASER_E_INVALID_ARG, "NULL argument");
    if (const int rc = check_w4(N, Kd, group)) return rc;
    const size_t groups = (size_t)N * (Kd / group);
    hipLaunchKernelGGL(w4_quantize_kernel, dim3((unsigned)((groups * 8 + 255) / 256)), dim3(256), 0, (hipStream_t)stream, w, groups, group, codes, scales, offsets);
    LASER_HIP_CHECK(hipGetLastError());
    return LASER_OK;
}

extern "C" int laser_w4_matmul(const laser_w4* h, const void* x, int64_t x_stride, int M, int dtype, void* out, int64_t out_stride, void* stream) {
    const W4* w = reinterpret_cast<const W4*>(h);
    LASER_REQUIRE(w != nullptr, LASER_E_INVALID_ARG, "w is NULL");
    LASER_REQUIRE(dtype == LASER_F16 || dtype == LASER_BF16, LASER_E_INVALID_ARG, "dtype %d: LASER_F16 or LASER_BF16", dtype);
    LASER_REQUIRE(M >= 0 && M <= 65535 * 32, LASER_E_INVALID_ARG, "M %d out of range", M);
    LASER_REQUIRE(x_stride >= w->Kd && out_stride >= w->N, LASER_E_INVALID_ARG, "rows overlap: strides %lld, %lld", (long long)x_stride, (long long)out_stride);
    if (M == 0) return LASER_OK;
    LASER_REQUIRE(x && out, LASER_E_INVALID_ARG, "NULL argument");
    LASER_REQUIRE((uintptr_t)x % 2 == 0 && (uintptr_t)out % 2 == 0, LASER_E_INVALID_ARG, "x or out is not aligned to its elements");
    return launch_w4(w, x, x_stride, M, dtype, W4_STORE, out, out_stride, (hipStream_t)stream);
}
