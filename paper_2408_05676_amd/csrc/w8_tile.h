// Products of many rows in 8-bit codes with 8-bit weights (see eight_bit.h): a tile of rows by four waves' columns a workgroup.
//
// out[r][n] = s_x[r] s_w[n] sum of c_x c_w: integers, so the order of the sums does not matter and nothing is rounded before the scales.
// All four waves multiply the same WM x 16 rows, each with WN x 16 columns of its own: rows come through LDS, once a workgroup, and weights straight into the registers of the
// one wave that needs them, in the order its lanes hold them. At 11 x 6 fragments a wave a stage (128 inputs) takes 110 KB through LDS, in and out, where waves arranged 2 x 2
// with both operands in it would take 212, and 70 KB from L2, 34 bytes a clock of its matrix instructions.
//
// Bound: few hundred rows, the weights' way from memory and the two ends of a launch (249 rows gated 2048 -> 2 x 5632, 128 x 128 tiles on 176 compute units: start 1.3 us, 16 stages 7.1, results
// 2.1, launch 2); many rows, the matrix instructions at the clock that the card holds under them (704 rows gated 4096 -> 2 x 11008, 176 x 384 tiles: start 3.6, 32 stages of 1.3 us,
// results 8.6; a stage's matrix instructions alone 0.90 us, all of it with zeros as data 1.15). 704 rows, six matrices in turn: 4096 -> 12288 39 us (1.8 POP/s), gated
// 4096 -> 2 x 11008 59 to 67 us (2.1 to 1.9, as the card's clock is), 11008 -> 4096 42 us, 4096 -> 4096 18 us (fp32 results 43, 44 and 20); three in turn 36 and 57; a library's int8 products of these sizes without the epilogue 64, 90 and 55 us (8192 cubed: 2.04 POP/s).
#pragma once

#include "eight_bit.h"

namespace laser {

struct W8Args {
    const uint8_t* w; const float* w_scales;
    const int8_t* x; const float* x_scales;
    void* out;
    int64_t x_stride, out_stride;
    int M, outs, rows, Kd, Kp;
    int dtype;
    int tiles_m, tiles_n;
};

// (v_rcp_f32 is within one unit of the last place; a division proper takes ten instructions)
__device__ inline float silu_times(float gate, float up) { return gate * __builtin_amdgcn_rcpf(1.f + __expf(-gate)) * up; }

// o[0..3]: results of outputs n .. n + 3
template <int DT>
__device__ inline void w8_store(const W8Args& a, int row, int n, const float (&o)[4]) {
    const int64_t at = row * a.out_stride + n;
    if (n + 4 <= a.outs) { store_elems<DT, 4>(a.out, at, o); return; }
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (n + i < a.outs) {
            if constexpr (DT == DT_F32) ((float*)a.out)[at + i] = o[i];
            else ((uint16_t*)a.out)[at + i] = DT == DT_BF16 ? f32_to_bf16(o[i]) : f32_to_f16(o[i]);
        }
}

// 16 bytes a lane from base + vo to LDS at `at`, lane after lane. m0 holds the address, one wait state before its use.
__device__ inline void load_to_lds(uint64_t base, uint32_t vo, uint32_t at) {
    const u32x4 srd{(uint32_t)base, (uint32_t)(base >> 32), 0xFFFFFFFFu, 0x00020000u};
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %2, 0 offen lds" ::"v"(vo), "s"(at), "s"(srd) : "memory", "m0");
}
__device__ inline void load_dword_to_lds(uint64_t base, uint32_t vo, uint32_t at) {          // four bytes a lane
    const u32x4 srd{(uint32_t)base, (uint32_t)(base >> 32), 0xFFFFFFFFu, 0x00020000u};
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tbuffer_load_dword %0, %2, 0 offen lds" ::"v"(vo), "s"(at), "s"(srd) : "memory", "m0");
}
__device__ inline uint32_t lds_address(const void* p) { return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const char*)p; }

// Accumulators are pinned to the accumulation registers by assembly (V: to vector registers, where those are full): left to itself the compiler moves them between the two.
template <bool V>
__device__ inline void mfma_i8_acc(const u32x4& w, const u32x4& x, int4_t& c) {
    if constexpr (V) asm volatile("v_mfma_i32_16x16x64_i8 %0, %1, %2, %0" : "+v"(c) : "v"(w), "v"(x));
    else asm volatile("v_mfma_i32_16x16x64_i8 %0, %1, %2, %0" : "+a"(c) : "v"(w), "v"(x));
}
template <bool V>
__device__ inline void mfma_i8_first(const u32x4& w, const u32x4& x, int4_t& c) {
    if constexpr (V) asm volatile("v_mfma_i32_16x16x64_i8 %0, %1, %2, 0" : "=&v"(c) : "v"(w), "v"(x));
    else asm volatile("v_mfma_i32_16x16x64_i8 %0, %1, %2, 0" : "=&a"(c) : "v"(w), "v"(x));
}

constexpr int kW8Waves = 4;
// a ring of four stages; the results of 16 rows at least fit in it
constexpr int w8_tile_lds(int wm, int wn) { return wm * 8192 > 16 * (wn * 256 + 16) ? wm * 8192 : 16 * (wn * 256 + 16); }

// WM x WN: 16-row and 16-column fragments of a wave. A stage is 128 inputs, two steps of the matrix instruction.
template <int WM, int WN, bool GATED>
__global__ __launch_bounds__(64 * kW8Waves, 1) void w8_gemm_tile_kernel(W8Args a) {
    constexpr int NW = kW8Waves, BM = WM * 16, NS = 4, WD = 4;
    constexpr int SBYTES = BM * 128, PIECES = 2 * WM, LPS = (PIECES + NW - 1) / NW;       // a piece: 8 rows, one load of a wave
    static_assert(!GATED || WN % 2 == 0, "gate and up fragments come in pairs");
    constexpr int LDS = w8_tile_lds(WM, WN);
    static_assert(LDS + 1024 <= 163840, "LDS");
    __shared__ __attribute__((aligned(1024))) char lds[LDS + 1024];

    const int units = a.tiles_m * a.tiles_n, per = (units + 7) / 8;
    const int li = blockIdx.x / 8, unit = (blockIdx.x % 8) * per + li;
    if (li >= per || unit >= units) return;
    const int tn = unit / a.tiles_m, tm = unit % a.tiles_m;

    const int lane = threadIdx.x & 63, lr = lane & 15, lg = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int nk = a.Kp / 128, nx = (a.Kd + 127) / 128;          // nk is even; where nx is odd the last stage of weights is zeros

    // ---- rows, through LDS: chunk c of row r sits at c ^ (r / 2 % 8)
    uint32_t voff[LPS];
#pragma unroll
    for (int j = 0; j < LPS; ++j) {
        const int p = min(wave + j * NW, PIECES - 1), row = p * 8 + (lane >> 3);
        voff[j] = (uint32_t)min(row, a.M - 1 - tm * BM) * (uint32_t)a.x_stride + (((lane & 7) ^ ((row >> 1) & 7)) * 16);
    }
    uint64_t xbase = (uint64_t)(uintptr_t)a.x + (uint64_t)tm * BM * a.x_stride;
    const uint32_t lds0 = lds_address(lds) + wave * 1024;
    const uint32_t last = lds0 + (PIECES - 1 - wave) * 1024;
    uint32_t lslot = 0;
    auto issue = [&](auto jc) {
        constexpr int j = decltype(jc)::value;
        const uint32_t at = (PIECES % NW != 0 && j == LPS - 1 && wave + j * NW >= PIECES ? last : lds0 + j * NW * 1024) + lslot;
        load_to_lds(xbase, voff[j], at);
    };
    int kreq = 0;
    auto next_stage = [&] {
        ++kreq;
        xbase += kreq < nx ? 128 : 0;
        lslot = lslot + SBYTES < SBYTES * NS ? lslot + SBYTES : 0;
    };

    // ---- weights, straight into registers, WD steps ahead
    const int col0 = (tn * NW + wave) * WN * 16, first = min(col0, a.rows - 16);
    uint32_t wo[WN];
#pragma unroll
    for (int j = 0; j < WN; ++j) wo[j] = (uint32_t)(min(col0 + j * 16, a.rows - 16) - first) * 64 + lane * 16;
    const uint8_t* wbase = a.w + (size_t)first * 64;
    const uint64_t wstep = (uint64_t)a.rows * 64;
    int wreq = 0;
    u32x4 fw[WD][WN];
    auto load_w = [&](auto sc, auto jc) {
        const auto rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(wbase), (short)0, -1, 0x00020000);
        fw[decltype(sc)::value][decltype(jc)::value] = __builtin_amdgcn_raw_buffer_load_b128(rsrc, wo[decltype(jc)::value], 0, 0);
    };
    auto next_w = [&] { ++wreq; wbase += wreq < 2 * nk ? wstep : 0; };

    // The workgroups of a column of tiles walk the same weights together. Each touches its share of their lines PD stages ahead, so that the others find them in L2: 704 rows of
    // 16384 -> 12288 129 -> 115 us with zeros as data, a few per cent with others (5 or 9 stages ahead no better).
    constexpr int PD = 3;
    const int line = min(tm + a.tiles_m * (wave * 64 + lane), WN * 16 * NW - 1);       // of a stage: 64-byte rows in pairs, step by step
    const int tile0 = tn * NW * WN * 16, step_lines = min(NW * WN * 16, a.rows - tile0) / 2;
    const uint32_t touch = (uint32_t)(line / (WN * 8 * NW)) * (uint32_t)wstep + (uint32_t)min(line % (WN * 8 * NW), step_lines - 1) * 128;
    uint64_t tbase = (uint64_t)(uintptr_t)a.w + (uint64_t)tile0 * 64;
    int treq = 0;
    const uint32_t junk = lds_address(lds) + SBYTES * NS + wave * 256;
    auto touch_ahead = [&] {
        if (a.tiles_m > 1) load_dword_to_lds(tbase, touch, junk);
        ++treq;
        tbase += treq < nk ? 2 * wstep : 0;
    };

    int4_t acc[WN][WM];                                             // (the first step writes it: zeros would be up to 264 writes before it)
    u32x4 fx[2][WM];
    uint32_t ox[2];
#pragma unroll
    for (int s = 0; s < 2; ++s) ox[s] = lr * 128 + (((s * 4 + lg) ^ ((lr >> 1) & 7)) * 16);
    auto read_x = [&](auto sc, auto ic, int slot) {
        constexpr int s = decltype(sc)::value, i = decltype(ic)::value;
        fx[s][i] = *reinterpret_cast<const u32x4*>(lds + slot * SBYTES + ox[s] + i * 2048);
    };
    // Multiplies step s of a stage (weights in ring slot q), reads the rows' fragments of the other step from rslot meanwhile, requests the weights
    // WD steps on, and the loads L0 .. L1 - 1 of a later stage's rows.
    auto multiply = [&](auto firstc, auto sc, auto qc, int rslot, auto l0c, auto l1c) __attribute__((always_inline)) {
        constexpr int s = decltype(sc)::value, q = decltype(qc)::value, L0 = decltype(l0c)::value, L1 = decltype(l1c)::value, NMUL = WM * WN;
        static_for<0, NMUL>([&](auto mc) {
            constexpr int m = decltype(mc)::value, j = m / WM, i = m % WM;
            constexpr int r0 = 2 * m * WM / NMUL, r1 = 2 * (m + 1) * WM / NMUL;              // (in the first half: the wait behind the step finds them done)
            static_for<(r0 < WM ? r0 : WM), (r1 < WM ? r1 : WM)>([&](auto ic) { read_x(std::integral_constant<int, 1 - s>{}, ic, rslot); });
            constexpr int l0 = L0 + (2 * m * (L1 - L0) + NMUL) / (2 * NMUL), l1 = L0 + (2 * (m + 1) * (L1 - L0) + NMUL) / (2 * NMUL);
            static_for<l0, l1>([&](auto jc) { issue(jc); });
            if constexpr (decltype(firstc)::value) mfma_i8_first<(m >= 64)>(fw[q][j], fx[s][i], acc[j][i]);
            else mfma_i8_acc<(m >= 64)>(fw[q][j], fx[s][i], acc[j][i]);
            if constexpr (i == WM - 1) load_w(qc, std::integral_constant<int, j>{});
            __builtin_amdgcn_sched_barrier(0);
        });
        next_w();
    };
    // newer requests of a wave than the rows of the stage that is waited for: those of the stages behind it and the weights between
    constexpr int NEWER = (NS - 2) * (LPS + 2 * WN);
    auto sync = [&] {
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(NEWER < 63 ? NEWER : 63) : "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    using C0 = std::integral_constant<int, 0>;
    using C1 = std::integral_constant<int, 1>;
    using LA = std::integral_constant<int, LPS>;
    using LH = std::integral_constant<int, (LPS + 1) / 2>;
    for (int s = 0; s < PD; ++s) touch_ahead();
#pragma unroll
    for (int s = 0; s < NS - 1; ++s) { static_for<0, LPS>([&](auto jc) { issue(jc); }); next_stage(); }
    static_for<0, LH::value>([&](auto jc) { issue(jc); });
    static_for<0, WD>([&](auto qc) { static_for<0, WN>([&](auto jc) { load_w(qc, jc); __builtin_amdgcn_sched_barrier(0); }); next_w(); });
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"((NS - 2) * LPS + LH::value + WD * WN < 63 ? (NS - 2) * LPS + LH::value + WD * WN : 63) : "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    static_for<0, WM>([&](auto ic) { read_x(C0{}, ic, 0); });
    int slot = 0;
    auto two_stages = [&](auto firstc) __attribute__((always_inline)) {                            // (nk is even: there is no way out between them, past which the accumulators would be copied)
        static_for<0, WD / 2>([&](auto uc) {
            constexpr int u = decltype(uc)::value;
            const int nslot = slot + 1 < NS ? slot + 1 : 0;
            touch_ahead();
            multiply(std::bool_constant<decltype(firstc)::value && u == 0>{}, C0{}, std::integral_constant<int, 2 * u>{}, slot, LH{}, LA{});
            next_stage();
            sync();
            multiply(std::false_type{}, C1{}, std::integral_constant<int, 2 * u + 1>{}, nslot, C0{}, LH{});
            slot = nslot;
        });
    };
    two_stages(std::true_type{});
    for (int kt0 = WD / 2; kt0 < nk; kt0 += WD / 2) two_stages(std::false_type{});
    // The surplus requests must not land in a later workgroup's LDS; the last matrix instructions must have written.
    asm volatile("s_waitcnt vmcnt(0)\n\ts_nop 15\n\ts_nop 15" ::: "memory");
    static_for<0, WM * WN>([&](auto mc) {
        constexpr int m = decltype(mc)::value;
        int4_t& c = acc[m / WM][m % WM];
        if constexpr (m >= 64) asm volatile("" : "+v"(c));
        else asm volatile("" : "+a"(c));
    });

    // ---- results: a lane holds columns 4 lg .. 4 lg + 3 of every fragment, row lr of every 16. They leave by way of LDS, so that threads side by
    // side store whole lines (in pieces of eight bytes 17 MB took 10 us, so 4). Sums put there as integers and scaled by the threads that store them: 704 rows gated 61 -> 66 us.
    auto store = [&](auto dt) {
        constexpr int DT = decltype(dt)::value, OC = (GATED ? WN / 2 : WN) * 16, ES = DT == DT_F32 ? 4 : 2;      // columns of a wave, bytes
        constexpr int PITCH = OC * NW * ES + 16, PPR = OC * NW * ES / 16, EPP = 16 / ES;                         // pieces of 16 bytes of a row
        constexpr int FIT = LDS / (16 * PITCH), CH = FIT < WM ? FIT : WM;      // fragment rows at a time
        static_assert(CH >= 1, "LDS");
        using T = std::conditional_t<DT == DT_F32, float, uint16_t>;
        const int out0 = tn * NW * OC;                       // first output of the tile
        static_for<0, (WM + CH - 1) / CH>([&](auto cc) {
            constexpr int i0 = decltype(cc)::value * CH, i1 = i0 + CH < WM ? i0 + CH : WM;
            __syncthreads();
            static_for<0, (GATED ? WN / 2 : WN)>([&](auto jc) {
                constexpr int j = decltype(jc)::value * (GATED ? 2 : 1);
                const int col = min(col0 + j * 16, a.rows - 16 * (GATED ? 2 : 1)) + 4 * lg;
                const float4_t sw = *reinterpret_cast<const float4_t*>(a.w_scales + col), su = GATED ? *reinterpret_cast<const float4_t*>(a.w_scales + col + 16) : sw;
#pragma unroll
                for (int i = i0; i < i1; ++i) {
                    const float sx = a.x_scales[min(tm * BM + i * 16 + lr, a.M - 1)];
                    float o[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        o[e] = (float)acc[j][i][e] * sw[e] * sx;
                        if constexpr (GATED) o[e] = silu_times(o[e], (float)acc[j + (GATED ? 1 : 0)][i][e] * su[e] * sx);
                    }
                    store_elems<DT, 4>(lds, ((i - i0) * 16 + lr) * (PITCH / ES) + wave * OC + decltype(jc)::value * 16 + 4 * lg, o);
                }
            });
            __syncthreads();
            for (int p = threadIdx.x; p < (i1 - i0) * 16 * PPR; p += 64 * NW) {
                const int r = p / PPR, c = p % PPR * EPP, row = tm * BM + i0 * 16 + r, left = a.outs - out0 - c;
                if (row >= a.M) break;
                const char* from = lds + r * PITCH + c * ES;
                T* to = (T*)a.out + row * a.out_stride + out0 + c;
                if (left >= EPP) {
                    const u32x4 v = *reinterpret_cast<const u32x4*>(from);
                    *reinterpret_cast<u32x4_a2*>(to) = v;
                } else
                    for (int e = 0; e < left; ++e) to[e] = reinterpret_cast<const T*>(from)[e];
            }
        });
    };
    if (a.dtype == DT_F16) store(std::integral_constant<int, DT_F16>{});
    else if (a.dtype == DT_BF16) store(std::integral_constant<int, DT_BF16>{});
    else store(std::integral_constant<int, DT_F32>{});
}

struct W8Shape { int wm, wn; };
constexpr W8Shape kW8Shapes[] = {{2, 2}, {3, 2}, {4, 2}, {5, 2}, {6, 2}, {8, 2}, {5, 4}, {8, 4}, {6, 6}, {8, 6}, {11, 6}};
constexpr int kW8ShapeN = (int)(sizeof(kW8Shapes) / sizeof(kW8Shapes[0]));

template <int J, int N, class F>
static void each(F&& f) {
    if constexpr (J < N) { f(std::integral_constant<int, J>{}); each<J + 1, N>(f); }
}

template <bool GATED>
inline void go_w8_tile(W8Args a, int v, hipStream_t stream) {
    each<0, kW8ShapeN>([&](auto vc) {
        if (decltype(vc)::value != v) return;
        constexpr int WM = kW8Shapes[decltype(vc)::value].wm, WN = kW8Shapes[decltype(vc)::value].wn;
        a.tiles_m = (a.M + WM * 16 - 1) / (WM * 16);
        a.tiles_n = (a.rows + WN * 64 - 1) / (WN * 64);
        const unsigned grid = 8u * (unsigned)((a.tiles_m * a.tiles_n + 7) / 8);
        launch(w8_gemm_tile_kernel<WM, WN, GATED>, dim3(grid), dim3(64 * kW8Waves), stream, a);
    });
}
void launch_w8_tile_plain(const W8Args& a, int v, hipStream_t stream);
void launch_w8_tile_gated(const W8Args& a, int v, hipStream_t stream);

}  // namespace laser
