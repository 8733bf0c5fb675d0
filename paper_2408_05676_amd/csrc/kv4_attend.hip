// Attention of a step's rows over the 4-bit paged cache (four_bit.h has its layout and how codes enter the matrix instructions).
//
// Query rows of one key/value head (row r of the step, query head j of the group: packed row r G + j) form tiles of 16. A wave
// walks its share of the context 32 tokens (two pages) at a time:
//   scores   S[t][row] = sum over groups c of s[t][c] (codes[t][c] . q[row][c]) + m[t][c] sum(q[row][c]): one matrix instruction per group and page,
//            K as the first operand, one for the offsets of all groups, then a multiply-add per score and group in fp32; the scales of four tokens
//            come out of the lane's row of sixteen by a lane broadcast that the multiply-add does itself. Queries are multiplied by a power of two of
//            their row so that fp16 holds them (bf16 exactly down to 2^-14 of the row's largest); fp32 queries are two planes.
//   softmax  against a reference m_ref per row that moves only when a score (an exponent of 2) exceeds it by 14: else nothing crosses lanes.
//   values   O[row][ch] += sum over t of (p[row][t] s[t][c]) codes[t][ch]: p s in fp16 is the first operand as it stands in the lanes, since the page order
//            gives both products the same tokens per lane; plus p m, one more instruction for all groups. p s and p are two planes where the output has more
//            than eight bits. One plane each for bf16 results: that rounding leaves them 4 to 8 % further off the formula than their own does
//            (two planes: 115 us against 87 for the prompt pieces below).
// Waves of a workgroup share a context, workgroups split it further when there are few rows; a second kernel joins the parts. Pages come
// straight into LDS, two pairs ahead of a wave, so that 60 KB a compute unit are on their way (through registers, one pair ahead, 64
// sequences took 55 us of what follows).
// Bound: vector instructions, some 300 a pair of pages (of them 80 take codes out of words, 64 apply the keys' scales, 48 the values'), beside
// the pages' way from memory. Calls in a row, bf16: 64 sequences of 11 rows, 32 heads, 448 tokens in the mean 42.3 us (150 MB, 3.5 TB/s; vector units
// busy for 25 us of it), fp16 47.4; one row of 32 + 8 heads behind 65000 tokens 21.9 with the joining (83 MB, 3.8 TB/s); 64 rows of 32 + 8 heads behind
// 8000 tokens, four sequences, 87 us (0.34 PFLOP/s), fp16 115.
#include <algorithm>

#include "four_bit.h"

namespace laser {

constexpr int kWaves = 4;                            // of a workgroup; one and two were slower (16 users' single tokens, 1024 behind them: 23.7, 22.1, 18.2 us)
constexpr float kSumUnit = 1.f / 256.f;              // sums of 32 queries below 2^15, in fp16: scores are in this unit until they are scaled
constexpr int kPartSlots = 2048;                     // (tile, split) results a launch may leave for the joining kernel
constexpr int part_floats(int dh) { return 32 + 16 * dh; }
size_t kv4_part_floats(int dh) { return (size_t)kPartSlots * part_floats(dh); }

__device__ inline Frag8 pack8(const float (&x)[8]) {
    Frag8 f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const half2_t t = {(_Float16)x[2 * i], (_Float16)x[2 * i + 1]};
        f.w[i] = __builtin_bit_cast(uint32_t, t);
    }
    return f;
}
__device__ inline float max_over_rows(float x) {     // over the four lanes l % 16
    x = fmaxf(x, __shfl_xor(x, 16));
    return fmaxf(x, __shfl_xor(x, 32));
}
__device__ inline float sum_over_rows(float x) {
    x += __shfl_xor(x, 16);
    return x + __shfl_xor(x, 32);
}

template <int DT>
__device__ inline void store_out(const AttendArgs& a, size_t o, const float (&x)[4]) {
    if constexpr (DT == DT_SPLIT) {
        float hi[4], lo[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) { hi[j] = (float)(_Float16)x[j]; lo[j] = (x[j] - hi[j]) * kLoScale; }
        store_elems<DT_F16, 4>(a.out.p, o, hi);
        store_elems<DT_F16, 4>(a.out_lo, o, lo);
    } else {
        store_elems<DT, 4>(a.out.p, o, x);
    }
}

// pi / G: packed rows are below 64 G, so the quotient is off by less than 2^-17, and never within 1 / (2 G) >= 2^-9 of a border
__device__ inline int row_of(const AttendArgs& a, int pi) { return (int)(((float)pi + 0.5f) * a.inv_g); }
__device__ inline size_t out_at(const AttendArgs& a, int b, int h, int pi) {
    const int row = row_of(a, pi);
    return (size_t)b * a.out.seq + (size_t)row * a.out.row + (size_t)(h * a.G + pi - row * a.G) * a.out.head;
}

// ---- a wave's ring of two pairs of pages in LDS, written by the loads themselves
// A pair: the codes of both pages one after the other, then both pages' scales and offsets; requests of 1 KB, 16 bytes a lane.
template <int DH>
struct Ring {
    static constexpr int kCodes = 16 * DH, kSm = 4 * DH;             // bytes of a page
    static constexpr int kFull = 2 * kCodes / 1024;                  // requests for the codes
    static constexpr int kLoads = kFull + 1;                         // and one for both pages' scales (half of it twice where they are 512 bytes)
    static constexpr int kSlot = kLoads * 1024;

    // m0: where a request's first lane writes, one wait state before its use
    __device__ static inline void request(uint32_t lds, const uint8_t* uniform, uint32_t off) {
        asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %2" ::"v"(off), "s"(lds), "s"(uniform) : "memory", "m0");
    }
    __device__ static inline void request(uint32_t lds, const uint8_t* per_lane) {
        asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(per_lane), "s"(lds) : "memory", "m0");
    }
    __device__ static inline void load(uint32_t lds, const uint8_t* a, const uint8_t* b, int lane) {
#pragma unroll
        for (int i = 0; i < kFull; ++i) request(lds + i * 1024, i < kFull / 2 ? a : b, (i % (kFull / 2)) * 1024 + lane * 16);
        const uint8_t* p = lane & (kSm / 16) ? b : a;
        request(lds + kFull * 1024, p + kCodes + (lane & (kSm / 16 - 1)) * 16);
    }
    template <int NEWER>
    __device__ static inline void wait() { asm volatile("s_waitcnt vmcnt(%0)" ::"i"(NEWER * kLoads) : "memory"); }
    __device__ static inline void have_read() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }
};

typedef const __attribute__((address_space(4))) int32_t* scalar_ints;       // (of arrays that no one writes while the kernel runs)

template <int CG>
__device__ inline float sum_over_groups(float x) {                   // over the CG lanes of a query row
    if constexpr (CG >= 2) x += __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), 0xB1, 0xF, 0xF, true));   // lanes 1 0 3 2
    if constexpr (CG >= 4) x += __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), 0x4E, 0xF, 0xF, true));   // lanes 2 3 0 1
    return x;
}

// IN: type of q; OUT: of the result. A workgroup takes a tile; its waves share the context.
// CG = 1: a tile is 16 rows, a column of the scores each. CG = all groups (4, or 2 at 64 channels): a tile is 16 / CG rows, and a column one
// group of a row: the operand holds that group's queries and zeros for the others, one chain of matrix instructions gives the scores'
// parts by group, each lane scales its own (four multiply-adds instead of thirty-two) and the lanes of a row add up; likewise p s is
// formed for one group a lane, and of the result the sixteen rows give each channel only that of its group.
template <int DH, int IN, int OUT, int CG>
__global__ __launch_bounds__(kWaves * 64, 3) void kv4_attend_kernel(AttendArgs a) {
    constexpr int NG = DH / 32, NT = DH / 16;        // groups, 16-channel tiles
    constexpr int J = 16 / CG;                       // rows of a tile
    constexpr bool kTwoQ = IN == DT_F32, kTwoP = OUT != DT_BF16;
    constexpr float kOdd = kTwoP ? 1.f : 16.f, kKeyUnit = kTwoP ? kCodeUnit / 16.f : kCodeUnit;       // of key codes (kTwoP: all in bits 4..7): odd groups by even ones; 1 / even ones
    constexpr int kStride = DH + 4;                  // of a row in LDS: four rows apart are sixteen banks apart
    constexpr int kWaveLds = 2 * Ring<DH>::kSlot > J * kStride * 4 ? 2 * Ring<DH>::kSlot : J * kStride * 4;
    __shared__ float sm_m[kWaves][J], sm_l[kWaves][J];
    __shared__ __attribute__((aligned(1024))) char lds[kWaves * kWaveLds];      // a wave's ring, later its results [J][kStride]
    // (heads side by side: with a multiple of eight of them, the tiles of a head, which read the same pages, share an XCD and its cache)
    const int h = blockIdx.x % a.H, tile = blockIdx.x / a.H, b = blockIdx.y, split = blockIdx.z;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int r = lane & 15, g = lane >> 4, j = r / CG, cc = r % CG;
    // (what the whole wave shares is kept in scalar registers: addresses, loop bounds and branches)
    const int slot = __builtin_amdgcn_readfirstlane(a.seqs.slot(b)), len = ((scalar_ints)a.lens)[slot], cap = ((scalar_ints)a.seqs.cap)[slot];
    int nr = a.n_rows ? min(max(a.n_rows[b], 0), a.R) : a.R;
    nr = __builtin_amdgcn_readfirstlane(max(0, min(nr, cap - len)));      // (a length beyond the pages: rows that have no slot are left out)
    const int P = nr * a.G;                          // packed rows
    if (tile * J >= P || len < 0) return;

    // ---- this workgroup's pages [p0, p1), this wave's pairs of them; the first two are on their way while the queries are made ready
    const int npages = (len + nr + kPageSize - 1) / kPageSize;
    const int per = ((npages + a.nsplit - 1) / a.nsplit + 1) & ~1;
    const int p0 = split * per, p1 = min(npages, p0 + per);
    const uint8_t* base = a.pages + (size_t)h * page4_bytes(DH);
    const size_t page_step = (size_t)a.H * page4_bytes(DH);
    const scalar_ints bt = (scalar_ints)(a.block_table + (size_t)slot * a.mpps);
    auto page_at = [&](int p) { return base + (size_t)(unsigned)__builtin_amdgcn_readfirstlane(bt[min(p, p1 - 1)]) * page_step; };
    constexpr int kStep = 2 * kWaves;
    char* const mine = lds + wave * kWaveLds;
    const uint32_t ring = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)mine);
    int p = p0 + 2 * wave;
    if (p < p1) Ring<DH>::load(ring, page_at(p), page_at(p + 1), lane);
    if (p + kStep < p1) Ring<DH>::load(ring + Ring<DH>::kSlot, page_at(p + kStep), page_at(p + kStep + 1), lane);

    // ---- which rows of the step each row sees: lane l works out row l's, by pointer doubling along the tree
    unsigned long long anc_l;
    if (a.row_anc) anc_l = a.row_anc[(size_t)b * a.R + min(lane, a.R - 1)];
    else if (!a.parent) anc_l = (2ull << lane) - 1;
    else {
        anc_l = 1ull << lane;
        int up = lane > 0 && lane < a.R ? up_row(a.parent + (size_t)b * (a.R - 1), lane) : 0;
#pragma unroll
        for (int i = 0; i < 6; ++i) {
            const unsigned lo = __shfl((unsigned)anc_l, up), hi = __shfl((unsigned)(anc_l >> 32), up);
            anc_l |= ((unsigned long long)hi << 32) | lo;
            up = __shfl(up, up);
        }
    }

    // ---- queries: multiplied by a power of two of their row, to below 2^15 (and by 1 / kOdd in odd groups, whose codes come out that
    // many times larger); cs > 0 takes scores back to the exponents of 2 (the sign of the scale has gone into the queries)
    Frag8 q[NG], ql[NG];
    Frag8 qsum;                                  // CG = 1, operand of the offsets: first input 8 g is the sum of group g, in two parts
    constexpr float kUnit = CG == 1 ? kKeyUnit * kSumUnit : 1.f;          // of the keys' scales: scores come in units of kSumUnit, else 1 / kKeyUnit
    const int pi = min(tile * J + j, P - 1), row = row_of(a, pi), hq = h * a.G + pi - row * a.G;
    const unsigned anc_lo = __shfl((unsigned)anc_l, row), anc_hi = __shfl((unsigned)(anc_l >> 32), row);
    const unsigned long long anc = ((unsigned long long)anc_hi << 32) | anc_lo;
    const size_t qo = (size_t)b * a.q.seq + (size_t)row * a.q.row + (size_t)hq * a.q.head + 8 * g;
    float x[NG][8], mx = 0.f;
#pragma unroll
    for (int c = 0; c < NG; ++c) {
        load_elems<IN, 8>(a.q.p, qo + 32 * c, x[c]);
#pragma unroll
        for (int i = 0; i < 8; ++i) mx = fmaxf(mx, fabsf(x[c][i]));
    }
    mx = max_over_rows(mx);
    int e = 0;
    if (mx > 0.f && mx < INFINITY) { (void)frexpf(mx, &e); e = min(15 - e, 100); }
    const float up = ldexpf(a.scale_log2 < 0.f ? -1.f : a.scale_log2 > 0.f ? 1.f : 0.f, e);
    Frag8 ones;
#pragma unroll
    for (int i = 0; i < 4; ++i) ones.w[i] = 0x3C003C00u;
    float own = 0.f;
#pragma unroll
    for (int c = 0; c < NG; ++c) {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[c][i] *= c & 1 ? up / kOdd : up;
        q[c] = pack8(x[c]);
        float4_t sum = mfma_16x16x32(ones, q[c], float4_t{0.f, 0.f, 0.f, 0.f});          // of the lane's query row
        if constexpr (kTwoQ) {
#pragma unroll
            for (int i = 0; i < 8; ++i) x[c][i] -= (float)q[c].v[i];
            ql[c] = pack8(x[c]);
            sum = mfma_16x16x32(ones, ql[c], sum);
        }
        if (c == (CG == 1 ? g : cc)) own = sum[0] * ((c & 1 ? kOdd : 1.f) * (CG == 1 ? kSumUnit : 1.f / kKeyUnit));
        if (CG > 1 && c != cc) {
            q[c].v4 = u32x4{0, 0, 0, 0};
            if constexpr (kTwoQ) ql[c].v4 = u32x4{0, 0, 0, 0};
        }
    }
    const float qs = own;                            // (CG > 1: the sum of the lane's own group)
    if constexpr (CG == 1) {
        const _Float16 hi = (_Float16)own;
        const half2_t two = {hi, (_Float16)(own - (float)hi)};
        qsum.v4 = u32x4{__builtin_bit_cast(uint32_t, two), 0u, 0u, 0u};
    }
    // (queries near the largest fp32 numbers: a power of two that cs cannot hold waits in sm_l)
    int se = 0;
    (void)frexpf(a.scale_log2, &se);
    const int sh = (CG == 1 ? 8 : kTwoP ? 20 : 24) - e, beyond = max(0, se + sh - 120);
    const float cs = a.scale_log2 == 0.f ? 1.f : fmaxf(ldexpf(fabsf(a.scale_log2), sh - beyond), 1e-37f);
    const bool huge = __any(beyond > 0);
    if (huge && g == 0 && cc == 0) sm_l[wave][j] = ldexpf(1.f, min(beyond, 127));

    // ---- the walk. Weights are p = 2^(score - ref); ref moves, and what was summed with it, when a score passes it by more than kOver,
    // and is then set to kBack below the row's largest score: a row's largest p is 2^11 to 2^14. Values' scales are multiplied by `lift`, a power of
    // 16 for each group that brings the largest scale met so far into [1/8, 2), and what was summed with it when a larger one comes. p and p s lift thus
    // stay within fp16, and what it rounds to 0 is below 2^-36 of the largest weight and 2^-33 of that weight times the group's largest scale: a long
    // tail of small weights keeps its share however small the values are. (Steps of 16: the first pair of pages sets it, and few change it.)
    constexpr float kOver = 14.f, kBack = 11.f;
    float4_t acc[NT], accm = {0.f, 0.f, 0.f, 0.f};
    float ref = -INFINITY, limit = -INFINITY, l_run = 0.f;               // limit: (ref + kOver) in units of the scores before cs
    bool far = false;                                // some row's reference is so large that fp32 holds it to 2^-7 or less: see below
    float lift = 16777216.f;                         // of group r / 4 (CG > 1: the lane's own); the smallest scale above 0 is 2^-24
#pragma unroll
    for (int n = 0; n < NT; ++n) acc[n] = float4_t{0.f, 0.f, 0.f, 0.f};
    auto rescale = [&](float ref_new) {
        const float alpha = ref == ref_new ? 1.f : __builtin_amdgcn_exp2f(ref - ref_new);
        l_run *= alpha;
        ref = ref_new;
        far = __any(fabsf(ref_new) > 131072.f && ref_new != -INFINITY);
        limit = (ref_new + kOver) / cs;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float al = __shfl(alpha, 4 * g + i);                   // accumulator rows are the score columns 4 g + i
            accm[i] *= al;
#pragma unroll
            for (int n = 0; n < NT; ++n) acc[n][i] *= al;
        }
    };

    uint32_t at = 0;                                 // of the pair in the ring
    for (; p < p1; p += kStep, at ^= Ring<DH>::kSlot) {
        // the pair behind the next one: its page numbers now, the request once this pair has been read
        const bool more = p + 2 * kStep < p1;
        const uint8_t *n0 = page_at(p + 2 * kStep), *n1 = page_at(p + 2 * kStep + 1);
        if (p + kStep < p1) Ring<DH>::template wait<1>();
        else Ring<DH>::template wait<0>();
        const char* from = mine + at;
        uint32_t kw[2][NG], vw[2][NG];
        uint32_t ksm[2][CG == 1 ? 1 : 4], vsm[2][CG == 1 ? 1 : 4], km[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const char *pk = from + u * Ring<DH>::kCodes + lane * 4 * NG, *pv = pk + page4_v(DH), *ps = from + 2 * Ring<DH>::kCodes + u * Ring<DH>::kSm;
            if constexpr (NG == 4) {
                const u32x4 k = *reinterpret_cast<const u32x4*>(pk), v = *reinterpret_cast<const u32x4*>(pv);
#pragma unroll
                for (int i = 0; i < 4; ++i) { kw[u][i] = k[i]; vw[u][i] = v[i]; }
            } else {
                const u32x2 k = *reinterpret_cast<const u32x2*>(pk), v = *reinterpret_cast<const u32x2*>(pv);
#pragma unroll
                for (int i = 0; i < 2; ++i) { kw[u][i] = k[i]; vw[u][i] = v[i]; }
            }
            if constexpr (CG == 1) {                 // lane r: of token 4 g + r % 4, group r / 4; km: of token r, group g
                const uint32_t* w = reinterpret_cast<const uint32_t*>(ps);
                ksm[u][0] = w[g * 4 * NG + (lane & (4 * NG - 1))];
                vsm[u][0] = w[16 * NG + g * 4 * NG + (lane & (4 * NG - 1))];
                km[u] = w[sm_index(DH, r, g & (NG - 1))];
            } else {                                 // of tokens 4 g .. 4 g + 3, the lane's own group
                const u32x4 k = *reinterpret_cast<const u32x4*>(ps + (g * NG + cc) * 16), v = *reinterpret_cast<const u32x4*>(ps + 64 * NG + (g * NG + cc) * 16);
#pragma unroll
                for (int i = 0; i < 4; ++i) { ksm[u][i] = k[i]; vsm[u][i] = v[i]; }
            }
        }
        Ring<DH>::have_read();
        if (more) Ring<DH>::load(ring + at, n0, n1, lane);

        // ---- scores: every lane has those of its tokens 4 g .. 4 g + 3 of each page and its row
        float s[8];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            Frag8 kf[NG];
#pragma unroll
            for (int c = 0; c < NG; c += 2)
#pragma unroll
                for (int w = 0; w < 2; ++w) {
                    const uint32_t a0 = kw[u][c + w], a1 = a0 >> 8;
                    kf[c].w[2 * w] = kTwoP ? (a0 << 4) & kCodeHi : a0 & kCodeLo;
                    kf[c].w[2 * w + 1] = kTwoP ? (a0 >> 4) & kCodeHi : a1 & kCodeLo;
                    kf[c + 1].w[2 * w] = a0 & kCodeHi;
                    kf[c + 1].w[2 * w + 1] = a1 & kCodeHi;
                }
            if constexpr (CG == 1) {
                const float ks = sm_scale(ksm[u][0]) * kUnit;
                Frag8 kmf;
                kmf.v4 = u32x4{__builtin_amdgcn_perm(km[u], km[u], 0x07060706u), 0u, 0u, 0u};
                float4_t sum = mfma_16x16x32(kmf, qsum, float4_t{0.f, 0.f, 0.f, 0.f});
                static_for<0, NG>([&](auto ci) {
                    constexpr int c = decltype(ci)::value;
                    float4_t d = {0.f, 0.f, 0.f, 0.f};
                    if constexpr (kTwoQ) d = mfma_16x16x32(kf[c], ql[c], d);
                    d = mfma_16x16x32(kf[c], q[c], d);
                    static_for<0, 4>([&](auto ii) {
                        constexpr int i = decltype(ii)::value;
                        sum[i] = fmaf(row_lane<c * 4 + i>(ks), d[i], sum[i]);
                    });
                });
#pragma unroll
                for (int i = 0; i < 4; ++i) s[4 * u + i] = sum[i];
            } else {
                float4_t d = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int c = 0; c < NG; ++c) {
                    if constexpr (kTwoQ) d = mfma_16x16x32(kf[c], ql[c], d);
                    d = mfma_16x16x32(kf[c], q[c], d);
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) s[4 * u + i] = sum_over_groups<CG>(fmaf(sm_scale(ksm[u][i]), d[i], sm_offset(ksm[u][i]) * qs));
            }
        }
        const bool tail = (p + 2) * kPageSize > len;
        if (tail || huge || p + 1 >= p1) {
            if (huge)
#pragma unroll
                for (int i = 0; i < 8; ++i) s[i] *= sm_l[wave][j];
            if (tail) {                              // slots behind the committed ones: along the row's own branch only
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    // the lane's four slots start rel behind the committed length: bits rel .. rel + 3 of the row's mask, ones below 0
                    const int rel = p + u < p1 ? (p + u) * kPageSize + 4 * g - len : 64;
                    const int up = min(max(rel, 0), 63), under = min(max(-rel, 0), 4);
                    const unsigned ahead = rel < 64 ? (unsigned)(anc >> up) : 0u, behind = ((unsigned)anc << under) | ((1u << under) - 1u);
                    const unsigned seen = rel >= 0 ? ahead : behind;
#pragma unroll
                    for (int i = 0; i < 4; ++i) s[4 * u + i] = (seen >> i) & 1u ? s[4 * u + i] : -INFINITY;
                }
            } else if (p + 1 >= p1) {                // an odd number of pages
#pragma unroll
                for (int i = 0; i < 4; ++i) s[4 + i] = -INFINITY;
            }
        }

        // ---- weights in place of scores, and their sums with the offsets
        Frag8 vm;                                    // offsets as an operand: column 4 c is group c (CG > 1: column r is group r % CG)
        constexpr int VS = CG == 1 ? 1 : 4;
        float vs[2][VS];                             // the values' scales, lifted
        bool large = false;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            if constexpr (CG == 1) {
                const uint32_t e0 = vsm[u][0], e1 = row_ahead<1>(e0), e2 = row_ahead<2>(e0), e3 = row_ahead<3>(e0);
                vm.w[2 * u] = __builtin_amdgcn_perm(e1, e0, 0x07060302u);
                vm.w[2 * u + 1] = __builtin_amdgcn_perm(e3, e2, 0x07060302u);
            } else {
                vm.w[2 * u] = __builtin_amdgcn_perm(vsm[u][1], vsm[u][0], 0x07060302u);
                vm.w[2 * u + 1] = __builtin_amdgcn_perm(vsm[u][3], vsm[u][2], 0x07060302u);
            }
#pragma unroll
            for (int i = 0; i < VS; ++i) {
                vs[u][i] = sm_scale(vsm[u][i]) * lift;
                large |= vs[u][i] >= 2.f;
            }
        }
        if (__any(large)) {
            float top = 0.f;                         // of tokens of the sequence: what lies behind them is someone else's and changes nothing
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const int here = len + nr - (p + u) * kPageSize - 4 * g;
#pragma unroll
                for (int i = 0; i < VS; ++i) top = fmaxf(top, (CG == 1 ? (r & 3) : i) < here ? sm_scale(vsm[u][i]) : 0.f);
            }
            if constexpr (CG == 1) {
                top = fmaxf(top, __shfl_xor(top, 1));
                top = fmaxf(top, __shfl_xor(top, 2));
            }
            top = max_over_rows(top);
            const int want = (127 - (int)(__float_as_uint(top) >> 23)) & ~3;     // exponent: top 2^want in [1/8, 2) (top = 0: large, lift stays)
            const float to = fminf(lift, __uint_as_float((unsigned)(127 + min(want, 24)) << 23));
            const float ratio = __uint_as_float(__float_as_uint(to) - __float_as_uint(lift) + 0x3F800000u);
            lift = to;
            if (p >= p0 + kStep) {                   // (else nothing has been summed)
                if constexpr (CG == 1)
                    static_for<0, NG>([&](auto ci) {
                        constexpr int c = decltype(ci)::value;
                        const float al = row_lane<4 * c>(ratio);
                        acc[2 * c] *= al;
                        acc[2 * c + 1] *= al;
                    });
                else
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float al = __shfl(ratio, 4 * g + i);
#pragma unroll
                        for (int n = 0; n < NT; ++n) acc[n][i] *= al;
                    }
            }
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int i = 0; i < VS; ++i) vs[u][i] = sm_scale(vsm[u][i]) * lift;
        }
        const float mx = fmaxf(fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3])), fmaxf(fmaxf(s[4], s[5]), fmaxf(s[6], s[7])));
        if (far || __any(mx > limit)) {
            if (__any(mx > limit)) rescale(fmaxf(ref, max_over_rows(mx) * cs - kBack));
            if (far) {                               // ref was rounded: the scores against it must be too, and stay within fp16
#pragma clang fp contract(off)
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float x = s[i] * cs, t = x - (ref == -INFINITY ? 0.f : ref);
                    s[i] = t > kOver ? kOver : t;    // (NaN stays)
                }
            }
        }
        const float mu = far || ref == -INFINITY ? 0.f : ref, unit = far ? 1.f : cs;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            s[i] = __builtin_amdgcn_exp2f(fmaf(s[i], unit, -mu));
            l_run += s[i];
        }
        const Frag8 ph = pack8(s);
        accm = mfma_16x16x32(ph, vm, accm);
        if constexpr (kTwoP) {
            float lo[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) lo[i] = s[i] - (float)ph.v[i];
            accm = mfma_16x16x32(pack8(lo), vm, accm);
        }

        // ---- values: operand fragments of tokens 4 g .. 4 g + 3 of both pages, p s of the group (CG > 1: of the lane's own) against them
        // (kTwoP: all codes in bits 4..7, see four_bit.h: in bits 0..3 they cost the sums 2^-20, and a result is the small difference of two
        // such sums: one row behind 65000 tokens came out three times as far off the formula as its rounding)
        Frag8 pv, pl;
        auto weigh = [&](auto ci) {
            constexpr int c = decltype(ci)::value;
            float ps[8];
            static_for<0, 8>([&](auto ii) {
                constexpr int i = decltype(ii)::value;
                if constexpr (CG == 1) ps[i] = row_lane<c * 4 + i % 4>(vs[i / 4][0]) * s[i];
                else ps[i] = vs[i / 4][i % 4] * s[i];
            });
            pv = pack8(ps);
            if constexpr (kTwoP) {
                float lo[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) lo[i] = ps[i] - (float)pv.v[i];
                pl = pack8(lo);
            }
        };
        static_for<0, NG>([&](auto ci) {
            constexpr int c = decltype(ci)::value;
            if constexpr (CG == 1 || c == 0) weigh(ci);
            Frag8 va, vb;
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const uint32_t a0 = vw[u][c], a1 = a0 >> 8;
                va.w[2 * u] = kTwoP ? (a0 << 4) & kCodeHi : a0 & kCodeLo;
                va.w[2 * u + 1] = kTwoP ? (a0 >> 4) & kCodeHi : a1 & kCodeLo;
                vb.w[2 * u] = a0 & kCodeHi;
                vb.w[2 * u + 1] = a1 & kCodeHi;
            }
            acc[2 * c] = mfma_16x16x32(pv, va, acc[2 * c]);
            acc[2 * c + 1] = mfma_16x16x32(pv, vb, acc[2 * c + 1]);
            if constexpr (kTwoP) {
                acc[2 * c] = mfma_16x16x32(pl, va, acc[2 * c]);
                acc[2 * c + 1] = mfma_16x16x32(pl, vb, acc[2 * c + 1]);
            }
        });
    }

    // ---- join the waves (a wave's results lie where its ring was: every request of it has been waited for)
    float* const res = reinterpret_cast<float*>(mine);
    const float l = sum_over_rows(l_run);
    if (g == 0 && cc == 0) { sm_m[wave][j] = ref; sm_l[wave][j] = l; }
    const float unlift = __uint_as_float(0x7F000000u - __float_as_uint(lift));           // 1 / lift
    static_for<0, NT>([&](auto ni) {
        constexpr int n = decltype(ni)::value, at = (CG == 1 ? 4 : 1) * (n / 2);         // of group n / 2 in a row of lanes
        const float unit = row_lane<at>(unlift) * (kTwoP || n & 1 ? kCodeUnit / 16.f : kCodeUnit);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (CG == 1 || i % CG == n / 2) {    // (row 4 g + i is group i % CG of query row (4 g + i) / CG)
                const float om = __shfl(accm[i], 16 * g + at);
                res[(4 * g + i) / CG * kStride + 16 * n + r] = fmaf(acc[n][i], unit, om);
            }
    });
    __syncthreads();
    for (int idx = threadIdx.x; idx < J * DH / 4; idx += kWaves * 64) {
        const int row = idx / (DH / 4), c = idx % (DH / 4) * 4;
        float M = sm_m[0][row], L = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 1; w < kWaves; ++w) M = fmaxf(M, sm_m[w][row]);
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            const float mw = sm_m[w][row], f = mw == M ? 1.f : __builtin_amdgcn_exp2f(mw - M);
            const float4_t v = *reinterpret_cast<const float4_t*>(lds + w * kWaveLds + (row * kStride + c) * 4);
            L += sm_l[w][row] * f;
#pragma unroll
            for (int i = 0; i < 4; ++i) o[i] += v[i] * f;
        }
        if (a.nsplit == 1) {
            const int pi = tile * J + row;
            if (pi < P) {
                const float inv = L == 0.f ? 0.f : 1.f / L;          // (nothing seen: 0; NaN stays)
#pragma unroll
                for (int i = 0; i < 4; ++i) o[i] *= inv;
                store_out<OUT>(a, out_at(a, b, h, pi) + c, o);
            }
        } else {
            float* part = a.part + ((((size_t)b * a.H + h) * a.nt + tile) * a.nsplit + split) * part_floats(DH);
            if (c == 0) { part[row] = M; part[16 + row] = L; }
            *reinterpret_cast<float4_t*>(part + 32 + row * DH + c) = float4_t{o[0], o[1], o[2], o[3]};
        }
    }
}

// Joins the parts of a split context: a workgroup per row, four channels a thread, the parts dealt round to 1024 / DH groups of threads.
template <int DH, int OUT>
__global__ __launch_bounds__(256) void kv4_join_kernel(AttendArgs a) {
    constexpr int C = DH / 4, S = 256 / C;
    __shared__ float sm_m[S], sm_l[S];
    __shared__ float4_t sm_o[S][C];
    const int row = blockIdx.x % a.J, tile = blockIdx.x / a.J % a.nt, h = blockIdx.x / a.J / a.nt, b = blockIdx.y, pi = tile * a.J + row;
    const int slot = a.seqs.slot(b), len = a.lens[slot];
    int nr = a.n_rows ? min(max(a.n_rows[b], 0), a.R) : a.R;
    nr = max(0, min(nr, a.seqs.cap[slot] - len));
    if (pi >= nr * a.G || len < 0) return;
    const float* part = a.part + (((size_t)b * a.H + h) * a.nt + tile) * a.nsplit * part_floats(DH);
    const int c = threadIdx.x % C, s0 = threadIdx.x / C;
    float M = -INFINITY, L = 0.f;
    float4_t o = {0.f, 0.f, 0.f, 0.f};
    constexpr int U = 4;                             // parts requested together
    for (int s = s0; s < a.nsplit; s += U * S) {
        float m[U], l[U];
        float4_t v[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const float* ps = part + (size_t)min(s + u * S, a.nsplit - 1) * part_floats(DH);
            m[u] = ps[row];
            l[u] = ps[16 + row];
            v[u] = *reinterpret_cast<const float4_t*>(ps + 32 + row * DH + 4 * c);
        }
        float top = M;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            m[u] = s + u * S < a.nsplit ? m[u] : -INFINITY;
            top = fmaxf(top, m[u]);
        }
        const float keep = M == top ? 1.f : __builtin_amdgcn_exp2f(M - top);
        L *= keep;
#pragma unroll
        for (int j = 0; j < 4; ++j) o[j] *= keep;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const float f = s + u * S >= a.nsplit ? 0.f : m[u] == top ? 1.f : __builtin_amdgcn_exp2f(m[u] - top);
            L += l[u] * f;                           // (0 times NaN stays NaN: a part that has met one)
#pragma unroll
            for (int j = 0; j < 4; ++j) o[j] += v[u][j] * f;
        }
        M = top;
    }
    if (c == 0) { sm_m[s0] = M; sm_l[s0] = L; }
    sm_o[s0][c] = o;
    __syncthreads();
    if (s0 != 0) return;
    float top = sm_m[0], sum = 0.f, x[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int s = 1; s < S; ++s) top = fmaxf(top, sm_m[s]);
#pragma unroll
    for (int s = 0; s < S; ++s) {
        const float f = sm_m[s] == top ? 1.f : __builtin_amdgcn_exp2f(sm_m[s] - top);
        const float4_t v = sm_o[s][c];
        sum += sm_l[s] * f;
#pragma unroll
        for (int j = 0; j < 4; ++j) x[j] += v[j] * f;
    }
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] *= inv;
    store_out<OUT>(a, out_at(a, b, h, pi) + 4 * c, x);
}

template <int DH, int IN, int OUT>
static void launch(const AttendArgs& a, hipStream_t stream) {
    const dim3 grid((unsigned)(a.H * a.nt), (unsigned)a.B, (unsigned)a.nsplit);
    if (a.J == 16) hipLaunchKernelGGL((kv4_attend_kernel<DH, IN, OUT, 1>), grid, dim3(kWaves * 64), 0, stream, a);
    else hipLaunchKernelGGL((kv4_attend_kernel<DH, IN, OUT, DH / 32>), grid, dim3(kWaves * 64), 0, stream, a);
    if (a.nsplit > 1) hipLaunchKernelGGL((kv4_join_kernel<DH, OUT>), dim3((unsigned)(a.H * a.nt * a.J), (unsigned)a.B), dim3(256), 0, stream, a);
}

// max_tokens: the most slots any of the sequences may have by the host's bounds
int launch_kv4_attend(AttendArgs a, int dh, int dtype, int max_tokens, hipStream_t stream) {
    int ncu = 0;
    LASER_HIP_CHECK(hipDeviceGetAttribute(&ncu, hipDeviceAttributeMultiprocessorCount, 0));
    // Up to 4 rows of a key/value head (8 at 64 channels) the columns of a tile are groups: 4 rows behind 65000 tokens 22.7 us (25.0 with rows
    // as columns), 1 row of 16 sequences behind 1024 18.1 (19.5); two such tiles for up to 8 rows 21.6 and one of 16 18.8 (8 rows, 4000 tokens).
    const int P = a.R * a.G, few = 16 * 32 / dh;
    a.inv_g = 1.f / (float)a.G;
    a.J = P <= few ? few : 16;
    a.nt = (P + a.J - 1) / a.J;
    // Split the context for two workgroups on every compute unit, as long as each wave has a pair of pages.
    const long tiles = (long)a.B * a.H * a.nt;
    const int pages = (max_tokens + kPageSize - 1) / kPageSize;
    long want = std::max(1l, 2l * ncu / tiles);
    want = std::min(want, (long)(pages + 2 * kWaves - 1) / (2 * kWaves));
    want = std::min(want, (long)kPartSlots / tiles);
    a.nsplit = (int)std::max(1l, want);
    const bool split_out = a.out_lo != nullptr;
    auto go = [&](auto dhc) {
        constexpr int D = decltype(dhc)::value;
        if (dtype == DT_F16) launch<D, DT_F16, DT_F16>(a, stream);
        else if (dtype == DT_BF16) launch<D, DT_BF16, DT_BF16>(a, stream);
        else if (!split_out) launch<D, DT_F32, DT_F32>(a, stream);
        else launch<D, DT_F32, DT_SPLIT>(a, stream);
    };
    if (dh == 128) go(std::integral_constant<int, 128>{});
    else go(std::integral_constant<int, 64>{});
    LASER_HIP_CHECK(hipGetLastError());
    return LASER_OK;
}

}  // namespace laser
