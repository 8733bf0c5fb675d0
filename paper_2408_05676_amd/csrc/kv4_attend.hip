// Attention of a step's rows over the 4-bit paged cache (four_bit.h has its layout and how codes enter the matrix instructions).
//
// Query rows of one key/value head (row r of the step, query head j of the group: packed row r G + j) form tiles of 16. A wave
// walks its share of the context 32 tokens (two pages) at a time:
//   scores   S[t][row] = sum over groups c of s[t][c] (codes[t][c] . q[row][c]) + m[t][c] sum(q[row][c]): one matrix instruction
//            per group and page, K as the first operand, then two multiply-adds per score and group in fp32; the scales of four tokens
//            come out of the lane's row of sixteen by a lane broadcast that the multiply-add does itself. Queries are multiplied by a power of two of
//            their row so that fp16 holds them (bf16 exactly down to 2^-14 of the row's largest); fp32 queries are two planes.
//   softmax  against a reference m_ref per row that moves only when a score exceeds it by 8x: else nothing crosses lanes.
//   values   O[row][ch] += sum over t of (p[row][t] s[t][c]) codes[t][ch]: p s in fp16 (two planes where the output has more than eight bits) is the first
//            operand as it stands in the lanes, since the page order gives both products the same tokens per lane; plus p m, one more
//            instruction for all groups.
// Waves of a workgroup share a context, workgroups split it further when there are few rows; a second kernel joins the parts.
#include <algorithm>

#include "four_bit.h"

namespace laser {

constexpr int kAttendWaves = 4;
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

template <int DH>
struct Page {                                        // one page's registers of a lane
    uint32_t k[DH / 32], v[DH / 32], ksm, km, vsm;   // ksm, vsm: of token 4 g + r / NG, group r % NG; km: of token r, group g
    __device__ inline void load(const uint8_t* p, int lane) {
        constexpr int NG = DH / 32;
        const int sm = 4 * ((lane >> 4) * 4 * NG + (lane & (4 * NG - 1)));
        if constexpr (NG == 4) {
            const u32x4 a = *reinterpret_cast<const u32x4*>(p + lane * 16), b = *reinterpret_cast<const u32x4*>(p + page4_v(DH) + lane * 16);
#pragma unroll
            for (int i = 0; i < 4; ++i) { k[i] = a[i]; v[i] = b[i]; }
        } else {
            const u32x2 a = *reinterpret_cast<const u32x2*>(p + lane * 8), b = *reinterpret_cast<const u32x2*>(p + page4_v(DH) + lane * 8);
#pragma unroll
            for (int i = 0; i < 2; ++i) { k[i] = a[i]; v[i] = b[i]; }
        }
        ksm = *reinterpret_cast<const uint32_t*>(p + page4_ksm(DH) + sm);
        km = *reinterpret_cast<const uint32_t*>(p + page4_ksm(DH) + 4 * ((lane & 15) * NG + (lane >> 4 & (NG - 1))));
        vsm = *reinterpret_cast<const uint32_t*>(p + page4_vsm(DH) + sm);
    }
};

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

// IN: type of q; OUT: of the result; RT: 16-row tiles a workgroup takes.
template <int DH, int IN, int OUT, int RT>
__global__ __launch_bounds__(kAttendWaves * 64, RT >= 4 ? 1 : RT == 2 ? 2 : 3) void kv4_attend_kernel(AttendArgs a) {
    constexpr int NG = DH / 32, NT = DH / 16;        // groups, 16-channel tiles
    constexpr bool kTwoQ = IN == DT_F32, kTwoP = OUT != DT_BF16;
    constexpr int kStride = DH + 4;                  // of a row in LDS: four rows apart are sixteen banks apart
    __shared__ float sm_m[kAttendWaves][16], sm_l[kAttendWaves][16];
    __shared__ float sm_o[kAttendWaves][16 * kStride];
    const int ntb = (a.nt + RT - 1) / RT;
    const int h = blockIdx.x / ntb, tile0 = blockIdx.x % ntb * RT, b = blockIdx.y, split = blockIdx.z;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int r = lane & 15, g = lane >> 4;
    // (what the whole wave shares is kept in scalar registers: addresses, loop bounds and branches)
    const int slot = __builtin_amdgcn_readfirstlane(a.seqs.slot(b)), len = __builtin_amdgcn_readfirstlane(a.lens[slot]), cap = a.seqs.tokens(b);
    int nr = a.n_rows ? min(max(a.n_rows[b], 0), a.R) : a.R;
    nr = __builtin_amdgcn_readfirstlane(max(0, min(nr, cap - len)));      // (a length beyond the pages: rows that have no slot are left out)
    const int P = nr * a.G;                          // packed rows
    if (tile0 * 16 >= P || len < 0) return;

    // ---- which rows of the step each row sees: lane l works out row l's, by pointer doubling along the tree
    unsigned long long anc_l;
    if (a.row_anc) anc_l = a.row_anc[(size_t)b * a.R + min(lane, a.R - 1)];
    else if (!a.parent) anc_l = lane >= 63 ? ~0ull : (2ull << lane) - 1;
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

    Frag8 q[RT][NG], ql[kTwoQ ? RT : 1][NG];
    Frag8 qsum[RT];                                  // operand of the offsets: first input 8 g is group g, in two parts
    float cs[RT];
    unsigned long long anc[RT];
#pragma unroll
    for (int t = 0; t < RT; ++t) {
        const int pi = min((tile0 + t) * 16 + r, P - 1), row = pi / a.G, hq = h * a.G + pi % a.G;
        {
            const unsigned lo = __shfl((unsigned)anc_l, row), hi = __shfl((unsigned)(anc_l >> 32), row);
            anc[t] = ((unsigned long long)hi << 32) | lo;
        }
        const size_t qo = (size_t)b * a.q.seq + (size_t)row * a.q.row + (size_t)hq * a.q.head + 8 * g;
        float x[NG][8], mx = 0.f;
#pragma unroll
        for (int c = 0; c < NG; ++c) {
            load_elems<IN, 8>(a.q.p, qo + 32 * c, x[c]);
#pragma unroll
            for (int j = 0; j < 8; ++j) mx = fmaxf(mx, fabsf(x[c][j]));
        }
        mx = max_over_rows(mx);
        int e = 0;
        if (mx > 0.f && mx < INFINITY) { (void)frexpf(mx, &e); e = min(max(15 - e, -80), 100); }
        float own = 0.f;                             // the sum of group g, by lane (r, g)
#pragma unroll
        for (int c = 0; c < NG; ++c) {
            float s = 0.f, y[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) x[c][j] = ldexpf(x[c][j], e);
            q[t][c] = pack8(x[c]);
#pragma unroll
            for (int j = 0; j < 8; ++j) y[j] = (float)q[t][c].v[j];
            if constexpr (kTwoQ) {
#pragma unroll
                for (int j = 0; j < 8; ++j) x[c][j] -= y[j];
                ql[t][c] = pack8(x[c]);
#pragma unroll
                for (int j = 0; j < 8; ++j) s += (float)ql[t][c].v[j];
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) s += y[j];
            s = sum_over_rows(s) * kSumUnit;
            if (c == g) own = s;
        }
        {
            const _Float16 hi = (_Float16)own;
            const half2_t two = {hi, (_Float16)(own - (float)hi)};
            qsum[t].v4 = u32x4{__builtin_bit_cast(uint32_t, two), 0u, 0u, 0u};
        }
        cs[t] = ldexpf(a.scale_log2 / kSumUnit, -e);
    }

    float4_t acc[RT][NT], accm[RT];
    float m_ref[RT], l_run[RT], pf = 16.f;           // pf: factor of p s; smaller once a scale beyond 511 was met, so that fp16 holds 8 s pf
#pragma unroll
    for (int t = 0; t < RT; ++t) {
        m_ref[t] = -INFINITY;
        l_run[t] = 0.f;
        accm[t] = float4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int n = 0; n < NT; ++n) acc[t][n] = float4_t{0.f, 0.f, 0.f, 0.f};
    }

    // ---- this workgroup's pages [p0, p1), this wave's pairs of them
    const int npages = (len + nr + kPageSize - 1) / kPageSize;
    const int per = ((npages + a.nsplit - 1) / a.nsplit + 1) & ~1;
    const int p0 = split * per, p1 = min(npages, p0 + per);
    const uint8_t* base = a.pages + (size_t)h * page4_bytes(DH);
    const size_t page_step = (size_t)a.H * page4_bytes(DH);
    typedef const __attribute__((address_space(4))) int32_t* scalar_ints;       // (not written while the kernel runs)
    const scalar_ints bt = (scalar_ints)(a.block_table + (size_t)slot * a.mpps);
    auto page_at = [&](int p) { return base + (size_t)(unsigned)__builtin_amdgcn_readfirstlane(bt[min(p, p1 - 1)]) * page_step; };
    constexpr int kStep = 2 * kAttendWaves;

    // Two pages p and p + 1 of this wave. Every lane has the scores of its tokens 4 g .. 4 g + 3 of each page and its query row r.
    const float ks_unit = kCodeUnit * kSumUnit * (lane & 1 ? 1.f / 16.f : 1.f);      // odd groups: codes from bits 4..7
    auto pair_of_pages = [&](const Page<DH> (&pg)[2], int p) {
        // Scales of values: fp16 holds p s pf as long as s <= 511
        if (pf == 16.f && __any(sm_scale(pg[0].vsm) > 511.f || sm_scale(pg[1].vsm) > 511.f)) {
            pf = 1.f / 16.f;
#pragma unroll
            for (int t = 0; t < RT; ++t)
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int i = 0; i < 4; ++i) acc[t][n][i] *= 1.f / 256.f;
        }
        float x[RT][8];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const float ks = sm_scale(pg[u].ksm) * ks_unit;
            Frag8 km;
            km.v4 = u32x4{__builtin_amdgcn_perm(pg[u].km, pg[u].km, 0x07060706u), 0u, 0u, 0u};
            Frag8 kf[NG];
#pragma unroll
            for (int c = 0; c < NG; c += 2)
#pragma unroll
                for (int w = 0; w < 2; ++w) {
                    const uint32_t a0 = pg[u].k[c + w], a1 = a0 >> 8;
                    kf[c].w[2 * w] = a0 & kCodeLo;
                    kf[c].w[2 * w + 1] = a1 & kCodeLo;
                    kf[c + 1].w[2 * w] = a0 & kCodeHi;
                    kf[c + 1].w[2 * w + 1] = a1 & kCodeHi;
                }
#pragma unroll
            for (int t = 0; t < RT; ++t) {
                float4_t d[NG], s = mfma_16x16x32(km, qsum[t], float4_t{0.f, 0.f, 0.f, 0.f});
#pragma unroll
                for (int c = 0; c < NG; ++c) {
                    d[c] = float4_t{0.f, 0.f, 0.f, 0.f};
                    if constexpr (kTwoQ) d[c] = mfma_16x16x32(kf[c], ql[t][c], d[c]);
                    d[c] = mfma_16x16x32(kf[c], q[t][c], d[c]);
                }
                static_for<0, NG>([&](auto cc) {
                    constexpr int c = decltype(cc)::value;
                    static_for<0, 4>([&](auto ii) {
                        constexpr int i = decltype(ii)::value;
                        s[i] = fmaf(row_lane<i * NG + c>(ks), d[c][i], s[i]);
                    });
                });
#pragma unroll
                for (int i = 0; i < 4; ++i) x[t][4 * u + i] = s[i] * cs[t];
            }
        }
        if ((p + 2) * kPageSize > len) {             // slots behind the committed ones: along the row's own branch only
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                // the lane's four slots start rel behind the committed length: bits rel .. rel + 3 of the row's mask, ones below 0
                const int rel = p + u < p1 ? (p + u) * kPageSize + 4 * g - len : 64;
                const int up = min(max(rel, 0), 63), under = min(max(-rel, 0), 4);
#pragma unroll
                for (int t = 0; t < RT; ++t) {
                    const unsigned ahead = rel < 64 ? (unsigned)(anc[t] >> up) : 0u, behind = ((unsigned)anc[t] << under) | ((1u << under) - 1u);
                    const unsigned seen = rel >= 0 ? ahead : behind;
#pragma unroll
                    for (int i = 0; i < 4; ++i) x[t][4 * u + i] = (seen >> i) & 1u ? x[t][4 * u + i] : -INFINITY;
                }
            }
        } else if (p + 1 >= p1) {                    // an odd number of pages
#pragma unroll
            for (int t = 0; t < RT; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) x[t][4 + i] = -INFINITY;
        }

        // ---- weights p = 2^(x - m_ref), in place of x; their sums with the offsets
        Frag8 vm;                                    // offsets as an operand: column r < NG is group r (the others are not used)
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const uint32_t e0 = pg[u].vsm, e1 = row_ahead<NG>(e0), e2 = row_ahead<2 * NG>(e0), e3 = row_ahead<3 * NG>(e0);
            vm.w[2 * u] = __builtin_amdgcn_perm(e1, e0, 0x07060302u);
            vm.w[2 * u + 1] = __builtin_amdgcn_perm(e3, e2, 0x07060302u);
        }
#pragma unroll
        for (int t = 0; t < RT; ++t) {
            const float mx = fmaxf(fmaxf(fmaxf(x[t][0], x[t][1]), fmaxf(x[t][2], x[t][3])), fmaxf(fmaxf(x[t][4], x[t][5]), fmaxf(x[t][6], x[t][7])));
            if (__any(mx > m_ref[t] + 3.f)) {
                const float m_new = fmaxf(m_ref[t], max_over_rows(mx));
                const float alpha = m_ref[t] == m_new ? 1.f : __builtin_amdgcn_exp2f(m_ref[t] - m_new);
                l_run[t] *= alpha;
                m_ref[t] = m_new;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float al = __shfl(alpha, 4 * g + i);       // accumulator rows are 4 g + i
                    accm[t][i] *= al;
#pragma unroll
                    for (int n = 0; n < NT; ++n) acc[t][n][i] *= al;
                }
            }
            const float mu = m_ref[t] == -INFINITY ? 0.f : m_ref[t];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                x[t][i] = __builtin_amdgcn_exp2f(x[t][i] - mu);
                l_run[t] += x[t][i];
            }
            const Frag8 ph = pack8(x[t]);
            accm[t] = mfma_16x16x32(ph, vm, accm[t]);
            if constexpr (kTwoP) {
                float lo[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) lo[i] = x[t][i] - (float)ph.v[i];
                accm[t] = mfma_16x16x32(pack8(lo), vm, accm[t]);
            }
        }
        // ---- values: operand fragments of tokens 4 g .. 4 g + 3 of both pages
        const float vs0 = sm_scale(pg[0].vsm) * pf, vs1 = sm_scale(pg[1].vsm) * pf;
        static_for<0, NG>([&](auto cc) {
            constexpr int c = decltype(cc)::value;
            Frag8 va, vb;
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const uint32_t a0 = pg[u].v[c], a1 = a0 >> 8;
                va.w[2 * u] = a0 & kCodeLo;
                va.w[2 * u + 1] = a1 & kCodeLo;
                vb.w[2 * u] = a0 & kCodeHi;
                vb.w[2 * u + 1] = a1 & kCodeHi;
            }
#pragma unroll
            for (int t = 0; t < RT; ++t) {
                float ps[8];
                static_for<0, 4>([&](auto ii) {
                    constexpr int i = decltype(ii)::value;
                    ps[i] = row_lane<i * NG + c>(vs0) * x[t][i];
                    ps[4 + i] = row_lane<i * NG + c>(vs1) * x[t][4 + i];
                });
                const Frag8 pv = pack8(ps);
                acc[t][2 * c] = mfma_16x16x32(pv, va, acc[t][2 * c]);
                acc[t][2 * c + 1] = mfma_16x16x32(pv, vb, acc[t][2 * c + 1]);
                if constexpr (kTwoP) {
                    float lo[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) lo[i] = ps[i] - (float)pv.v[i];
                    const Frag8 pl = pack8(lo);
                    acc[t][2 * c] = mfma_16x16x32(pl, va, acc[t][2 * c]);
                    acc[t][2 * c + 1] = mfma_16x16x32(pl, vb, acc[t][2 * c + 1]);
                }
            }
        });
    };

    // Each turn first requests the next pair (past the end: the last page again) and the page numbers of the pair behind it.
    Page<DH> pa[2], pb[2];
    int p = p0 + 2 * wave;
    if (p < p1) {
        pa[0].load(page_at(p), lane);
        pa[1].load(page_at(p + 1), lane);
        const uint8_t *n0 = page_at(p + kStep), *n1 = page_at(p + kStep + 1);
        auto turn = [&](Page<DH> (&now)[2], Page<DH> (&next)[2]) {
            next[0].load(n0, lane);
            next[1].load(n1, lane);
            n0 = page_at(p + 2 * kStep);
            n1 = page_at(p + 2 * kStep + 1);
            pair_of_pages(now, p);
            p += kStep;
        };
        while (true) {
            turn(pa, pb);
            if (p >= p1) break;
            turn(pb, pa);
            if (p >= p1) break;
        }
    }

    // ---- join the waves, one tile at a time
    const float unit = kCodeUnit / pf;
#pragma unroll
    for (int t = 0; t < RT; ++t) {
        if ((tile0 + t) * 16 >= P) break;            // (the same for the whole workgroup)
        const float l = sum_over_rows(l_run[t]);
        if (t > 0) __syncthreads();                  // the tile before has been read
        if (g == 0) { sm_m[wave][r] = m_ref[t]; sm_l[wave][r] = l; }
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                sm_o[wave][(4 * g + i) * kStride + 16 * n + r] = fmaf(acc[t][n][i], n & 1 ? unit / 16.f : unit, __shfl(accm[t][i], 16 * g + n / 2));
        __syncthreads();
        for (int idx = threadIdx.x; idx < 4 * DH; idx += kAttendWaves * 64) {
            const int row = idx / (DH / 4), c = idx % (DH / 4) * 4;
            float M = sm_m[0][row], L = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int w = 1; w < kAttendWaves; ++w) M = fmaxf(M, sm_m[w][row]);
#pragma unroll
            for (int w = 0; w < kAttendWaves; ++w) {
                const float mw = sm_m[w][row], f = mw == M ? 1.f : __builtin_amdgcn_exp2f(mw - M);
                L += sm_l[w][row] * f;
#pragma unroll
                for (int j = 0; j < 4; ++j) o[j] += sm_o[w][row * kStride + c + j] * f;
            }
            if (a.nsplit == 1) {
                const int pi = (tile0 + t) * 16 + row;
                if (pi < P) {
                    const float inv = L == 0.f ? 0.f : 1.f / L;          // (nothing seen: 0; NaN stays)
#pragma unroll
                    for (int j = 0; j < 4; ++j) o[j] *= inv;
                    store_out<OUT>(a, (size_t)b * a.out.seq + (size_t)(pi / a.G) * a.out.row + (size_t)(h * a.G + pi % a.G) * a.out.head + c, o);
                }
            } else {
                float* part = a.part + ((((size_t)b * a.H + h) * a.nt + tile0 + t) * a.nsplit + split) * part_floats(DH);
                if (c == 0) { part[row] = M; part[16 + row] = L; }
                *reinterpret_cast<float4_t*>(part + 32 + row * DH + c) = float4_t{o[0], o[1], o[2], o[3]};
            }
        }
    }
}

// Joins the parts of a split context: a workgroup per tile.
template <int DH, int OUT>
__global__ __launch_bounds__(256) void kv4_join_kernel(AttendArgs a) {
    const int h = blockIdx.x / a.nt, tile = blockIdx.x % a.nt, b = blockIdx.y;
    const int slot = a.seqs.slot(b), len = a.lens[slot];
    int nr = a.n_rows ? min(max(a.n_rows[b], 0), a.R) : a.R;
    nr = max(0, min(nr, a.seqs.tokens(b) - len));
    const int P = nr * a.G;
    if (len < 0) return;
    const float* part = a.part + (((size_t)b * a.H + h) * a.nt + tile) * a.nsplit * part_floats(DH);
    for (int idx = threadIdx.x; idx < 4 * DH; idx += 256) {
        const int row = idx / (DH / 4), c = idx % (DH / 4) * 4, pi = tile * 16 + row;
        if (pi >= P) continue;
        float M = -INFINITY, L = 0.f;
        float4_t o = {0.f, 0.f, 0.f, 0.f};
        for (int s = 0; s < a.nsplit; ++s) M = fmaxf(M, part[(size_t)s * part_floats(DH) + row]);
        for (int s = 0; s < a.nsplit; ++s) {
            const float* ps = part + (size_t)s * part_floats(DH);
            const float ms = ps[row], f = ms == M ? 1.f : __builtin_amdgcn_exp2f(ms - M);
            const float4_t v = *reinterpret_cast<const float4_t*>(ps + 32 + row * DH + c);
            L += ps[16 + row] * f;
#pragma unroll
            for (int j = 0; j < 4; ++j) o[j] += v[j] * f;
        }
        const float inv = L == 0.f ? 0.f : 1.f / L;
        const float x[4] = {o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv};
        store_out<OUT>(a, (size_t)b * a.out.seq + (size_t)(pi / a.G) * a.out.row + (size_t)(h * a.G + pi % a.G) * a.out.head + c, x);
    }
}

template <int DH, int IN, int OUT>
static void launch(const AttendArgs& a, int rt, hipStream_t stream) {
    const dim3 grid((unsigned)(a.H * ((a.nt + rt - 1) / rt)), (unsigned)a.B, (unsigned)a.nsplit);
    if (rt == 1) hipLaunchKernelGGL((kv4_attend_kernel<DH, IN, OUT, 1>), grid, dim3(kAttendWaves * 64), 0, stream, a);
    else if (rt == 2) hipLaunchKernelGGL((kv4_attend_kernel<DH, IN, OUT, 2>), grid, dim3(kAttendWaves * 64), 0, stream, a);
    else hipLaunchKernelGGL((kv4_attend_kernel<DH, IN, OUT, 4>), grid, dim3(kAttendWaves * 64), 0, stream, a);
    if (a.nsplit > 1) hipLaunchKernelGGL((kv4_join_kernel<DH, OUT>), dim3((unsigned)(a.H * a.nt), (unsigned)a.B), dim3(256), 0, stream, a);
}

// max_tokens: the most slots any of the sequences may have by the host's bounds
int launch_kv4_attend(AttendArgs a, int dh, int dtype, int max_tokens, hipStream_t stream) {
    int ncu = 0;
    LASER_HIP_CHECK(hipDeviceGetAttribute(&ncu, hipDeviceAttributeMultiprocessorCount, 0));
    a.nt = (a.R * a.G + 15) / 16;
    const int rt = a.nt >= 4 ? 4 : a.nt >= 2 ? 2 : 1;
    const long groups = (long)a.B * a.H * ((a.nt + rt - 1) / rt), tiles = (long)a.B * a.H * a.nt;
    // Split the context until every compute unit has a few workgroups, as long as each has a pair of pages for every wave.
    const int pages = (max_tokens + kPageSize - 1) / kPageSize;
    long want = std::max(1l, 3l * ncu / groups);
    want = std::min(want, (long)(pages + 2 * kAttendWaves - 1) / (2 * kAttendWaves));
    want = std::min(want, (long)kPartSlots / tiles);
    a.nsplit = (int)std::max(1l, want);
    const bool split_out = a.out_lo != nullptr;
    auto go = [&](auto dhc) {
        constexpr int D = decltype(dhc)::value;
        if (dtype == DT_F16) launch<D, DT_F16, DT_F16>(a, rt, stream);
        else if (dtype == DT_BF16) launch<D, DT_BF16, DT_BF16>(a, rt, stream);
        else if (!split_out) launch<D, DT_F32, DT_F32>(a, rt, stream);
        else launch<D, DT_F32, DT_SPLIT>(a, rt, stream);
    };
    if (dh == 128) go(std::integral_constant<int, 128>{});
    else go(std::integral_constant<int, 64>{});
    LASER_HIP_CHECK(hipGetLastError());
    return LASER_OK;
}

}  // namespace laser
