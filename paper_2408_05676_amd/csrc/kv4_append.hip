// Keys and values of new rows into the 4-bit paged cache, with the rotary positions applied on the way (queries too), and back.
//
// Rotation (pairs i, i + D/2 of the first D channels): a' = a cos - b sin, b' = a sin + b cos. A group of 32 channels of a token
// and head, x = its values: s = f16((max - min) / 15), m = f16(min), c = round((x - m) / s) within 0..15 (s = 0: 0).
// Keys are rotated in 64 bits: products of 24-bit operands are exact there, so that a value half-way between two codes falls to the side that
// the formula puts it on, whatever the order of the operations.
// Bound: latency (a chain of length, page number, inputs, four shuffles, page) until there are some thousand rows, then the values' single bytes:
// a token's codes of a head lie in 64 places (four_bit.h). 64 tokens of 32 + 32 heads of 128 6.6 us (1.7 MB), 1024 rows of 8 + 32 heads 12.2 us (20 MB);
// with all of a head's channels in four threads, keys and values one after the other, 11.3 and 24.4. Reading back 4.3 and 4.7.
#include <algorithm>
#include <utility>
#include <vector>

#include "four_bit.h"

namespace laser {

// A thread takes two groups' worth of a quarter g of a token and head, keys, values or queries: channels 8 g .. 8 g + 7 of groups `half` and half + 2
// (0 and 1 at 64 channels) of keys and queries, whose rotary partners are then its own or its neighbour's; of values channels 4 g .. + 3 and
// 16 + 4 g .. + 3 of its groups, which are whole bytes of the page. Keys, values and queries are in different waves.
template <class T>
__device__ inline T quad_min(T x) { x = min(x, __shfl_xor(x, 1)); return min(x, __shfl_xor(x, 2)); }
template <class T>
__device__ inline T quad_max(T x) { x = max(x, __shfl_xor(x, 1)); return max(x, __shfl_xor(x, 2)); }

struct Group { float s, m; uint32_t sm; };
// lo, hi: the group's extremes. Values beyond fp16 saturate.
__device__ inline Group make_group(double lo, double hi) {
    const _Float16 s = f64_to_f16(fmin((hi - lo) / 15.0, 65504.0)), m = f64_to_f16(fmin(fmax(lo, -65504.0), 65504.0));
    return Group{(float)s, (float)m, (uint32_t)__builtin_bit_cast(uint16_t, s) | ((uint32_t)__builtin_bit_cast(uint16_t, m) << 16)};
}
// round((x - m) / s): in 32 bits unless that comes near a border between two codes
__device__ inline uint32_t code_of(double x, const Group& g, float inv) {
    const double d = x - (double)g.m;
    const float y = (float)d * inv;
    float n = rintf(y);
    if (fabsf(y - n) > 0.499f) n = (float)rint(d / (double)g.s);
    return g.s > 0.f ? (uint32_t)fminf(fmaxf(n, 0.f), 15.f) : 0u;
}

template <int DT, int N>
__device__ inline void load_sum(const Heads& h, size_t o, int n_part, int64_t part_stride, float (&x)[N]) {
    load_elems<DT, N>(h.p, o, x);
    if constexpr (DT == DT_F32)
        for (int s = 1; s < n_part; ++s) {
            float y[N];
            load_elems<DT, N>(h.p, o + s * part_stride, y);
#pragma unroll
            for (int i = 0; i < N; ++i) x[i] += y[i];
        }
}

template <class T>
__device__ inline T quad_or(T x) { x |= __shfl_xor(x, 1); return x | __shfl_xor(x, 2); }

template <int DH, int DT>
__global__ __launch_bounds__(256) void kv4_append_kernel(AppendArgs a) {
    constexpr int NG = DH / 32, SP = NG / 2, STEP = NG / 2;              // threads of a quarter; a thread's groups are half and half + STEP
    const int what = blockIdx.y;                                         // 0: keys, 1: values, 2: queries
    const int heads = what == 2 ? a.Hq : a.H;
    const long t = (long)blockIdx.x * 256 + threadIdx.x;
    const int g = threadIdx.x & 3, half = threadIdx.x >> 2 & (SP - 1);
    const long item = t / (4 * SP), row = item / heads;
    const int h = (int)(item % heads);
    if (row >= (long)a.B * a.R) return;                                  // (the threads of a head together, as every exit below)
    const int b = (int)(row / a.R), r = (int)(row % a.R);
    if (a.n_rows && r >= a.n_rows[b]) return;
    const int slot_id = a.seqs.slot(b);
    const int len = a.start >= 0 ? a.start : a.lens[slot_id];
    const int slot = len + r;
    if (what < 2 && (slot >= a.seqs.cap[slot_id] || slot < 0)) return;

    // ---- positions; (cos, sin) of the eight channels of a rotated group c: turn + 32 c (c counts within the first half of the rotated ones)
    const int hg = a.rope_dim / 64;                                      // groups in half of the rotated channels
    const float2* turn = nullptr;
    if (hg && what != 1) {
        int pos = slot;
        if (a.row_pos) pos = a.row_pos[row];
        else if (a.parent) {
            const int32_t* parent = a.parent + (size_t)b * (a.R - 1);
            pos = len;
            for (int i = r; i > 0; i = up_row(parent, i)) ++pos;
        }
        turn = a.rope + (size_t)min(max(pos, 0), a.max_pos - 1) * (32 * hg) + 8 * g;
    }
    // Rotates x[0], x[1] in T. hg == STEP: they are each other's partners. 64 of 128 channels: groups 0 and 1 are, which two threads hold.
    auto rotate = [&](auto& x) {
        typedef typename std::remove_reference<decltype(x[0][0])>::type T;
        if (!hg) return;
        float cs[16];
        const float2* tp = turn + (hg == STEP ? 32 * half : 0);
        load_elems<DT_F32, 8>(tp, 0, *reinterpret_cast<float(*)[8]>(cs));
        load_elems<DT_F32, 8>(tp + 4, 0, *reinterpret_cast<float(*)[8]>(cs + 8));
        if (hg == STEP) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const T p = x[0][j], q = x[1][j], co = cs[2 * j], si = cs[2 * j + 1];
                x[0][j] = p * co - q * si;
                x[1][j] = p * si + q * co;
            }
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const T mine = x[0][j], other = __shfl_xor((float)mine, 4), co = cs[2 * j], si = cs[2 * j + 1];      // (inputs: fp32 holds them)
                x[0][j] = half ? other * si + mine * co : mine * co - other * si;
            }
        }
    };
    const Heads& in = what == 0 ? a.k : what == 1 ? a.v : a.q;
    const size_t at = (size_t)b * in.seq + (size_t)r * in.row + (size_t)h * in.head;

    if (what == 2) {                                                     // ---- queries: in their own type
        const size_t to = (size_t)b * a.q_out.seq + (size_t)r * a.q_out.row + (size_t)h * a.q_out.head;
        float x[2][8];
#pragma unroll
        for (int c = 0; c < 2; ++c) load_sum<DT, 8>(in, at + 32 * (half + c * STEP) + 8 * g, a.n_part, a.part_stride, x[c]);
        rotate(x);
#pragma unroll
        for (int c = 0; c < 2; ++c) store_elems<DT, 8>(a.q_out.p, to + 32 * (half + c * STEP) + 8 * g, x[c]);
        return;
    }

    const int tp = slot % kPageSize;
    const int pg = a.block_table[(size_t)slot_id * a.mpps + slot / kPageSize];
    uint8_t* page = a.pages + ((size_t)pg * a.H + h) * page4_bytes(DH);
    // A key or value that is not finite makes the token's key NaN: every row that sees the token gets NaN from this head, and no
    // other row meets it. The codes and the values' scales stay finite, so that what a mask hides never enters a product.
    auto finite = [&](float (&x)[8]) {
        bool all = true;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const bool f = __builtin_isfinite(x[j]);
            all &= f;
            x[j] = f ? x[j] : 0.f;
        }
        return all;
    };
    float x[2][8];
    if (what == 0) {                                                     // ---- keys
        bool bad = false;
#pragma unroll
        for (int c = 0; c < 2; ++c) load_sum<DT, 8>(in, at + 32 * (half + c * STEP) + 8 * g, a.n_part, a.part_stride, x[c]);
        {
            const size_t va = (size_t)b * a.v.seq + (size_t)r * a.v.row + (size_t)h * a.v.head;
            float v[2][8];
#pragma unroll
            for (int c = 0; c < 2; ++c) load_sum<DT, 8>(a.v, va + 32 * (half + c * STEP) + 8 * g, a.n_part, a.part_stride, v[c]);
#pragma unroll
            for (int c = 0; c < 2; ++c) bad |= !finite(v[c]) | !finite(x[c]);
        }
        bad = quad_or((int)bad);
        if (SP == 2) bad |= (bool)__shfl_xor((int)bad, 4);
        double y[2][8];
#pragma unroll
        for (int c = 0; c < 2; ++c)
#pragma unroll
            for (int j = 0; j < 8; ++j) y[c][j] = x[c][j];
        rotate(y);
        uint32_t code[2][2] = {{0, 0}, {0, 0}};                          // of groups half, half + STEP: bits 0..3 of the bytes of two words
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            double lo = y[c][0], hi = y[c][0];
#pragma unroll
            for (int j = 1; j < 8; ++j) { lo = fmin(lo, y[c][j]); hi = fmax(hi, y[c][j]); }
            const Group gr = make_group(quad_min(lo), quad_max(hi));
            const float inv = 1.f / gr.s;
#pragma unroll
            for (int j = 0; j < 8; ++j) code[c][j >> 2] |= code_of(y[c][j], gr, inv) << (8 * code_byte(j & 3));
            if (g == 0) reinterpret_cast<uint32_t*>(page + page4_ksm(DH))[sm_index(DH, tp, half + c * STEP)] = bad ? (gr.sm & 0xFFFFu) | 0x7E000000u : gr.sm;
        }
        uint8_t* kp = page + (g * 16 + tp) * (DH / 8);
        if constexpr (SP == 1) {
            *reinterpret_cast<u32x2*>(kp) = u32x2{code[0][0] | (code[1][0] << 4), code[0][1] | (code[1][1] << 4)};
        } else {
            // words 0, 1 are groups 0 (low) and 1 (high), words 2, 3 groups 2 and 3: a thread keeps its own half and gets the other's codes
            const uint32_t o0 = __shfl_xor(half ? code[0][0] : code[1][0], 4), o1 = __shfl_xor(half ? code[0][1] : code[1][1], 4);
            const u32x2 w = half ? u32x2{o0 | (code[1][0] << 4), o1 | (code[1][1] << 4)} : u32x2{code[0][0] | (o0 << 4), code[0][1] | (o1 << 4)};
            *reinterpret_cast<u32x2*>(kp + 8 * half) = w;
        }
        return;
    }
    // ---- values
#pragma unroll
    for (int c = 0; c < 2; ++c) {
        const size_t vi = at + 32 * (half + c * STEP) + 4 * g;
        load_sum<DT, 4>(in, vi, a.n_part, a.part_stride, *reinterpret_cast<float(*)[4]>(&x[c][0]));
        load_sum<DT, 4>(in, vi + 16, a.n_part, a.part_stride, *reinterpret_cast<float(*)[4]>(&x[c][4]));
    }
    uint8_t* vp = page + page4_v(DH) + ((tp >> 2) * 16 + 4 * g) * (DH / 8) + code_byte(tp & 3);
#pragma unroll
    for (int c = 0; c < 2; ++c) {
        (void)finite(x[c]);
        const int grp = half + c * STEP;
        float lo = x[c][0], hi = x[c][0];
#pragma unroll
        for (int j = 1; j < 8; ++j) { lo = fminf(lo, x[c][j]); hi = fmaxf(hi, x[c][j]); }
        const Group gr = make_group((double)quad_min(lo), (double)quad_max(hi));
        const float inv = 1.f / gr.s;
#pragma unroll
        for (int e = 0; e < 4; ++e)
            vp[e * (DH / 8) + 4 * grp] = (uint8_t)(code_of((double)x[c][e], gr, inv) | (code_of((double)x[c][4 + e], gr, inv) << 4));
        if (g == 0) reinterpret_cast<uint32_t*>(page + page4_vsm(DH))[sm_index(DH, tp, grp)] = gr.sm;
    }
}

constexpr long kMaxThreads = (1l << 32) - 256;                           // of a launch's dimension

int launch_kv4_append(const AppendArgs& a, int dh, int dtype, hipStream_t stream) {
    const long threads = (long)a.B * a.R * 4 * (dh / 64) * std::max(a.H, a.Hq);
    LASER_REQUIRE(threads <= kMaxThreads, LASER_E_LIMIT, "%ld rows and heads in one call", threads / (4 * (dh / 64)));
    const dim3 grid((unsigned)((threads + 255) / 256), a.Hq > 0 ? 3 : 2);
    auto go = [&](auto dhc) {
        constexpr int D = decltype(dhc)::value;
        if (dtype == DT_F16) hipLaunchKernelGGL((kv4_append_kernel<D, DT_F16>), grid, dim3(256), 0, stream, a);
        else if (dtype == DT_BF16) hipLaunchKernelGGL((kv4_append_kernel<D, DT_BF16>), grid, dim3(256), 0, stream, a);
        else hipLaunchKernelGGL((kv4_append_kernel<D, DT_F32>), grid, dim3(256), 0, stream, a);
    };
    if (dh == 128) go(std::integral_constant<int, 128>{});
    else go(std::integral_constant<int, 64>{});
    LASER_HIP_CHECK(hipGetLastError());
    return LASER_OK;
}

// ------------------------------------------------------------------------------------------------
// The values that cached tokens stand for: threads as in the kernel above.
struct ReadArgs {
    SeqList seqs;
    const int32_t* lens; const int32_t* block_table;
    const uint8_t* pages;
    Heads k, v;
    int B, n, H, mpps, start;
};

template <int DH, int DT>
__global__ __launch_bounds__(256) void kv4_read_kernel(ReadArgs a) {
    constexpr int NG = DH / 32, SP = NG / 2;
    const long t = (long)blockIdx.x * 256 + threadIdx.x;
    const int g = threadIdx.x & 3, half = threadIdx.x >> 2 & (SP - 1);
    const long item = t / (4 * SP), row = item / a.H;
    const int h = (int)(item % a.H);
    if (row >= (long)a.B * a.n) return;
    const int b = (int)(row / a.n), r = (int)(row % a.n);
    const int id = a.seqs.slot(b);
    const int slot = (a.start >= 0 ? a.start : a.lens[id]) + r;
    if (slot < 0 || slot >= a.seqs.cap[id]) return;
    const int tp = slot % kPageSize;
    const int pg = a.block_table[(size_t)id * a.mpps + slot / kPageSize];
    const uint8_t* page = a.pages + ((size_t)pg * a.H + h) * page4_bytes(DH);
    if (blockIdx.y == 0) {                           // keys of groups 2 half (low) and 2 half + 1 (high)
        const u32x2 w = *reinterpret_cast<const u32x2*>(page + (g * 16 + tp) * (DH / 8) + 8 * half);
        const size_t ko = (size_t)b * a.k.seq + (size_t)r * a.k.row + (size_t)h * a.k.head + 64 * half + 8 * g;
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            const uint32_t sm = reinterpret_cast<const uint32_t*>(page + page4_ksm(DH))[sm_index(DH, tp, 2 * half + c)];
            float x[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] = fmaf(sm_scale(sm), (float)((w[j >> 2] >> (8 * code_byte(j & 3) + 4 * c)) & 15u), sm_offset(sm));
            store_elems<DT, 8>(a.k.p, ko + 32 * c, x);
        }
        return;
    }
    const uint8_t* vp = page + page4_v(DH) + ((tp >> 2) * 16 + 4 * g) * (DH / 8) + code_byte(tp & 3);
    const size_t vo = (size_t)b * a.v.seq + (size_t)r * a.v.row + (size_t)h * a.v.head + 64 * half + 4 * g;
#pragma unroll
    for (int c = 0; c < 2; ++c) {
        const uint32_t sm = reinterpret_cast<const uint32_t*>(page + page4_vsm(DH))[sm_index(DH, tp, 2 * half + c)];
        float u[4], w[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const uint32_t byte = vp[e * (DH / 8) + 4 * (2 * half + c)];
            u[e] = fmaf(sm_scale(sm), (float)(byte & 15u), sm_offset(sm));
            w[e] = fmaf(sm_scale(sm), (float)(byte >> 4), sm_offset(sm));
        }
        store_elems<DT, 4>(a.v.p, vo + 32 * c, u);
        store_elems<DT, 4>(a.v.p, vo + 32 * c + 16, w);
    }
}

// laser_kv_commit_tree's move of the accepted branch (see kv_compact_kernel): a lane owns one key byte and one value byte of a
// token's dh / 2, four of them a word of sm, and moves them branch position by branch position.
__global__ void kv4_compact_kernel(uint8_t* pages, const int32_t* block_table, const int32_t* len, const int32_t* cap, const int32_t* seq_ids,
                                   const int32_t* accept_len, const int32_t* accept_path, int K, int H, int dh, int mpps, int n_pages) {
    const int h = blockIdx.x, l = blockIdx.y, b = blockIdx.z, c = threadIdx.x, ng = dh / 32;
    const int id = seq_ids[b], len0 = len[id], have = cap[id];
    int acc = accept_len[b];
    acc = acc < 0 ? 0 : (acc > K ? K : acc);
    const int32_t* bt = block_table + (size_t)id * mpps;
    const int kb = dh / 8;                                  // bytes a lane of the page holds
    for (int j = 0; j < acc; ++j) {
        const int i = accept_path[(size_t)b * K + j];
        if (i < j || i >= K) break;
        if (i == j) continue;
        const int src = len0 + 1 + i, dst = len0 + 1 + j, st = src % kPageSize, dt = dst % kPageSize;
        if (src >= have) break;                             // (dst < src < later sources)
        const uint8_t* sp = pages + (((size_t)l * n_pages + bt[src / kPageSize]) * H + h) * page4_bytes(dh);
        uint8_t* dp = pages + (((size_t)l * n_pages + bt[dst / kPageSize]) * H + h) * page4_bytes(dh);
        if (c < dh / 2) {
            dp[(c / kb * 16 + dt) * kb + c % kb] = sp[(c / kb * 16 + st) * kb + c % kb];
            const int r = c / ng, p = c % ng;
            dp[page4_v(dh) + ((dt >> 2) * 16 + r) * kb + 4 * p + code_byte(dt & 3)] = sp[page4_v(dh) + ((st >> 2) * 16 + r) * kb + 4 * p + code_byte(st & 3)];
        }
        if (c < 2 * ng) {
            const int o = c < ng ? page4_ksm(dh) : page4_vsm(dh);
            *reinterpret_cast<uint32_t*>(dp + o + 4 * sm_index(dh, dt, c % ng)) = *reinterpret_cast<const uint32_t*>(sp + o + 4 * sm_index(dh, st, c % ng));
        }
    }
}

int launch_kv4_compact(const KV* kv, const int32_t* ids_dev, const int32_t* accept_len, const int32_t* accept_path, int B, int K, hipStream_t stream) {
    hipLaunchKernelGGL(kv4_compact_kernel, dim3(kv->d.n_heads, kv->d.n_layers, B), dim3(64), 0, stream, kv->pages4, kv->block_table, kv->len, kv->cap,
                       ids_dev, accept_len, accept_path, K, kv->d.n_heads, kv->d.head_dim, kv->d.max_pages_per_seq, kv->d.n_pages);
    LASER_HIP_CHECK(hipGetLastError());
    return LASER_OK;
}

__global__ void rope_table4_kernel(float2* tab, int max_pos, int half, double base) {
    const size_t i = (size_t)blockIdx.x * blockDim.x + threadIdx.x;
    if (i >= (size_t)max_pos * half) return;
    const double ang = (double)(i / half) * pow(base, -(double)(i % half) / (double)half);
    tab[i] = make_float2((float)cos(ang), (float)sin(ang));
}

// ---- checks that the three calls share -----------------------------------------------------------
static int check_four_bit(const KV* kv, int layer, const int32_t* seq_ids, int B, int dtype) {
    LASER_REQUIRE(kv != nullptr, LASER_E_INVALID_ARG, "kv is NULL");
    LASER_REQUIRE(kv->pages4 != nullptr, LASER_E_SHAPE, "the cache was not made by laser_kv_create_4bit");
    LASER_REQUIRE(layer >= 0 && layer < kv->d.n_layers, LASER_E_INVALID_ARG, "layer %d out of range", layer);
    LASER_REQUIRE(dtype == LASER_F16 || dtype == LASER_BF16 || dtype == LASER_F32, LASER_E_INVALID_ARG, "unknown dtype %d", dtype);
    LASER_REQUIRE(B >= 0 && B <= kv->d.max_seqs, LASER_E_INVALID_ARG, "B %d outside 0..max_seqs %d", B, kv->d.max_seqs);
    LASER_REQUIRE(B == 0 || seq_ids, LASER_E_INVALID_ARG, "seq_ids is NULL");
    std::vector<char> seen(kv->d.max_seqs, 0);
    for (int b = 0; b < B; ++b) {
        const int s = seq_ids[b];
        LASER_REQUIRE(s >= 0 && s < kv->d.max_seqs, LASER_E_INVALID_ARG, "sequence slot %d out of range", s);
        LASER_REQUIRE(!seen[s], LASER_E_INVALID_ARG, "sequence slot %d appears twice", s);
        seen[s] = 1;
    }
    return LASER_OK;
}

static int check_heads(const laser_heads* t, const char* name, int dtype) {
    LASER_REQUIRE(t && t->data, LASER_E_INVALID_ARG, "%s is NULL", name);
    LASER_REQUIRE(t->seq >= 0 && t->row >= 0 && t->head >= 0, LASER_E_INVALID_ARG, "%s: negative stride", name);
    LASER_REQUIRE((uintptr_t)t->data % dtype_bytes(dtype) == 0, LASER_E_INVALID_ARG, "%s is not aligned to its elements", name);
    return LASER_OK;
}

// Results: no two heads of dh elements may share memory.
static int check_apart(const laser_heads* t, const char* name, long B, long R, long H, int dh) {
    std::pair<int64_t, long> dims[3] = {{t->seq, B}, {t->row, R}, {t->head, H}};
    std::sort(dims, dims + 3);
    int64_t extent = dh;                                                 // of what the strides so far reach over
    bool nested = true;
    for (const auto& [stride, n] : dims) {
        if (n <= 1) continue;
        nested &= stride >= extent;
        extent += stride * (n - 1);
    }
    if (nested) return LASER_OK;
    std::vector<int64_t> at;                                             // strides that interleave: by looking
    if (B * R * H <= 1l << 22) {
        for (long b = 0; b < B; ++b)
            for (long r = 0; r < R; ++r)
                for (long h = 0; h < H; ++h) at.push_back(b * t->seq + r * t->row + h * t->head);
        std::sort(at.begin(), at.end());
    }
    bool apart = !at.empty();
    for (size_t i = 1; i < at.size(); ++i) apart &= at[i] - at[i - 1] >= dh;
    LASER_REQUIRE(apart, LASER_E_INVALID_ARG, "%s: rows or heads overlap (strides %lld, %lld, %lld)", name, (long long)t->seq, (long long)t->row, (long long)t->head);
    return LASER_OK;
}

static Heads heads_from(const laser_heads* t, int b0, int dtype) {
    if (!t || !t->data) return Heads{nullptr, 0, 0, 0};
    return Heads{(char*)t->data + (size_t)b0 * t->seq * dtype_bytes(dtype), t->seq, t->row, t->head};
}

static void fill_seqs(const KV* kv, const int32_t* ids, int B, SeqList& s) {
    s.dev = nullptr;
    s.cap = kv->cap;
    std::copy(ids, ids + B, s.id);
}

static int check_rows(const KV* kv, const int32_t* seq_ids, int B, int R) {
    LASER_REQUIRE(R >= 1 && R <= LASER_MAX_DRAFT + 1, LASER_E_INVALID_ARG, "R %d outside 1..%d", R, LASER_MAX_DRAFT + 1);
    for (int b = 0; b < B; ++b) {
        const int s = seq_ids[b];
        LASER_REQUIRE(kv->h_len_ub[s] + R <= kv->h_npages[s] * kPageSize, LASER_E_OOM_PAGES, "slot %d: length bound %d + %d rows exceeds the %d tokens reserved",
                      s, kv->h_len_ub[s], R, kv->h_npages[s] * kPageSize);
    }
    return LASER_OK;
}

static uint8_t* layer_pages(const KV* kv, int layer) {
    return kv->pages4 + (size_t)layer * kv->d.n_pages * kv->d.n_heads * page4_bytes(kv->d.head_dim);
}

int kv4_import(KV* kv, int seq, int layer, const uint16_t* k, const uint16_t* v, int n_tokens, hipStream_t stream) {
    const int64_t row = (int64_t)kv->d.n_heads * kv->d.head_dim;
    AppendArgs a{};
    fill_seqs(kv, &seq, 1, a.seqs);
    a.block_table = kv->block_table;
    a.pages = layer_pages(kv, layer);
    a.k = Heads{(void*)k, 0, row, kv->d.head_dim};
    a.v = Heads{(void*)v, 0, row, kv->d.head_dim};
    a.B = 1; a.R = n_tokens; a.H = kv->d.n_heads; a.mpps = kv->d.max_pages_per_seq; a.n_part = 1;
    return launch_kv4_append(a, kv->d.head_dim, DT_F16, stream);
}

}  // namespace laser

using namespace laser;

extern "C" int laser_rope_table(float* table, int max_pos, int rope_dim, double base, void* stream) {
    LASER_REQUIRE(table != nullptr, LASER_E_INVALID_ARG, "table is NULL");
    LASER_REQUIRE(max_pos > 0 && rope_dim > 0 && rope_dim % 2 == 0 && base > 0.0, LASER_E_INVALID_ARG, "bad size or base");
    const size_t n = (size_t)max_pos * (rope_dim / 2);
    LASER_REQUIRE(n <= kMaxThreads, LASER_E_LIMIT, "table too large");
    hipLaunchKernelGGL(rope_table4_kernel, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, (hipStream_t)stream, (float2*)table, max_pos, rope_dim / 2, base);
    LASER_HIP_CHECK(hipGetLastError());
    return LASER_OK;
}

extern "C" int laser_kv_append(laser_kv* h, int layer, const int32_t* seq_ids, const int32_t* n_rows, const int32_t* tree_parent,
                               int B, int R, int dtype, const laser_heads* k, const laser_heads* v, const laser_heads* q,
                               const laser_heads* q_out, int n_heads, const float* rope, int rope_dim, int max_pos, void* stream) {
    KV* kv = reinterpret_cast<KV*>(h);
    int rc = check_four_bit(kv, layer, seq_ids, B, dtype);
    if (rc) return rc;
    if ((rc = check_rows(kv, seq_ids, B, R))) return rc;
    if (B == 0) return LASER_OK;
    if ((rc = check_heads(k, "k", dtype)) || (rc = check_heads(v, "v", dtype))) return rc;
    LASER_REQUIRE(n_heads >= 0 && n_heads <= (1 << 20), LASER_E_INVALID_ARG, "n_heads %d out of range", n_heads);
    if (n_heads > 0 && ((rc = check_heads(q, "q", dtype)) || (rc = check_heads(q_out, "q_out", dtype)) || (rc = check_apart(q_out, "q_out", B, R, n_heads, kv->d.head_dim)))) return rc;
    const int dh = kv->d.head_dim;
    LASER_REQUIRE(rope_dim == 0 || rope_dim == dh || (rope_dim == 64 && dh == 128), LASER_E_SHAPE, "rope_dim %d: 0, 64 or head_dim", rope_dim);
    if (rope_dim) {
        LASER_REQUIRE(rope != nullptr && (uintptr_t)rope % 8 == 0, LASER_E_INVALID_ARG, "rope is NULL or not aligned to 8 bytes");
        LASER_REQUIRE(max_pos > 0, LASER_E_INVALID_ARG, "max_pos must be positive");
        for (int b = 0; b < B; ++b)
            LASER_REQUIRE(kv->h_len_ub[seq_ids[b]] + R <= max_pos, LASER_E_LIMIT, "slot %d: position would exceed max_pos %d", seq_ids[b], max_pos);
    }
    for (int b0 = 0; b0 < B; b0 += kSeqChunk) {
        AppendArgs a{};
        a.B = std::min(kSeqChunk, B - b0);
        fill_seqs(kv, seq_ids + b0, a.B, a.seqs);
        a.lens = kv->len; a.block_table = kv->block_table;
        a.pages = layer_pages(kv, layer);
        a.n_rows = n_rows ? n_rows + b0 : nullptr;
        a.parent = tree_parent && R > 1 ? tree_parent + (size_t)b0 * (R - 1) : nullptr;
        a.rope = (const float2*)rope;
        a.k = heads_from(k, b0, dtype); a.v = heads_from(v, b0, dtype);
        if (n_heads > 0) { a.q = heads_from(q, b0, dtype); a.q_out = heads_from(q_out, b0, dtype); }
        a.R = R; a.H = kv->d.n_heads; a.Hq = n_heads; a.mpps = kv->d.max_pages_per_seq; a.start = -1;
        a.rope_dim = rope_dim; a.max_pos = max_pos; a.n_part = 1;
        if ((rc = launch_kv4_append(a, dh, dtype, (hipStream_t)stream))) return rc;
    }
    for (int b = 0; b < B; ++b) kv->h_last_rows[seq_ids[b]] = R;         // what a commit may add
    return LASER_OK;
}

extern "C" int laser_kv_attend(laser_kv* h, int layer, const int32_t* seq_ids, const int32_t* n_rows, const int32_t* tree_parent,
                               int B, int R, int n_heads, int dtype, const laser_heads* q, float scale, const laser_heads* out, void* stream) {
    KV* kv = reinterpret_cast<KV*>(h);
    int rc = check_four_bit(kv, layer, seq_ids, B, dtype);
    if (rc) return rc;
    if ((rc = check_rows(kv, seq_ids, B, R))) return rc;
    if (B == 0) return LASER_OK;
    if ((rc = check_heads(q, "q", dtype)) || (rc = check_heads(out, "out", dtype))) return rc;
    LASER_REQUIRE(n_heads > 0 && n_heads % kv->d.n_heads == 0, LASER_E_SHAPE, "n_heads %d is not a multiple of the cache's %d", n_heads, kv->d.n_heads);
    if ((rc = check_apart(out, "out", B, R, n_heads, kv->d.head_dim))) return rc;
    LASER_REQUIRE(n_heads / kv->d.n_heads <= 256, LASER_E_LIMIT, "more than 256 query heads per key/value head");
    LASER_REQUIRE(std::isfinite(scale * 1.44269504f), LASER_E_INVALID_ARG, "scale is not finite, or too large");
    for (int b0 = 0; b0 < B; b0 += kSeqChunk) {
        AttendArgs a{};
        a.B = std::min(kSeqChunk, B - b0);
        fill_seqs(kv, seq_ids + b0, a.B, a.seqs);
        int most = 0;
        for (int b = b0; b < b0 + a.B; ++b) most = std::max(most, kv->h_len_ub[seq_ids[b]] + R);
        a.lens = kv->len; a.block_table = kv->block_table;
        a.pages = layer_pages(kv, layer);
        a.n_rows = n_rows ? n_rows + b0 : nullptr;
        a.parent = tree_parent && R > 1 ? tree_parent + (size_t)b0 * (R - 1) : nullptr;
        a.q = heads_from(q, b0, dtype); a.out = heads_from(out, b0, dtype);
        a.part = kv->part4;
        a.R = R; a.H = kv->d.n_heads; a.G = n_heads / kv->d.n_heads; a.mpps = kv->d.max_pages_per_seq;
        a.scale_log2 = scale * 1.44269504f;
        if ((rc = launch_kv4_attend(a, kv->d.head_dim, dtype, most, (hipStream_t)stream))) return rc;
    }
    return LASER_OK;
}

extern "C" int laser_kv_read(laser_kv* h, int layer, const int32_t* seq_ids, int B, int start, int n, int dtype, const laser_heads* k,
                             const laser_heads* v, void* stream) {
    KV* kv = reinterpret_cast<KV*>(h);
    int rc = check_four_bit(kv, layer, seq_ids, B, dtype);
    if (rc) return rc;
    LASER_REQUIRE(start >= -1 && n >= 0, LASER_E_INVALID_ARG, "start %d, n %d", start, n);
    for (int b = 0; b < B; ++b) {
        const int s = seq_ids[b], first = start >= 0 ? start : kv->h_len_ub[s];
        LASER_REQUIRE((long)first + n <= (long)kv->h_npages[s] * kPageSize, LASER_E_OOM_PAGES, "slot %d: tokens %d .. %ld exceed the %d reserved", s, first,
                      (long)first + n, kv->h_npages[s] * kPageSize);
    }
    if (B == 0 || n == 0) return LASER_OK;
    if ((rc = check_heads(k, "k", dtype)) || (rc = check_heads(v, "v", dtype))) return rc;
    const int H = kv->d.n_heads, dh = kv->d.head_dim;
    if ((rc = check_apart(k, "k", B, n, H, dh)) || (rc = check_apart(v, "v", B, n, H, dh))) return rc;
    LASER_REQUIRE(k->data != v->data, LASER_E_INVALID_ARG, "k and v are the same memory");
    for (int b0 = 0; b0 < B; b0 += kSeqChunk) {
        ReadArgs a{};
        a.B = std::min(kSeqChunk, B - b0);
        fill_seqs(kv, seq_ids + b0, a.B, a.seqs);
        a.lens = kv->len; a.block_table = kv->block_table;
        a.pages = layer_pages(kv, layer);
        a.k = heads_from(k, b0, dtype); a.v = heads_from(v, b0, dtype);
        a.n = n; a.H = kv->d.n_heads; a.mpps = kv->d.max_pages_per_seq; a.start = start;
        const long threads = (long)a.B * n * a.H * 4 * (kv->d.head_dim / 64);
        LASER_REQUIRE(threads <= kMaxThreads, LASER_E_LIMIT, "%ld tokens and heads in one call", threads / (4 * (kv->d.head_dim / 64)));
        const dim3 grid((unsigned)((threads + 255) / 256), 2);
        auto go = [&](auto dhc) {
            constexpr int D = decltype(dhc)::value;
            if (dtype == DT_F16) hipLaunchKernelGGL((kv4_read_kernel<D, DT_F16>), grid, dim3(256), 0, (hipStream_t)stream, a);
            else if (dtype == DT_BF16) hipLaunchKernelGGL((kv4_read_kernel<D, DT_BF16>), grid, dim3(256), 0, (hipStream_t)stream, a);
            else hipLaunchKernelGGL((kv4_read_kernel<D, DT_F32>), grid, dim3(256), 0, (hipStream_t)stream, a);
        };
        if (kv->d.head_dim == 128) go(std::integral_constant<int, 128>{});
        else go(std::integral_constant<int, 64>{});
        LASER_HIP_CHECK(hipGetLastError());
    }
    return LASER_OK;
}
