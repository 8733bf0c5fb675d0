// What the kernels on 4-bit weights and caches share: element types, rows of heads, how codes lie in words, and the cache's pages.
//
// An element held in four bits is a code c = 0..15 with a scale s and an offset m (fp16, "sm" below: s in the low half of 32
// bits, m in the high half) that a group of elements shares: it stands for m + s c.
//
// Codes go into the matrix instructions without a conversion: a code masked out of its word is the fp16 number c 2^-24 (bits
// 0..3) or c 2^-20 (bits 4..7), a subnormal; the power of two is paid for once,
// in a factor that is applied anyway. A 32-bit word of codes therefore gives, with four ANDs and one shift, two operand
// registers of one fragment (bits 0..3 of its four bytes) and two of another (bits 4..7), the second scaled by 16.
// Products are exact, but an instruction cuts its 32 off some 2^-24 below the largest, and goes by exponents there, of which a subnormal
// has that of 2^-14: products of bits 0..3 count as 2^7 to 2^10 times larger than they are, those of bits 4..7 as 2^3 to 2^6 times. Measured, relative
// to a sum of weights e^N(0, 1.4) times codes: 10^-6 for bits 0..3, below 10^-7 for bits 4..7, where two more shifts a word bring all codes.
#pragma once

#include "mfma.h"
#include "state.h"

namespace laser {

constexpr int kCacheGroup = 32;                      // channels of a token and head that share a scale in the cache
constexpr uint32_t kCodeLo = 0x000F000Fu, kCodeHi = 0x00F000F0u;
constexpr float kCodeUnit = 16777216.f;              // 2^24: what a code masked out of bits 0..3 has to be multiplied by

// Where the code of element j = 0..3 of a word lies: byte (0, 2, 1, 3)[j], so that (word >> 8 (j / 2)) & mask holds elements
// 2 (j / 2) and 2 (j / 2) + 1 in its two halves.
__host__ __device__ constexpr int code_byte(int j) { return (j >> 1) + 2 * (j & 1); }

// One page of one head in the 4-bit cache: 16 tokens' key codes (8 dh bytes), value codes (8 dh), the keys' sm (2 dh), the values' sm:
// 20 dh bytes at ((l * n_pages + page) * H + h) * 20 dh. Codes lie as the 64 lanes of a wave hold a matrix operand, dh / 8
// bytes a lane; lane (r = lane % 16, g = lane / 16) holds
//   keys    token r, channels 8 g .. 8 g + 7 of each group: groups 2 p (low) and 2 p + 1 (high) in words 2 p (channels 0..3 of
//           the eight) and 2 p + 1 (4..7)
//   values  tokens 4 g .. 4 g + 3 of channels 32 p + r (low) and 32 p + 16 + r (high) in word p
// and a page's sm are [token / 4][group][token % 4]: those of a lane's four tokens and one group are 16 bytes, those of all groups a row of lanes.
__host__ __device__ constexpr int page4_bytes(int dh) { return 20 * dh; }
__host__ __device__ constexpr int page4_v(int dh) { return 8 * dh; }
__host__ __device__ constexpr int page4_ksm(int dh) { return 16 * dh; }
__host__ __device__ constexpr int page4_vsm(int dh) { return 18 * dh; }
// place of token t, group c among a page's sm
__host__ __device__ constexpr int sm_index(int dh, int t, int c) { return (t >> 2) * (dh / 8) + c * 4 + (t & 3); }

// [host] ids of up to kSeqChunk sequences ride in the kernel arguments: nothing is staged, and a captured launch keeps its own.
// cap: tokens that a slot's pages hold as the launch runs; slots beyond are neither read nor written, whatever the length on the device says.
constexpr int kSeqChunk = 256;
struct SeqList {
    const int32_t* dev;                              // ids on the device instead (a step of the model)
    const int32_t* cap;                              // [dev] of all slots (KV::cap)
    int32_t id[kSeqChunk];
    __device__ int slot(int b) const { return dev ? dev[b] : id[b]; }
};

struct Heads { void* p; int64_t seq, row, head; };   // element (b, r, h, c) at p + b seq + r row + h head + c

enum { DT_F16 = LASER_F16, DT_BF16 = LASER_BF16, DT_F32 = LASER_F32, DT_SPLIT = 3 };   // DT_SPLIT: two fp16 planes, out only
inline size_t dtype_bytes(int dt) { return dt == DT_F32 ? 4 : 2; }

typedef unsigned u32x4_a2 __attribute__((ext_vector_type(4), aligned(2)));   // rows are aligned to their elements only
typedef unsigned u32x2_a2 __attribute__((ext_vector_type(2), aligned(2)));
typedef float f32x4_a4 __attribute__((ext_vector_type(4), aligned(4)));

// N = 4 or 8 consecutive elements at element offset o
template <int DT, int N>
__device__ inline void load_elems(const void* p, size_t o, float (&x)[N]) {
    if constexpr (DT == DT_F32) {
#pragma unroll
        for (int i = 0; i < N / 4; ++i) {
            const f32x4_a4 t = reinterpret_cast<const f32x4_a4*>((const float*)p + o)[i];
#pragma unroll
            for (int j = 0; j < 4; ++j) x[4 * i + j] = t[j];
        }
    } else {
        uint32_t w[N / 2];
        if constexpr (N == 8) {
            const u32x4_a2 t = *reinterpret_cast<const u32x4_a2*>((const uint16_t*)p + o);
            w[0] = t[0]; w[1] = t[1]; w[2] = t[2]; w[3] = t[3];
        } else {
            const u32x2_a2 t = *reinterpret_cast<const u32x2_a2*>((const uint16_t*)p + o);
            w[0] = t[0]; w[1] = t[1];
        }
#pragma unroll
        for (int i = 0; i < N / 2; ++i) {
            x[2 * i] = DT == DT_BF16 ? __uint_as_float(w[i] << 16) : f16_to_f32((uint16_t)w[i]);
            x[2 * i + 1] = DT == DT_BF16 ? __uint_as_float(w[i] & 0xFFFF0000u) : f16_to_f32((uint16_t)(w[i] >> 16));
        }
    }
}

__device__ inline uint16_t f32_to_bf16(float f) {           // round to nearest even; NaN stays NaN
    const uint32_t u = __float_as_uint(f);
    if ((u & 0x7FFFFFFFu) > 0x7F800000u) return (uint16_t)((u >> 16) | 0x40u);
    return (uint16_t)((u + 0x7FFFu + ((u >> 16) & 1u)) >> 16);
}

template <int DT, int N>
__device__ inline void store_elems(void* p, size_t o, const float (&x)[N]) {
    if constexpr (DT == DT_F32) {
#pragma unroll
        for (int i = 0; i < N / 4; ++i) {
            f32x4_a4 t;
#pragma unroll
            for (int j = 0; j < 4; ++j) t[j] = x[4 * i + j];
            reinterpret_cast<f32x4_a4*>((float*)p + o)[i] = t;
        }
    } else {
        uint32_t w[N / 2];
#pragma unroll
        for (int i = 0; i < N / 2; ++i) {
            const uint32_t a = DT == DT_BF16 ? f32_to_bf16(x[2 * i]) : f32_to_f16(x[2 * i]);
            const uint32_t b = DT == DT_BF16 ? f32_to_bf16(x[2 * i + 1]) : f32_to_f16(x[2 * i + 1]);
            w[i] = a | (b << 16);
        }
        if constexpr (N == 8) {
            u32x4_a2 t = {w[0], w[1], w[2], w[3]};
            *reinterpret_cast<u32x4_a2*>((uint16_t*)p + o) = t;
        } else {
            u32x2_a2 t = {w[0], w[1]};
            *reinterpret_cast<u32x2_a2*>((uint16_t*)p + o) = t;
        }
    }
}

// By way of fp32, as the definition of a group's scale and offset says (the empty statement keeps the two roundings apart).
__device__ inline _Float16 f64_to_f16(double x) {
    float f = (float)x;
    asm("" : "+v"(f));
    return (_Float16)f;
}

// x of lane N (0..15) of this lane's row of sixteen; the compiler folds it into the instruction that uses it
template <int N>
__device__ inline float row_lane(float x) {
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), 0x150 + N, 0xF, 0xF, true));
}
// x of the lane N behind (within the row of sixteen; 0 past its end)
template <int N>
__device__ inline uint32_t row_ahead(uint32_t x) {
    if constexpr (N == 0) return x;
    else return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x100 + N, 0xF, 0xF, true);
}
__device__ inline float sm_scale(uint32_t sm) { return f16_to_f32((uint16_t)sm); }
__device__ inline float sm_offset(uint32_t sm) { return f16_to_f32((uint16_t)(sm >> 16)); }

// The row (of its step's R) that row r hangs off: NULL parent: a chain. Entries that do not name an earlier node count as -1.
__device__ inline int up_row(const int32_t* parent, int r) {
    if (!parent) return r - 1;
    const int p = parent[r - 1];
    return p < -1 || p >= r - 1 ? 0 : p + 1;
}

// ---- the cache's kernels, on one layer of sequences whose arguments have been checked ------------
struct AppendArgs {
    SeqList seqs;
    const int32_t* lens; const int32_t* block_table;
    uint8_t* pages;                                  // of the layer
    const int32_t* n_rows; const int32_t* parent;    // or NULL
    const int32_t* row_pos;                          // [B][R] positions, or NULL: len + depth in the tree
    const float2* rope;
    Heads q, k, v, q_out;
    int B, R, H, Hq, mpps, start, rope_dim, max_pos; // start >= 0: slots start + r (no positions), else len + r
    int n_part; int64_t part_stride;                 // DT_F32: inputs are the sums of n_part arrays
};
struct AttendArgs {
    SeqList seqs;
    const int32_t* lens; const int32_t* block_table;
    const uint8_t* pages;
    const int32_t* n_rows; const int32_t* parent;
    const unsigned long long* row_anc;               // [B][R] masks, or NULL: from parent
    Heads q, out;
    void* out_lo;                                    // not NULL: the result is two fp16 planes (see split_f16), this is the low one
    float* part;
    int B, R, H, G, mpps, nsplit, nt, J;             // G = query heads per key/value head; nt = tiles of J packed rows per key/value head
    float scale_log2, inv_g;
};
int launch_kv4_append(const AppendArgs& a, int dh, int dtype, hipStream_t stream);
int launch_kv4_attend(AttendArgs a, int dh, int dtype, int max_tokens, hipStream_t stream);
int launch_kv4_compact(const KV* kv, const int32_t* ids_dev, const int32_t* accept_len, const int32_t* accept_path, int B, int K, hipStream_t stream);
size_t kv4_part_floats(int dh);

// ---- products with 4-bit weights (w4.hip) ----------------------------------------------------------
struct W4 { int N, Kd, group, nkb; uint8_t* blocks; };
enum { W4_STORE, W4_F32, W4_ADD_F32, W4_SWIGLU };    // results in the rows' type; as fp32; added to fp32; fp16 silu(gate) up, W's rows being gate | up
int launch_w4(const W4* w, const void* x, int64_t x_stride, int M, int dtype, int epi, void* out, int64_t out_stride, hipStream_t stream);

}  // namespace laser
