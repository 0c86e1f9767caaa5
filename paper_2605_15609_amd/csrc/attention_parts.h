// Pieces that the attention kernels of the shared keys and of the 8-bit caches have in common: fragments of the 32x32 products, the rows of
// a tile, and where their results go.
#pragma once
#include "psd_internal.h"
#include "device_types.h"

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float floatx16 __attribute__((ext_vector_type(16)));

constexpr float LOG2E = 1.4426950408889634f;

// A row of 8 slots of T, as a lane of a 32x32 product holds it: bf16 in one 16-byte load, fp32 in two.
template <typename T>
struct Frag;
template <>
struct Frag<bf16_t> {
    uint4 v;
    __device__ void load(const bf16_t *p) { v = *reinterpret_cast<const uint4 *>(p); }
    // keeps the slots of keys before `left`; the lane's slots are keys 0 - 3 and 8 - 11 (from its half on)
    __device__ void keep(int left) {
        const int hi = left - 8;
        v.x &= left >= 2 ? 0xffffffffu : left == 1 ? 0x0000ffffu : 0u;
        v.y &= left >= 4 ? 0xffffffffu : left == 3 ? 0x0000ffffu : 0u;
        v.z &= hi >= 2 ? 0xffffffffu : hi == 1 ? 0x0000ffffu : 0u;
        v.w &= hi >= 4 ? 0xffffffffu : hi == 3 ? 0x0000ffffu : 0u;
    }
};
template <>
struct Frag<float> {
    float v[8];
    __device__ void load(const float *p) {
        const float4 a = *reinterpret_cast<const float4 *>(p), b = *reinterpret_cast<const float4 *>(p + 4);
        v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
    }
    __device__ void keep(int left) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if ((i >= 4 ? i + 4 : i) >= left) v[i] = 0.f;
    }
};

// acc += A B over 16 contraction slots, 8 in each half of the wavefront
__device__ __forceinline__ void product(const Frag<bf16_t> &a, const Frag<bf16_t> &b, floatx16 &acc) {
    acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a.v), __builtin_bit_cast(bf16x8, b.v), acc, 0, 0, 0);
}
__device__ __forceinline__ void product(const Frag<float> &a, const Frag<float> &b, floatx16 &acc) {
#pragma unroll
    for (int e = 0; e < 8; ++e) acc = __builtin_amdgcn_mfma_f32_32x32x2f32(a.v[e], b.v[e], acc, 0, 0, 0);
}
// The probabilities of 16 keys as the second product takes them.  bf16: rounded to 8 bits of mantissa, as the other attention
// kernels of the bf16 path do (their sum l is taken from the unrounded ones); fp32: as they are.
__device__ __forceinline__ void probabilities(const float *p, Frag<bf16_t> &f) {
    f.v = make_uint4(pack_bf16x2(p[0], p[1]), pack_bf16x2(p[2], p[3]), pack_bf16x2(p[4], p[5]), pack_bf16x2(p[6], p[7]));
}
__device__ __forceinline__ void probabilities(const float *p, Frag<float> &f) {
#pragma unroll
    for (int e = 0; e < 8; ++e) f.v[e] = p[e];
}

// row r of a unit that starts at sequence s0: token row and query head
struct RowOf {
    int64_t token;
    int head;
    __device__ RowOf(const SharedShape &sh, int64_t s0, int kvh, int r) {
        const int group = sh.n_heads / sh.n_kv_heads;
        token = s0 * sh.L + r / group;
        head = kvh * group + r % group;
    }
};

// Where a row's result over the keys of one workgroup goes: a part that the join reads, or, where it is the only one, the output
template <typename T, int DH>
struct PartOut {
    const AttentionParts &ln;
    const bool direct;
    int64_t at;      // of the row in [parts][n_rows], or among the rows
    float *o;
    T *out;
    __device__ PartOut(const SharedShape &sh, const AttentionParts &l, int part, const RowOf &row) : ln(l), direct(l.parts == 0) {
        const int64_t r = row.token * sh.n_heads + row.head;
        at = direct ? r : part * sh.n_rows + r;
        o = l.o + at * DH;
        out = (T *)l.out + row.token * sh.ld_out + row.head * DH;
    }
    // maximum m (what l is relative to) and sum l of the row
    __device__ void sums(float m, float l, float sl2) const {
        if (!direct) ln.ml[at] = make_float2(m, l);
        else if (ln.lse) ln.lse[at] = log_sum(m, l, sl2);
    }
    __device__ static float log_sum(float m, float l, float sl2) { return l == 0.f ? -INFINITY : m * sl2 / LOG2E + logf(l); }
    // what values() multiplies by; 0 where there were no keys
    __device__ float factor(float l) const { return l == 0.f ? 0.f : direct ? 1.0f / l : 1.0f; }
    __device__ void values(int c, const float *v, float f) const {
        if (!direct) {
            *reinterpret_cast<float4 *>(o + c) = make_float4(v[0], v[1], v[2], v[3]);
        } else if constexpr (sizeof(T) == 2) {
            *reinterpret_cast<uint2 *>(out + c) = make_uint2(pack_bf16x2(v[0] * f, v[1] * f), pack_bf16x2(v[2] * f, v[3] * f));
        } else {
            *reinterpret_cast<float4 *>(out + c) = make_float4(v[0] * f, v[1] * f, v[2] * f, v[3] * f);
        }
    }
};

// of a value and of the other half's
__device__ __forceinline__ float both_max(float v) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float both_sum(float v) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

}   // namespace
