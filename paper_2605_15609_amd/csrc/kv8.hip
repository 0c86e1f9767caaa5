// Caches that hold keys and values in 8 bits: rows into codes (psd_kv8_store) and back (psd_kv8_load).
//
// A block of positions and a KV head have one scale for their keys and one for their values,
//     s = max(what the block's kept positions have, fl(largest magnitude of the new rows / M)),   code = RN(x / s),   value = code * s,
// M = 127 (whole numbers) or 448 (floats of 4 and 3 bits), RN to the nearest code, ties to even.  Where s grows, kept codes are rounded again:
// RN(code * s_kept / s).  The quotients are exact before they are rounded, so a code does not depend on how the division is done.
//
// Bound: memory, rows read once and codes written once: 4 prompts of 1024 positions of the 8B shape (67 MB of rows, 34 of codes) are stored in 20 - 23 us and
// read back in 17 where they have just been written and 22 out of memory (12 such caches in turn); a copy of as many bytes takes 20.  The store's vector
// instructions, some 17 a number, take most of its time beside that; deciding the quotients next to a border on a path of their own took 27 us, for in a third
// of the blocks some are.
// A token of 32 requests (7B shape) takes 5.5 us: lengths, then rows, scale and codes, then the largest of a block, each a round trip.
#include "psd_internal.h"
#include "kv8_device.h"

namespace {

constexpr int THREADS = 256;

template <int FORMAT>
__device__ __forceinline__ float number_of(uint32_t code) {
    if constexpr (FORMAT == PSD_KV8_INT8) return (float)(int8_t)code;
    else return __builtin_amdgcn_cvt_f32_fp8((int)code, 0);
}
// four numbers that codes stand for, as their bytes
template <int FORMAT>
__device__ __forceinline__ uint32_t pack_codes(float a, float b, float c, float d) {
    if constexpr (FORMAT == PSD_KV8_INT8) {
        const uint32_t lo = __builtin_amdgcn_perm((uint32_t)(int)b, (uint32_t)(int)a, 0x0c0c0400u), hi = __builtin_amdgcn_perm((uint32_t)(int)d, (uint32_t)(int)c, 0x0c0c0400u);
        return lo | hi << 16;
    } else {
        return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false), true);
    }
}

// RN(x / s) to a code, the largest where x / s is beyond it: M (1 + 2^-23) at most, or, where s is below the normal numbers and off by up to half of its
// last place, 1.5 M at most (190 * 2^-149 has a scale of 2^-149 in int8).  t = x * fl(1 / s) is off by 2^-23 of itself, so the nearest code v to t
// is the right one or next to it; x - v s tells which, and in fp32 it is exact: v is 0 and it is x, or x is hardly less than half a step and it is a
// multiple of 2^-25 steps that is hardly more than half a step.  (Scales below 2^-100, where it might not be, are lifted with x.)
template <int FORMAT>
struct Rounding {
    float s, inv, lift;
    __device__ explicit Rounding(float scale) {
        lift = scale < 0x1p-100f ? 0x1p64f : 1.f;
        s = scale * lift;
        inv = 1.0f / s;
    }
    // power of two that the codes around t are apart
    static __device__ __forceinline__ float step_of(float t) {
        return FORMAT == PSD_KV8_INT8 ? 1.f : fmaxf(__uint_as_float(__float_as_uint(t) & 0x7f800000u), 0x1p-6f) * 0.125f;
    }
    // x + low (what x itself was rounded off by: both 0 or x the larger)
    __device__ __forceinline__ float exact(float x, float low) const {
        const float t = x * inv, step = step_of(t), per = FORMAT == PSD_KV8_INT8 ? 1.f : __uint_as_float(0x7f000000u - __float_as_uint(step));
        const float n = rintf(t * per), v = n * step, rest = __builtin_fmaf(-v, s, x), half = 0.5f * step * s;
        const float over = (fabsf(rest) - half) + (rest < 0.f ? -low : low);
        return (over > 0.f) | ((over == 0.f) & (((int)n & 1) != 0)) ? v + copysignf(step, rest) : v;
    }
    // Four of them as bytes.  Numbers of bf16 are often next to a border: half of the largest, of which 127 codes make 63.5, or three quarters of it, 336 with
    // 448.  So t is taken to b, the nearest half step -- a code or a border -- and a little to the side that x - b s is on, whose sign is exact: it is
    // 2^-25 of s or more (int8), 2^-29 of b s (e4m3), or nothing, and then b decides (ties to even).  A code is not left by that, nor is one next to it reached.
    __device__ __forceinline__ uint32_t codes(float (&x)[4]) const {
        if (lift != 1.f) {
            const float most = s * kv8_most(FORMAT);
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] = __builtin_amdgcn_fmed3f(x[i] * lift, -most, most);
        }
        const float far = inv * 0x1p24f;   // (a lifted scale is 2^-100 or more)
        if constexpr (FORMAT == PSD_KV8_INT8) {
            constexpr float HALVES = 0x1.8p22f, WHOLE = 0x1.8p23f;   // sums with them are rounded to halves, and to whole numbers, whose last byte is the code
            uint32_t r[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float b = __builtin_fmaf(x[i], inv, HALVES) - HALVES, side = __builtin_fmaf(-b, s, x[i]) * far;
                r[i] = __float_as_uint((b + __builtin_amdgcn_fmed3f(side, -0.125f, 0.125f)) + WHOLE);
            }
            return __builtin_amdgcn_perm(__builtin_amdgcn_perm(r[3], r[2], 0x0c0c0400u), __builtin_amdgcn_perm(r[1], r[0], 0x0c0c0400u), 0x05040100u);
        } else {
            float r[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                // (5 bits; below the normal numbers finer than half steps)
                const float b = __uint_as_float((__float_as_uint(x[i] * inv) + 0x40000u) & 0xfff80000u), side = __builtin_fmaf(-b, s, x[i]) * far, most = fabsf(b) * 0x1p-8f;
                r[i] = b + __builtin_amdgcn_fmed3f(side, -most, most);
            }
            return pack_codes<FORMAT>(r[0], r[1], r[2], r[3]);
        }
    }
    // kept codes under a scale of `had` rounded again, the first n of four
    __device__ __forceinline__ uint32_t regrown(uint32_t codes, float had, int n) const {
        float v[4];
        had *= lift;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float code = number_of<FORMAT>(codes >> (8 * i) & 0xff), x = code * had;
            v[i] = exact(x, __builtin_fmaf(code, had, -x));
        }
        const uint32_t first = n >= 4 ? ~0u : (1u << (8 * max(n, 0))) - 1;
        return (codes & ~first) | (pack_codes<FORMAT>(v[0], v[1], v[2], v[3]) & first);
    }
};

// 8 numbers of a row as they were loaded
template <typename T>
struct Raw;
template <>
struct Raw<bf16_t> {
    uint32_t w[4];
    __device__ __forceinline__ void load(const bf16_t *p) {
        const uint4 v = *reinterpret_cast<const uint4 *>(p);
        w[0] = v.x, w[1] = v.y, w[2] = v.z, w[3] = v.w;
    }
    __device__ __forceinline__ float at(int e) const { return __uint_as_float(e & 1 ? w[e >> 1] & 0xffff0000u : w[e >> 1] << 16); }
    // the largest magnitude's bits: infinities and NaN are above all numbers
    typedef uint16_t pair __attribute__((ext_vector_type(2)));
    __device__ __forceinline__ uint32_t top(uint32_t so_far) const {
        pair m = {0, 0};
#pragma unroll
        for (int i = 0; i < 4; ++i) m = __builtin_elementwise_max(m, __builtin_bit_cast(pair, w[i] & 0x7fff7fffu));
        return max(so_far, (uint32_t)max(m.x, m.y) << 16);
    }
};
template <>
struct Raw<float> {
    float v[8];
    __device__ __forceinline__ void load(const float *p) {
        const float4 a = *reinterpret_cast<const float4 *>(p), b = *reinterpret_cast<const float4 *>(p + 4);
        v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
    }
    __device__ __forceinline__ float at(int e) const { return v[e]; }
    __device__ __forceinline__ uint32_t top(uint32_t so_far) const {
#pragma unroll
        for (int e = 0; e < 8; ++e) so_far = max(so_far, __float_as_uint(v[e]) & 0x7fffffffu);
        return so_far;
    }
};

// Codes of a tile in LDS: rows of 4 words -- of values the 16 positions of a half and channel, of keys 16 channels of a position -- 5 words apart, so that
// neither the pieces that threads put there nor the rows meet in few banks.
__device__ __forceinline__ int value_word(int h, int c, int b, int d) { return (h * (d + 4) + c) * 5 + b; }
__device__ __forceinline__ int key_word(int position, int c, int d) { return ((c >> 4) * KV8_TILE + position) * 5 + (c >> 2 & 3); }
constexpr int tile_words(int d) { return (2 * d + 8) * 5; }
// the row that the i-th 16 bytes of a tile are
__device__ __forceinline__ int row_word(int i, int which, int d) {
    const int w = min(d, 32), ws = d < 32 ? 4 : 5;
    return which ? value_word(i >> ws & 1, (i >> (ws + 1) << ws) + (i & (w - 1)), 0, d) : i * 5;
}

// Task i of units x heads x parts x (keys, values), of which there are fewer than 2^24 (what a launch holds)
struct Task {
    bool there;
    int which, part, head, unit;
    __device__ Task(uint32_t i, uint32_t tasks, uint32_t parts, uint32_t heads) {
        there = i < tasks;
        i = there ? i : 0;
        which = i & 1;
        i >>= 1;
        part = i % parts;
        i /= parts;
        head = i % heads;
        unit = i / heads;
    }
};

// The thread's task among its workgroup's.  With heads of 64 and 128 (D; 0: any other) a wavefront has one, so what follows from it is kept once for all lanes.
template <int D>
__device__ __forceinline__ int task_in_group(int ds) {
    if constexpr (D != 0) return __builtin_amdgcn_readfirstlane(threadIdx.x >> ds);
    else return threadIdx.x >> ds;
}

// A task is what the rows of a unit put into one block of a KV head, keys or values; d_head threads take one, tile by tile, a thread 4 positions of 8
// channels.  Their codes are words of a position's channels (keys) or of a channel's positions (values), put together in LDS and written as they
// lie in the cache.
template <typename T, int FORMAT, int NB, int D>
__global__ __launch_bounds__(THREADS) void kv8_store_kernel(Kv8 c, Kv8Rows rows, const int32_t *starts, const int32_t *counts, uint32_t blocks, uint32_t tasks) {
    extern __shared__ __align__(16) uint32_t words[];   // [tasks][NB][tile_words]
    __shared__ uint32_t tops[THREADS / 64];
    const int ds = D ? __builtin_ctz(D | 256) : __ffs(c.d_head) - 1, d = 1 << ds, block = 1 << c.block_shift, mine = task_in_group<D>(ds), t = threadIdx.x & (d - 1);
    const Task of(blockIdx.x * (THREADS >> ds) + mine, tasks, blocks, c.n_kv_heads);
    const int which = of.which, b = of.part, head = of.head;
    const int64_t u = of.unit;
    const int64_t start = starts ? starts[u] : rows.first, count = counts ? min(max(counts[u], 0), rows.n) : rows.n;
    const int64_t end = min(start + count, (int64_t)c.capacity);
    // the b-th block that the unit's rows touch
    const int64_t p0 = ((max(start, (int64_t)0) >> c.block_shift) + b) << c.block_shift;
    const int lo = (int)(max(start, p0) - p0), hi = (int)max(min(end - p0, (int64_t)block), (int64_t)-1);
    const bool live = of.there && lo < hi;
    const int64_t ld = which ? rows.ld_v : rows.ld_k;
    const T *x = (const T *)(which ? rows.v : rows.k) + (u * rows.n + (p0 - start)) * ld + (int64_t)head * d;   // of position p0
    const int row0 = (int)(p0 & (KV8_TILE - 1));   // of the block in its first tile
    uint8_t *codes = c.codes + u * c.stride_codes + ((int64_t)head * (c.capacity / KV8_TILE) + p0 / KV8_TILE) * (64 * d) + which * (32 * d);
    float *scale = &c.scales[u * c.stride_scales + (int64_t)head * (c.capacity >> c.block_shift) + (p0 >> c.block_shift)].x + which;
    uint32_t *lds = words + mine * NB * tile_words(d);
    const int rg = t >> (ds - 3), c8 = (t & ((d >> 3) - 1)) * 8;   // the thread's positions 4 rg .. and channels c8 ..
    const bool partial = live && (lo > 0 || hi < block);

    Raw<T> raw[NB][4];
    uint32_t top = 0;
    float had = 0.f;
    if (live) {
        if (lo > 0) had = *scale;   // (a block that begins with a new row starts afresh)
        if (!partial) {
            const T *from = x + (int64_t)(4 * rg - row0) * ld + c8;
            if (block < KV8_TILE && (4 * rg < row0 || 4 * rg >= row0 + block)) from = x + c8;   // (the other half of a tile: any row)
#pragma unroll
            for (int n = 0; n < NB; ++n)
#pragma unroll
                for (int j = 0; j < 4; ++j) raw[n][j].load(from + (n * KV8_TILE + j) * ld);
        } else {
#pragma unroll
            for (int n = 0; n < NB; ++n)
#pragma unroll
                for (int j = 0; j < 4; ++j)   // (positions without a new row repeat one that has)
                    raw[n][j].load(x + min(max(n * KV8_TILE - row0 + 4 * rg + j, lo), hi - 1) * ld + c8);
        }
        if (partial)   // (codes that stay, and those behind the rows)
#pragma unroll
            for (int n = 0; n < NB; ++n)
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const int i = t + d * k;
                    const uint4 old = *reinterpret_cast<const uint4 *>(codes + (int64_t)n * (64 * d) + i * 16);
                    uint32_t *to = lds + n * tile_words(d) + row_word(i, which, d);
                    to[0] = old.x, to[1] = old.y, to[2] = old.z, to[3] = old.w;
                }
#pragma unroll
        for (int n = 0; n < NB; ++n)
#pragma unroll
            for (int j = 0; j < 4; ++j)
                top = raw[n][j].top(top);
    }
    for (int s = min(d, 64) >> 1; s > 0; s >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, s, 64));
    if ((threadIdx.x & 63) == 0) tops[threadIdx.x >> 6] = top;
    __syncthreads();
    if (d == 128) top = max(tops[mine * 2], tops[mine * 2 + 1]);
    const float need = __uint_as_float(top) / kv8_most(FORMAT);
    const bool finite = top < 0x7f800000u && had < INFINITY;   // (else nothing that the block holds can be told: all of it reads as NaN)
    const float s = finite ? fmaxf(had, need) : NAN;
    const bool grown = finite && had > 0.f && s > had, some = finite && s > 0.f;
    if (live) {
        const Rounding<FORMAT> round(some ? s : 1.f);
        // word i of the thread's 8 in tile n: where it is, and which of its bytes (positions of a channel, or channels of a position) are new
        auto word_at = [&](int n, int i) {
            return lds + n * tile_words(d) + (which ? value_word(rg & 1, c8 + i, rg >> 1, d) : key_word(4 * rg + (i >> 1), c8 + 4 * (i & 1), d));
        };
        auto new_bytes = [&](int n, int i) {
            const int p = n * KV8_TILE - row0 + 4 * rg;   // of the thread's first position in the block
            if (!which) return p + (i >> 1) >= lo && p + (i >> 1) < hi ? 0xffffffffu : 0u;
            uint32_t fresh = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j) fresh |= p + j >= lo && p + j < hi ? 0xffu << (8 * j) : 0u;
            return fresh;
        };
        auto put = [&](int n, int i, uint32_t code) {
            uint32_t *word = word_at(n, i), fresh = partial ? new_bytes(n, i) : 0xffffffffu;
            code = some ? code : 0u;
            if (fresh == 0xffffffffu) *word = code;
            else if (fresh != 0) *word = (*word & ~fresh) | (code & fresh);
        };
        if (partial && grown) {
#pragma unroll 4
            for (int i = 0; i < 8 * NB; ++i) {
                const int p = (i >> 3) * KV8_TILE - row0 + 4 * rg;
                uint32_t *word = word_at(i >> 3, i & 7);
                if (p >= 0 && p < block) *word = round.regrown(*word, had, which ? lo - p : p + ((i & 7) >> 1) < lo ? 4 : 0);
            }
        }
        if (which) {
#pragma unroll
            for (int i = 0; i < 8 * NB; ++i) {
                float v[4] = {raw[i >> 3][0].at(i & 7), raw[i >> 3][1].at(i & 7), raw[i >> 3][2].at(i & 7), raw[i >> 3][3].at(i & 7)};
                put(i >> 3, i & 7, round.codes(v));
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8 * NB; ++i) {
                const Raw<T> &from = raw[i >> 3][(i & 7) >> 1];
                const int e = 4 * (i & 1);
                float v[4] = {from.at(e), from.at(e + 1), from.at(e + 2), from.at(e + 3)};
                put(i >> 3, i & 7, round.codes(v));
            }
        }
        if (t == 0) *scale = s;
    }
    __syncthreads();
    if (!live) return;
#pragma unroll
    for (int n = 0; n < NB; ++n)
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const int i = t + d * k;
            const uint32_t *from = lds + n * tile_words(d) + row_word(i, which, d);
            uint8_t *to = codes + (int64_t)n * (64 * d) + i * 16;
            if (block == KV8_TILE / 2) {   // half of a tile's positions are another block's: rows of keys, 8 bytes of a row of values
                if (which) *reinterpret_cast<uint2 *>(to + (row0 >> 1)) = make_uint2(from[row0 >> 3], from[(row0 >> 3) + 1]);
                else if ((i & 16) == row0) *reinterpret_cast<uint4 *>(to) = make_uint4(from[0], from[1], from[2], from[3]);
            } else {
                *reinterpret_cast<uint4 *>(to) = make_uint4(from[0], from[1], from[2], from[3]);
            }
        }
}

// byte i of a word as a number
template <int FORMAT>
__device__ __forceinline__ float byte_of(uint32_t w, int i) {
    if constexpr (FORMAT == PSD_KV8_INT8) return (float)(int8_t)(w >> (8 * i));
    else return i == 0 ? __builtin_amdgcn_cvt_f32_fp8((int)w, 0) : i == 1 ? __builtin_amdgcn_cvt_f32_fp8((int)w, 1) : i == 2 ? __builtin_amdgcn_cvt_f32_fp8((int)w, 2)
                                                                                                            : __builtin_amdgcn_cvt_f32_fp8((int)w, 3);
}
// 8 codes times s, exact before they are rounded, to a row.  code * s in fp32 is rounded already, and bf16 rounds that once more: wrong only where the first
// rounding ended halfway between two numbers of bf16.  Then (__any of the wavefront) all are rounded to odd first -- the last bit set where something was cut off --
// which bf16 rounds as it would the exact product.  (What was cut off a product below the normal numbers may be below the smallest one: lifted.)
template <int FORMAT>
__device__ __forceinline__ void store_values(bf16_t *to, const float (&code)[8], float s) {
    typedef uint16_t pair __attribute__((ext_vector_type(2)));
    float p[8];
    pair least = {0xffff, 0xffff};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        p[2 * i] = code[2 * i] * s, p[2 * i + 1] = code[2 * i + 1] * s;
        const uint32_t ends = __builtin_amdgcn_perm(__float_as_uint(p[2 * i + 1]), __float_as_uint(p[2 * i]), 0x05040100u) ^ 0x80008000u;
        least = __builtin_elementwise_min(least, __builtin_bit_cast(pair, ends));
    }
    if (__any(least.x == 0 || least.y == 0)) {
        const float lift = s < 1.f ? 0x1p64f : 1.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float rest = __builtin_fmaf(code[i], s * lift, -(p[i] * lift));
            const uint32_t bits = __float_as_uint(p[i]);
            if (rest != 0.f && p[i] != 0.f && !(bits & 1)) p[i] = __uint_as_float((rest > 0.f) == (p[i] > 0.f) ? bits | 1 : bits - 1);
        }
    }
    *reinterpret_cast<uint4 *>(to) = make_uint4(pack_bf16x2(p[0], p[1]), pack_bf16x2(p[2], p[3]), pack_bf16x2(p[4], p[5]), pack_bf16x2(p[6], p[7]));
}
template <int FORMAT>
__device__ __forceinline__ void store_values(float *to, const float (&code)[8], float s) {
    *reinterpret_cast<float4 *>(to) = make_float4(code[0] * s, code[1] * s, code[2] * s, code[3] * s);
    *reinterpret_cast<float4 *>(to + 4) = make_float4(code[4] * s, code[5] * s, code[6] * s, code[7] * s);
}

// A task is one tile of a unit and KV head, keys or values, and d_head threads: codes into LDS as they lie in memory, and a thread takes 4
// positions of 8 channels out of it.
template <typename T, int FORMAT, int D>
__global__ __launch_bounds__(THREADS) void kv8_load_kernel(Kv8 c, Kv8Rows rows, uint32_t tiles, uint32_t tasks) {
    extern __shared__ __align__(16) uint32_t words[];   // [tasks][tile_words]
    const int ds = D ? __builtin_ctz(D | 256) : __ffs(c.d_head) - 1, d = 1 << ds, mine = task_in_group<D>(ds), t = threadIdx.x & (d - 1);
    const Task of(blockIdx.x * (THREADS >> ds) + mine, tasks, tiles, c.n_kv_heads);
    const int which = of.which, tile = rows.first / KV8_TILE + of.part, head = of.head;
    const int64_t u = of.unit;
    const int lo = max(rows.first - tile * KV8_TILE, 0), hi = min(min(rows.first + rows.n, kv8_keys(c, (int)u)) - tile * KV8_TILE, KV8_TILE);
    const bool live = of.there && lo < hi;
    uint32_t *lds = words + mine * tile_words(d);
    const int rg = t >> (ds - 3), c8 = (t & ((d >> 3) - 1)) * 8;
    const int64_t ld = which ? rows.ld_v : rows.ld_k;
    T *out = (T *)(which ? rows.v : rows.k) + (u * rows.n + ((int64_t)tile * KV8_TILE - rows.first)) * ld + (int64_t)head * d + c8;   // of the tile's position 0
    float s = 0.f;
    if (live) {
        const uint8_t *codes = c.codes + u * c.stride_codes + ((int64_t)head * (c.capacity / KV8_TILE) + tile) * (64 * d) + which * (32 * d);
        // (4 positions are of one block)
        s = (&c.scales[u * c.stride_scales + (int64_t)head * (c.capacity >> c.block_shift) + ((tile * KV8_TILE + 4 * rg) >> c.block_shift)].x)[which];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const int i = t + d * k;
            const uint4 v = *reinterpret_cast<const uint4 *>(codes + i * 16);
            uint32_t *to = lds + row_word(i, which, d);
            to[0] = v.x, to[1] = v.y, to[2] = v.z, to[3] = v.w;
        }
    }
    __syncthreads();
    if (!live) return;
    if (which) {
        uint32_t w[8];   // a channel's 4 positions
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e] = lds[value_word(rg & 1, c8 + e, rg >> 1, d)];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            float code[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) code[e] = byte_of<FORMAT>(w[e], j);
            if (4 * rg + j >= lo && 4 * rg + j < hi) store_values<FORMAT>(out + (4 * rg + j) * ld, code, s);
        }
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t *from = lds + key_word(4 * rg + j, c8, d), w0 = from[0], w1 = from[1];   // a position's 8 channels
            float code[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) code[e] = byte_of<FORMAT>(e < 4 ? w0 : w1, e & 3);
            if (4 * rg + j >= lo && 4 * rg + j < hi) store_values<FORMAT>(out + (4 * rg + j) * ld, code, s);
        }
    }
}

int store_blocks(const Kv8 &c, int n) { return ((n + (1 << c.block_shift) - 2) >> c.block_shift) + 1; }   // blocks that n rows touch at most
int load_tiles(int first, int n) { return (first + n - 1) / KV8_TILE - first / KV8_TILE + 1; }

}   // namespace

bool kv8_store_launchable(const Kv8 &c, int units, int n) { return n < 1 || (double)units * c.n_kv_heads * store_blocks(c, n) * 2 * THREADS < 0x1p32; }
bool kv8_load_launchable(const Kv8 &c, int units, int n) { return (double)units * c.n_kv_heads * ((n + 30) / KV8_TILE + 1) * 2 * THREADS < 0x1p32; }

template <typename T, int FORMAT, int D>
static void store_as(const dim3 &grid, int smem, int nb, hipStream_t st, const Kv8 &c, const Kv8Rows &rows, const int32_t *starts, const int32_t *counts, int blocks, uint32_t tasks) {
    if (nb == 1) hipLaunchKernelGGL((kv8_store_kernel<T, FORMAT, 1, D>), grid, dim3(THREADS), smem, st, c, rows, starts, counts, blocks, tasks);
    else if (nb == 2) hipLaunchKernelGGL((kv8_store_kernel<T, FORMAT, 2, D>), grid, dim3(THREADS), smem, st, c, rows, starts, counts, blocks, tasks);
    else hipLaunchKernelGGL((kv8_store_kernel<T, FORMAT, 4, D>), grid, dim3(THREADS), smem, st, c, rows, starts, counts, blocks, tasks);
}

// call(T(), format, d): the types and the head width that kernels are built for
template <int FORMAT, typename T, typename Call>
static void kv8_by_width(int d_head, Call call) {
    if (d_head == 128) call(T(), std::integral_constant<int, FORMAT>(), std::integral_constant<int, 128>());
    else if (d_head == 64) call(T(), std::integral_constant<int, FORMAT>(), std::integral_constant<int, 64>());
    else call(T(), std::integral_constant<int, FORMAT>(), std::integral_constant<int, 0>());
}
template <typename Call>
static void kv8_dispatch(const Kv8 &c, int dtype, Call call) {
    if (dtype == PSD_DTYPE_BF16 && c.format == PSD_KV8_INT8) kv8_by_width<PSD_KV8_INT8, bf16_t>(c.d_head, call);
    else if (dtype == PSD_DTYPE_BF16) kv8_by_width<PSD_KV8_E4M3, bf16_t>(c.d_head, call);
    else if (c.format == PSD_KV8_INT8) kv8_by_width<PSD_KV8_INT8, float>(c.d_head, call);
    else kv8_by_width<PSD_KV8_E4M3, float>(c.d_head, call);
}

void launch_kv8_store(const Kv8 &c, int units, const Kv8Rows &rows, const int32_t *starts, const int32_t *counts, hipStream_t st) {
    if (rows.n < 1) return;
    const int blocks = store_blocks(c, rows.n), per = THREADS / c.d_head, nb = std::max((1 << c.block_shift) / KV8_TILE, 1);
    const uint32_t tasks = (uint32_t)(units * c.n_kv_heads * blocks * 2);
    const int smem = per * nb * tile_words(c.d_head) * 4;
    const dim3 grid((unsigned)((tasks + per - 1) / per));
    kv8_dispatch(c, rows.dtype, [&](auto type, auto format, auto width) {
        store_as<decltype(type), decltype(format)::value, decltype(width)::value>(grid, smem, nb, st, c, rows, starts, counts, blocks, tasks);
    });
}

void launch_kv8_load(const Kv8 &c, int units, const Kv8Rows &rows, hipStream_t st) {
    if (rows.n < 1) return;
    const int tiles = load_tiles(rows.first, rows.n), per = THREADS / c.d_head;
    const uint32_t tasks = (uint32_t)(units * c.n_kv_heads * tiles * 2);
    const dim3 grid((unsigned)((tasks + per - 1) / per));
    kv8_dispatch(c, rows.dtype, [&](auto type, auto format, auto width) {
        hipLaunchKernelGGL((kv8_load_kernel<decltype(type), decltype(format)::value, decltype(width)::value>), grid, dim3(THREADS), per * tile_words(c.d_head) * 4, st, c, rows, tiles, tasks);
    });
}
