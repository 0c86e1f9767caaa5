// Caches that hold keys and values in 8 bits: rows into codes (psd_kv8_store) and back (psd_kv8_load).
//
// A block of positions and a KV head have one scale for their keys and one for their values,
//     s = max(what the block's kept positions have, fl(largest magnitude of the new rows / M)),   code = RN(x / s),   value = code * s,
// M = 127 (whole numbers) or 448 (floats of 4 and 3 bits), RN to the nearest code, ties to even.  Where s grows, kept codes are rounded again:
// RN(code * s_kept / s).  The quotients are exact before they are rounded, so a code does not depend on how the division is done: one in
// fp32 decides where it is further from a border between two codes than it can be off, one in 64 bits where it is not.
//
// Bound: memory (rows read once, codes written once); a single token a chain of round trips in one launch.
#include "psd_internal.h"
#include "kv8_device.h"

namespace {

constexpr int THREADS = 256;

// RN to a code, as its byte
template <int FORMAT>
__device__ __forceinline__ uint32_t code_of(double y) {
    if constexpr (FORMAT == PSD_KV8_INT8) {
        return (uint32_t)(int)fmin(fmax(rint(y), -127.0), 127.0) & 0xffu;
    } else {
        int e;
        (void)frexp(y, &e);
        const int step = (e < -5 ? -5 : e) - 4;                               // of the codes around y: 2^step
        const double r = fmin(fabs(rint(ldexp(y, -step))), ldexp(448.0, -step));   // 0 .. 16 steps
        const int n = (int)r;
        // n steps above 2^(step + 3) or, below the smallest normal number, above 0
        const uint32_t bits = n < 8 ? n : ((uint32_t)(step + 9) << 3) + n;
        return bits | (y < 0.0 ? 0x80u : 0u);
    }
}
template <int FORMAT>
__device__ __forceinline__ float number_of(uint32_t code) {
    if constexpr (FORMAT == PSD_KV8_INT8) return (float)(int8_t)code;
    else return __builtin_amdgcn_cvt_f32_fp8((int)code, 0);
}

template <typename T>
__device__ __forceinline__ void load8(const T *p, float (&x)[8]) {
    if constexpr (sizeof(T) == 2) {
        const uint4 v = *reinterpret_cast<const uint4 *>(p);
        const uint32_t u[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] = __uint_as_float(u[i] << 16);
            x[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
        }
    } else {
        const float4 v = *reinterpret_cast<const float4 *>(p), w = *reinterpret_cast<const float4 *>(p + 4);
        x[0] = v.x, x[1] = v.y, x[2] = v.z, x[3] = v.w, x[4] = w.x, x[5] = w.y, x[6] = w.z, x[7] = w.w;
    }
}

// A workgroup stores what the rows of a unit put into one block of a KV head, keys or values.  Codes are put together in LDS, as they lie in the
// cache (whole tiles, of a block of 16 positions half of one).
template <typename T, int FORMAT>
__global__ __launch_bounds__(THREADS) void kv8_store_kernel(Kv8 c, Kv8Rows rows, const int32_t *starts, const int32_t *counts, int blocks) {
    extern __shared__ __align__(16) uint8_t tile[];
    __shared__ float tops[THREADS / 64];
    const int d = c.d_head, block = 1 << c.block_shift;
    int64_t at = blockIdx.x;
    const int which = (int)(at & 1);
    at >>= 1;
    const int b = (int)(at % blocks);
    at /= blocks;
    const int head = (int)(at % c.n_kv_heads);
    const int64_t u = at / c.n_kv_heads;
    const int64_t start = starts ? starts[u] : rows.first, count = counts ? min(max(counts[u], 0), rows.n) : rows.n;
    const int64_t end = min(start + count, (int64_t)c.capacity);
    // the b-th block that the unit's rows touch
    const int64_t p0 = ((max(start, (int64_t)0) >> c.block_shift) + b) << c.block_shift;
    const int lo = (int)(max(start, p0) - p0), hi = (int)min(end - p0, (int64_t)block);
    if (p0 >= end || lo >= hi) return;
    const T *x = (const T *)(which ? rows.v : rows.k) + (u * rows.n + (p0 - start)) * (which ? rows.ld_v : rows.ld_k) + (int64_t)head * d;   // of position p0
    const int64_t ld = which ? rows.ld_v : rows.ld_k;
    const int pieces = d >> 3, n = (hi - lo) * pieces;
    float top = 0.f;
    bool bad = false;
    for (int i = threadIdx.x; i < n; i += THREADS) {
        float v[8];
        load8(x + (lo + i / pieces) * ld + i % pieces * 8, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            bad |= !(fabsf(v[e]) < INFINITY);
            top = fmaxf(top, fabsf(v[e]));
        }
    }
    if (bad) top = INFINITY;
    for (int s = 32; s > 0; s >>= 1) top = fmaxf(top, __shfl_xor(top, s, 64));
    if ((threadIdx.x & 63) == 0) tops[threadIdx.x >> 6] = top;
    // codes that stay, and those behind the rows: as they are
    const bool partial = lo > 0 || hi < block;
    const int row0 = (int)(p0 & (KV8_TILE - 1)), tiles = max(block / KV8_TILE, 1);
    uint8_t *codes = c.codes + u * c.stride_codes + ((int64_t)head * (c.capacity / KV8_TILE) + p0 / KV8_TILE) * (64 * d) + which * (32 * d);
    if (partial)
        for (int i = threadIdx.x; i < tiles * 2 * d; i += THREADS)
            *reinterpret_cast<uint4 *>(tile + i * 16) = *reinterpret_cast<const uint4 *>(codes + (int64_t)(i / (2 * d)) * (64 * d) + i % (2 * d) * 16);
    float *scale = &c.scales[u * c.stride_scales + (int64_t)head * (c.capacity >> c.block_shift) + (p0 >> c.block_shift)].x + which;
    const float had = lo > 0 ? *scale : 0.f;   // (a block that begins with a new row starts afresh)
    __syncthreads();
    top = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
    const float need = top / kv8_most(FORMAT);
    const bool finite = need < INFINITY && had < INFINITY;   // (else nothing that the block holds can be told: all of it reads as NaN)
    const float s = finite ? fmaxf(had, need) : NAN;
    auto place = [&](int p, int ch) { return (row0 + p) / KV8_TILE * (32 * d) + (which ? kv8_value_at((row0 + p) % KV8_TILE, ch, d) : kv8_key_at((row0 + p) % KV8_TILE, ch)); };
    if (finite && had > 0.f && s > had)
        for (int i = threadIdx.x; i < lo * d; i += THREADS) {
            uint8_t *q = tile + place(i / d, i % d);
            *q = (uint8_t)code_of<FORMAT>((double)number_of<FORMAT>(*q) * (double)had / (double)s);
        }
    for (int i = threadIdx.x; i < n; i += THREADS) {
        const int p = lo + i / pieces, ch = i % pieces * 8;
        float v[8];
        load8(x + p * ld + ch, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) tile[place(p, ch + e)] = (uint8_t)(finite && s > 0.f ? code_of<FORMAT>((double)v[e] / (double)s) : 0u);
    }
    if (threadIdx.x == 0) *scale = s;
    __syncthreads();
    // Blocks of 16 share the 16 bytes of a value's positions: 8 bytes are one block's alone.
    for (int i = threadIdx.x; i < tiles * 4 * d; i += THREADS) {
        const int in_tile = i % (4 * d) * 8;
        if (block < KV8_TILE && (which ? in_tile & 8 : in_tile >> 4 & 16) != (which ? row0 >> 1 : row0)) continue;
        *reinterpret_cast<uint2 *>(codes + (int64_t)(i / (4 * d)) * (64 * d) + in_tile) = *reinterpret_cast<const uint2 *>(tile + i * 8);
    }
}

// code * s to T: exact before it is rounded.  In fp32 the product is rounded already; bf16 takes it with the last bit set where something was cut off
// (rounded to odd), which rounds as the exact product does.
template <typename T>
__device__ __forceinline__ T value_of(float code, float s) {
    float p = code * s;
    if constexpr (sizeof(T) == 2) {
        const float rest = __builtin_fmaf(code, s, -p);
        const uint32_t bits = __float_as_uint(p);
        if (rest != 0.f && !(bits & 1)) p = __uint_as_float((rest > 0.f) == (p > 0.f) ? bits | 1 : bits - 1);
    }
    return from_float<T>(p);
}

// A workgroup loads the positions of one tile of a unit and KV head, keys or values.
template <typename T, int FORMAT>
__global__ __launch_bounds__(THREADS) void kv8_load_kernel(Kv8 c, Kv8Rows rows, int tiles) {
    extern __shared__ __align__(16) uint8_t tile[];
    const int d = c.d_head;
    int64_t at = blockIdx.x;
    const int which = (int)(at & 1);
    at >>= 1;
    const int t = rows.first / KV8_TILE + (int)(at % tiles);
    at /= tiles;
    const int head = (int)(at % c.n_kv_heads);
    const int64_t u = at / c.n_kv_heads;
    const int lo = max(rows.first - t * KV8_TILE, 0), hi = min(min(rows.first + rows.n, kv8_keys(c, (int)u)) - t * KV8_TILE, KV8_TILE);
    if (lo >= hi) return;
    const uint8_t *codes = c.codes + u * c.stride_codes + ((int64_t)head * (c.capacity / KV8_TILE) + t) * (64 * d) + which * (32 * d);
    for (int i = threadIdx.x; i < 2 * d; i += THREADS) *reinterpret_cast<uint4 *>(tile + i * 16) = *reinterpret_cast<const uint4 *>(codes + i * 16);
    __syncthreads();
    const float *scales = &c.scales[u * c.stride_scales + (int64_t)head * (c.capacity >> c.block_shift)].x + which;
    const int64_t ld = which ? rows.ld_v : rows.ld_k;
    T *out = (T *)(which ? rows.v : rows.k) + (u * rows.n + ((int64_t)t * KV8_TILE - rows.first)) * ld + (int64_t)head * d;   // of the tile's position 0
    for (int i = threadIdx.x; i < (hi - lo) * d; i += THREADS) {
        const int p = lo + i / d, ch = i % d;
        const float s = scales[2 * (int64_t)((t * KV8_TILE + p) >> c.block_shift)];
        out[p * ld + ch] = value_of<T>(number_of<FORMAT>(tile[which ? kv8_value_at(p, ch, d) : kv8_key_at(p, ch)]), s);
    }
}

int store_blocks(const Kv8 &c, int n) { return ((n + (1 << c.block_shift) - 2) >> c.block_shift) + 1; }   // blocks that n rows touch at most
int load_tiles(int first, int n) { return (first + n - 1) / KV8_TILE - first / KV8_TILE + 1; }

}   // namespace

bool kv8_store_launchable(const Kv8 &c, int units, int n) { return n < 1 || (double)units * c.n_kv_heads * store_blocks(c, n) * 2 * THREADS < 0x1p32; }
bool kv8_load_launchable(const Kv8 &c, int units, int n) { return (double)units * c.n_kv_heads * ((n + 30) / KV8_TILE + 1) * 2 * THREADS < 0x1p32; }

#define PSD_KV8_DISPATCH(call)                                                   \
    if (rows.dtype == PSD_DTYPE_BF16) {                                          \
        using T = bf16_t;                                                        \
        if (c.format == PSD_KV8_INT8) { constexpr int F = PSD_KV8_INT8; call; }  \
        else { constexpr int F = PSD_KV8_E4M3; call; }                           \
    } else {                                                                     \
        using T = float;                                                         \
        if (c.format == PSD_KV8_INT8) { constexpr int F = PSD_KV8_INT8; call; }  \
        else { constexpr int F = PSD_KV8_E4M3; call; }                           \
    }

void launch_kv8_store(const Kv8 &c, int units, const Kv8Rows &rows, const int32_t *starts, const int32_t *counts, hipStream_t st) {
    if (rows.n < 1) return;
    const int blocks = store_blocks(c, rows.n), smem = std::max(1 << c.block_shift, KV8_TILE) * c.d_head;
    const dim3 grid((unsigned)((int64_t)units * c.n_kv_heads * blocks * 2));
    PSD_KV8_DISPATCH(hipLaunchKernelGGL((kv8_store_kernel<T, F>), grid, dim3(THREADS), smem, st, c, rows, starts, counts, blocks))
}

void launch_kv8_load(const Kv8 &c, int units, const Kv8Rows &rows, hipStream_t st) {
    if (rows.n < 1) return;
    const int tiles = load_tiles(rows.first, rows.n), smem = KV8_TILE * c.d_head;
    const dim3 grid((unsigned)((int64_t)units * c.n_kv_heads * tiles * 2));
    PSD_KV8_DISPATCH(hipLaunchKernelGGL((kv8_load_kernel<T, F>), grid, dim3(THREADS), smem, st, c, rows, tiles))
}
