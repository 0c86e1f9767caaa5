// Norms of heads and rotary positions (psd_rotary): of every head of a token's queries and keys
//     y = x / sqrt(mean x^2 + eps) * gain                                     (where there are gains)
//     (y_a, y_b) <- f (y_a cos t - y_b sin t, y_b cos t + y_a sin t),  t = position * frequency of the pair,
// for the pairs (j, j + r/2) or (2j, 2j + 1) of the first r channels; the others stay as they are.
//
// An angle of a far position has more turns than fp32 can count, so position * frequency / 2 pi is taken in 64 bits and only what is left of
// whole turns is rounded: off by 2^-25 of a turn and, for the three products in 64 bits, 2^-51 of the angle's turns (as much at 2^26 of them).
// Everything else is fp32, rounded to the type once.
//
// Bound: memory, every channel read and written once: 20480 rows of 64 heads of 128 take 115 - 122 us (671 MB, 5.5 - 5.8 TB/s; a copy has 5.2),
// normed; 6126 rows of 32 heads, half of each turned, 17 - 19 us (100 MB).  One block of the small model 3.5 us, a launch.
// Heads or halves that are not whole pieces of 16 bytes go by wavefronts, which turn the angles of every head anew and are bound by that: 20480 rows of 64
// heads of 128 with 120 channels turned in halves take 636 us, 16 heads of 64 with 24 channels 97 (with 32, by pieces, 15).
#include "psd_internal.h"
#include "device_types.h"

namespace {

constexpr int THREADS = 256;

__device__ __forceinline__ int position_of(const Rotary &a, int64_t token) {
    return a.positions ? a.positions[token] : a.first + (int)(token % a.rows_per_seq);
}

// factor * (cos, sin) of pair j at a position
__device__ __forceinline__ float2 turn_of(const Rotary &a, int position, int j) {
    const double turns = position * (a.frequencies[j] * 0.15915494309189535);
    float s, c;
    sincospif((float)(2.0 * (turns - rint(turns))), &s, &c);
    return make_float2(a.factor * c, a.factor * s);
}

// 8 channels of T
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
template <typename T>
__device__ __forceinline__ void store8(T *p, const float (&x)[8]) {
    if constexpr (sizeof(T) == 2) {
        *reinterpret_cast<uint4 *>(p) = make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7]));
    } else {
        *reinterpret_cast<float4 *>(p) = make_float4(x[0], x[1], x[2], x[3]);
        *reinterpret_cast<float4 *>(p + 4) = make_float4(x[4], x[5], x[6], x[7]);
    }
}

// Heads of whole 16 channels, and of halves that are whole 8: a lane takes two pieces of 8 channels whose channels are each other's partners
// (or that are not rotated), lpu lanes (a power of two, those behind the last piece idle) a head.  A workgroup turns the angles of its
// tokens once, for all of their heads.
template <typename T>
__global__ __launch_bounds__(THREADS) void rotary_kernel(Rotary a, int lpu, int tokens) {
    extern __shared__ float2 turns[];   // [tokens][rotated / 2]
    const int pairs = a.rotated >> 1, heads = a.rows[0].heads + a.rows[1].heads, units = a.d_head >> 4;
    const int64_t token0 = (int64_t)blockIdx.x * tokens;
    const int here = (int)min((int64_t)tokens, a.n_tokens - token0);
    for (int i = threadIdx.x; i < here * pairs; i += THREADS) turns[i] = turn_of(a, position_of(a, token0 + i / pairs), i % pairs);
    __syncthreads();
    const int unit = threadIdx.x & (lpu - 1);
    // where the two pieces are, and which pairs the first one begins with
    int c0 = 16 * unit, c1 = 16 * unit + 8;
    if (!a.interleaved && 16 * unit < a.rotated) c0 = 8 * unit, c1 = 8 * unit + pairs;
    const int pair0 = 8 * unit;
    for (int i = threadIdx.x / lpu; i < here * heads; i += THREADS / lpu) {
        const int t = i / heads, h = i % heads, which = h >= a.rows[0].heads;
        const RotaryRows &rows = a.rows[which];
        const int head = h - (which ? a.rows[0].heads : 0);
        const T *in = (const T *)rows.in + (token0 + t) * rows.ld_in + (int64_t)head * a.d_head;
        T *out = (T *)rows.out + (token0 + t) * rows.ld_out + (int64_t)head * a.d_head;
        float x[8], y[8];
        if (unit < units) {
            load8(in + c0, x);
            load8(in + c1, y);
        }
        if (rows.gain) {
            float sum = 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) sum = unit < units ? __builtin_fmaf(x[e], x[e], __builtin_fmaf(y[e], y[e], sum)) : 0.f;
            for (int d = lpu >> 1; d > 0; d >>= 1) sum += __shfl_xor(sum, d, 64);
            const float inv = 1.0f / sqrtf(sum / (float)a.d_head + a.eps);
            if (unit < units) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    x[e] *= inv * rows.gain[c0 + e];
                    y[e] *= inv * rows.gain[c1 + e];
                }
            }
        }
        if (unit >= units) continue;
        const float2 *cs = turns + t * pairs + pair0;
        if (a.interleaved) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if (pair0 + e < pairs) {
                    const float2 w = cs[e];
                    const float p = x[2 * e], q = x[2 * e + 1];
                    x[2 * e] = p * w.x - q * w.y;
                    x[2 * e + 1] = q * w.x + p * w.y;
                }
                if (pair0 + 4 + e < pairs) {
                    const float2 w = cs[4 + e];
                    const float p = y[2 * e], q = y[2 * e + 1];
                    y[2 * e] = p * w.x - q * w.y;
                    y[2 * e + 1] = q * w.x + p * w.y;
                }
            }
        } else if (16 * unit < a.rotated) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float2 w = cs[e];
                const float p = x[e], q = y[e];
                x[e] = p * w.x - q * w.y;
                y[e] = q * w.x + p * w.y;
            }
        }
        store8(out + c0, x);
        store8(out + c1, y);
    }
}

// Any even head width and rotated part, rows on any element: a wavefront a head, a lane a channel and every 64th behind it.
template <typename T>
__global__ __launch_bounds__(THREADS) void rotary_any_kernel(Rotary a) {
    constexpr int MOST = PSD_MAX_ROTARY_HEAD / 64;
    const int lane = threadIdx.x & 63, heads = a.rows[0].heads + a.rows[1].heads, pairs = a.rotated >> 1;
    const int64_t i = (int64_t)blockIdx.x * (THREADS / 64) + (threadIdx.x >> 6);
    if (i >= a.n_tokens * heads) return;
    const int64_t token = i / heads;
    const int h = (int)(i % heads), which = h >= a.rows[0].heads, position = position_of(a, token);
    const RotaryRows &rows = a.rows[which];
    const int head = h - (which ? a.rows[0].heads : 0);
    const T *in = (const T *)rows.in + token * rows.ld_in + (int64_t)head * a.d_head;
    T *out = (T *)rows.out + token * rows.ld_out + (int64_t)head * a.d_head;
    float x[MOST], y[MOST], sum = 0.f;   // a channel and its partner (all are read before any is written: out may be in)
#pragma unroll
    for (int n = 0; n < MOST; ++n) {
        const int c = lane + 64 * n;
        const int partner = c >= a.rotated ? c : a.interleaved ? c ^ 1 : c < pairs ? c + pairs : c - pairs;
        x[n] = c < a.d_head ? to_float(in[c]) : 0.f;
        y[n] = c < a.d_head ? to_float(in[partner]) : 0.f;
        sum = __builtin_fmaf(x[n], x[n], sum);
        if (rows.gain && c < a.d_head) y[n] *= rows.gain[partner];
    }
    float inv = 1.f;
    if (rows.gain) {
        for (int d = 32; d > 0; d >>= 1) sum += __shfl_xor(sum, d, 64);
        inv = 1.0f / sqrtf(sum / (float)a.d_head + a.eps);
    }
#pragma unroll
    for (int n = 0; n < MOST; ++n) {
        const int c = lane + 64 * n;
        if (c >= a.d_head) continue;
        float v = rows.gain ? x[n] * rows.gain[c] * inv : x[n];
        if (c < a.rotated) {
            const bool second = a.interleaved ? c & 1 : c >= pairs;
            const float2 w = turn_of(a, position, a.interleaved ? c >> 1 : second ? c - pairs : c);
            const float other = y[n] * inv;
            v = second ? v * w.x + other * w.y : v * w.x - other * w.y;
        }
        out[c] = from_float<T>(v);
    }
}

bool by_pieces(const Rotary &a) {
    const int chunk = a.dtype == PSD_DTYPE_BF16 ? 8 : 4;   // elements of 16 bytes
    if (a.d_head % 16 || (!a.interleaved && a.rotated % 16)) return false;
    for (const RotaryRows &r : a.rows)
        if (r.heads > 0 && (reinterpret_cast<uintptr_t>(r.in) % 16 || reinterpret_cast<uintptr_t>(r.out) % 16 || r.ld_in % chunk || r.ld_out % chunk)) return false;
    return true;
}

struct Grid {
    int lpu, tokens;
    int64_t blocks;
};
Grid grid_of(const Rotary &a) {
    const int heads = a.rows[0].heads + a.rows[1].heads;
    if (!by_pieces(a)) return {0, 0, (a.n_tokens * heads + THREADS / 64 - 1) / (THREADS / 64)};
    int lpu = 1;
    while (lpu < a.d_head / 16) lpu *= 2;
    const int tokens = std::min(std::max(THREADS / lpu / heads, 1), 8);   // (8: the angles of heads of 256 channels are 8 KB)
    return {lpu, tokens, (a.n_tokens + tokens - 1) / tokens};
}

template <typename T>
void run(const Rotary &a, hipStream_t st) {
    const Grid g = grid_of(a);
    if (g.lpu > 0) hipLaunchKernelGGL(rotary_kernel<T>, dim3((unsigned)g.blocks), dim3(THREADS), g.tokens * (a.rotated / 2) * sizeof(float2), st, a, g.lpu, g.tokens);
    else hipLaunchKernelGGL(rotary_any_kernel<T>, dim3((unsigned)g.blocks), dim3(THREADS), 0, st, a);
}

}   // namespace

bool rotary_launchable(const Rotary &a) { return launchable(grid_of(a).blocks, THREADS); }

void launch_rotary(const Rotary &a, hipStream_t st) {
    if (a.dtype == PSD_DTYPE_BF16) run<bf16_t>(a, st);
    else run<float>(a, st);
}
