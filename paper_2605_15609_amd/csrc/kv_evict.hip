// Eviction of cached positions by the attention weight that they drew (psd_kv_evict): of every unit (a cache, or one layer of it)
// and KV head the `keep` positions with the largest weight, in ascending order, gathered into another cache.
//
// Selection, one workgroup per (unit, head): the weights as integers of the same order, the keep-th largest by four histograms of 8
// bits, then one walk in ascending order that takes what is above it and, of what is equal, the first ones.  Whole numbers throughout,
// so the result does not depend on the order in which the histogram's atomics arrive.
// Gathering, one launch: 16 bytes per thread of a key row; of a value row (transposed) 8 slots per thread.
#include "psd_internal.h"
#include "device_types.h"

namespace {

constexpr int ST = 512;        // threads of a selection
constexpr int GT = 256;        // threads of a gather
constexpr int KP = 4;          // 16-byte pieces of keys per thread
constexpr int VPOS = 512;      // kept positions that a workgroup of the value gather takes
constexpr int VCH = 32;        // channels that it takes

__device__ __forceinline__ int unit_length(const SharedSegment &s, int u) { return s.lens ? min(max(s.lens[u], 0), s.len) : s.len; }

// larger weight <-> larger integer; both zeros alike, NaN below everything; a position that stays whatever it drew is above everything
__device__ __forceinline__ uint32_t order_of(float w, bool stays) {
    if (stays) return 0xffffffffu;
    if (w != w) return 0u;
    const uint32_t b = __float_as_uint(w == 0.f ? 0.f : w);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}

__global__ __launch_bounds__(ST) void evict_select_kernel(SharedSegment src, int n_kv_heads, int keep, int n_first, int n_last,
                                                          int32_t *__restrict__ kept, int32_t *__restrict__ kept_lens) {
    __shared__ uint32_t hist[256];
    __shared__ uint32_t found[2];          // digit, how many of the digit's keys are still to be taken
    __shared__ int sums[2][ST / 64];
    const int u = blockIdx.x / n_kv_heads, g = blockIdx.x % n_kv_heads, t = threadIdx.x, lane = t & 63, wave = t >> 6;
    const int len = unit_length(src, u), n = min(len, keep);
    const float *w = src.weights + (int64_t)u * src.stride_w + (int64_t)g * src.ld_w;
    int32_t *out = kept + (int64_t)blockIdx.x * keep;
    if (g == 0 && t == 0 && kept_lens) kept_lens[u] = n;
    for (int i = n + t; i < keep; i += ST) out[i] = -1;
    if (len <= keep) {
        for (int i = t; i < n; i += ST) out[i] = i;
        return;
    }
    auto key = [&](int i) { return order_of(w[i], i < n_first || i >= len - n_last); };
    // the keep-th largest key, 8 bits at a time
    uint32_t prefix = 0, need = keep;
    for (int shift = 24; shift >= 0; shift -= 8) {
        if (t < 256) hist[t] = 0;
        __syncthreads();
        for (int i = t; i < len; i += ST) {
            const uint32_t k = key(i);
            if (shift == 24 || (k >> (shift + 8)) == prefix) atomicAdd(&hist[(k >> shift) & 255], 1u);
        }
        __syncthreads();
        if (wave == 0) {   // lane l: digits 255 - 4 l .. 252 - 4 l, the largest first
            uint32_t c[4], mine = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) mine += c[e] = hist[255 - 4 * lane - e];
            uint32_t upto = mine;
#pragma unroll
            for (int d = 1; d < 64; d <<= 1) {
                const uint32_t v = __shfl_up(upto, d, 64);
                if (lane >= d) upto += v;
            }
            uint32_t above = upto - mine;
            if (above < need && upto >= need) {   // one lane
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if (above < need && above + c[e] >= need) {
                        found[0] = 255 - 4 * lane - e;
                        found[1] = need - above;
                    }
                    above += c[e];
                }
            }
        }
        __syncthreads();
        prefix = prefix << 8 | found[0];
        need = found[1];
    }
    // a thread walks `each` positions in a row: what is above the key, and what is equal to it
    const int each = (len + ST - 1) / ST, lo = min(t * each, len), hi = min(lo + each, len);
    int above = 0, equal = 0;
    for (int i = lo; i < hi; ++i) {
        const uint32_t k = key(i);
        above += k > prefix;
        equal += k == prefix;
    }
    int above_upto = above, equal_upto = equal;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int a = __shfl_up(above_upto, d, 64), e = __shfl_up(equal_upto, d, 64);
        if (lane >= d) above_upto += a, equal_upto += e;
    }
    if (lane == 63) sums[0][wave] = above_upto, sums[1][wave] = equal_upto;
    __syncthreads();
    int above_before = above_upto - above, equal_before = equal_upto - equal;
    for (int v = 0; v < wave; ++v) above_before += sums[0][v], equal_before += sums[1][v];
    int at = above_before + min(equal_before, (int)need), left = (int)need - equal_before;
    for (int i = lo; i < hi; ++i) {
        const uint32_t k = key(i);
        if (k > prefix || (k == prefix && left-- > 0)) out[at++] = i;
    }
}

// Workgroups [0, key_wgs): keys and weights, KP 16-byte pieces a thread; the rest: values of VPOS kept positions and VCH channels of one
// (unit, head).  What bounds it: memory, and of the values whole lines of the source, whatever share of a line's positions stays.
template <typename T>
__global__ __launch_bounds__(GT) void evict_gather_kernel(SharedSegment src, SharedSegment dst, int n_kv_heads, int d_head, int keep,
                                                          const int32_t *__restrict__ kept, int wgs_per_unit, int64_t key_wgs) {
    constexpr int C = 16 / sizeof(T);
    if ((int64_t)blockIdx.x < key_wgs) {
        const int u = (int)(blockIdx.x / wgs_per_unit), pieces = n_kv_heads * d_head / C, n = min(unit_length(src, u), keep);
        const int64_t x0 = (int64_t)(blockIdx.x % wgs_per_unit) * (GT * KP) + threadIdx.x;
        int from[KP];
        uint4 v[KP];
#pragma unroll
        for (int e = 0; e < KP; ++e) {
            const int64_t x = x0 + e * GT;
            const int i = (int)(x / pieces), g = (int)(x % pieces) * C / d_head;
            from[e] = i < n ? kept[((int64_t)u * n_kv_heads + g) * keep + i] : -1;
        }
#pragma unroll
        for (int e = 0; e < KP; ++e)
            if (from[e] >= 0)
                v[e] = *reinterpret_cast<const uint4 *>((const T *)src.k + (int64_t)u * src.stride_k + (int64_t)from[e] * src.ld_k + (x0 + e * GT) % pieces * C);
#pragma unroll
        for (int e = 0; e < KP; ++e) {
            if (from[e] < 0) continue;
            const int64_t x = x0 + e * GT;
            const int i = (int)(x / pieces), c = (int)(x % pieces) * C, g = c / d_head;
            *reinterpret_cast<uint4 *>((T *)dst.k + (int64_t)u * dst.stride_k + (int64_t)i * dst.ld_k + c) = v[e];
            if (dst.weights && c % d_head == 0)
                dst.weights[(int64_t)u * dst.stride_w + (int64_t)g * dst.ld_w + i] = src.weights[(int64_t)u * src.stride_w + (int64_t)g * src.ld_w + from[e]];
        }
        return;
    }
    const int tiles = (keep + VPOS - 1) / VPOS, groups = (d_head + VCH - 1) / VCH;
    const int64_t x = (int64_t)blockIdx.x - key_wgs;
    const int c0 = (int)(x % groups) * VCH, i0 = (int)(x / groups % tiles) * VPOS, ug = (int)(x / groups / tiles), u = ug / n_kv_heads, g = ug % n_kv_heads;
    const int n = min(min(unit_length(src, u), keep) - i0, VPOS);   // positions of this workgroup
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int first = (lane >> 1) * 16 + 4 * (lane & 1);            // the lane's 8 slots: positions first .. + 3 and first + 8 .. + 11
    if (first >= n) return;
    const bool whole = first + 11 < n;                              // (else the last group: slots behind the last position stay as they were)
    int slot[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) slot[e] = vt_key_slot(kept[(int64_t)ug * keep + i0 + min(first + (e & 3) + 8 * (e >> 2), n - 1)]);
    const T *from = (const T *)src.vt + (int64_t)u * src.stride_vt + (int64_t)g * d_head * src.ld_vt;
    T *to = (T *)dst.vt + (int64_t)u * dst.stride_vt + (int64_t)g * d_head * dst.ld_vt + i0 + lane * 8;
    for (int c = c0 + wave; c < min(c0 + VCH, d_head); c += 4 * (GT / 64)) {
        T v[4][8];
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
            for (int e = 0; e < 8; ++e) v[k][e] = from[(int64_t)min(c + k * (GT / 64), d_head - 1) * src.ld_vt + slot[e]];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if (c + k * (GT / 64) >= min(c0 + VCH, d_head)) break;
            T *row = to + (int64_t)(c + k * (GT / 64)) * dst.ld_vt;
            if (whole) {
#pragma unroll
                for (int h = 0; h < 8 / C; ++h) reinterpret_cast<uint4 *>(row)[h] = reinterpret_cast<const uint4 *>(v[k])[h];
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (first + (e & 3) + 8 * (e >> 2) < n) row[e] = v[k][e];
            }
        }
    }
}

// workgroups of the gather: those of the keys of a unit, and all of the values
struct GatherGrid {
    int64_t per_unit, values;
};
GatherGrid gather_grid(const SharedSegment &src, int units, int n_kv_heads, int d_head, int dtype, int keep) {
    const int c = dtype == PSD_DTYPE_BF16 ? 8 : 4;
    return {((int64_t)std::min(keep, src.len) * (n_kv_heads * d_head / c) + GT * KP - 1) / (GT * KP),
            (int64_t)units * n_kv_heads * ((keep + VPOS - 1) / VPOS) * ((d_head + VCH - 1) / VCH)};
}

}   // namespace

void launch_kv_evict(const SharedSegment &src, const SharedSegment &dst, int units, int n_kv_heads, int d_head, int dtype, int keep, int n_first,
                     int n_last, int32_t *kept, int32_t *kept_lens, hipStream_t st) {
    hipLaunchKernelGGL(evict_select_kernel, dim3((unsigned)(units * n_kv_heads)), dim3(ST), 0, st, src, n_kv_heads, keep, n_first, n_last, kept, kept_lens);
    if (src.len == 0) return;
    const GatherGrid gr = gather_grid(src, units, n_kv_heads, d_head, dtype, keep);
    const int64_t key_wgs = gr.per_unit * units;
    const dim3 grid((unsigned)(key_wgs + gr.values));
    if (dtype == PSD_DTYPE_BF16)
        hipLaunchKernelGGL(evict_gather_kernel<bf16_t>, grid, dim3(GT), 0, st, src, dst, n_kv_heads, d_head, keep, kept, (int)gr.per_unit, key_wgs);
    else
        hipLaunchKernelGGL(evict_gather_kernel<float>, grid, dim3(GT), 0, st, src, dst, n_kv_heads, d_head, keep, kept, (int)gr.per_unit, key_wgs);
}

int64_t kv_evict_workgroups(const SharedSegment &src, int units, int n_kv_heads, int d_head, int dtype, int keep) {
    const GatherGrid gr = gather_grid(src, units, n_kv_heads, d_head, dtype, keep);
    return gr.per_unit * units + gr.values;
}
