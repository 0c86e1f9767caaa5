// Eviction of cached positions by the attention weight that they drew (psd_kv_evict): of every unit (a cache, or one layer of it)
// and KV head the `keep` positions with the largest weight, in ascending order, gathered into another cache.
//
// Selection, one workgroup per (unit, head): the weights as integers of the same order, held in registers up to 32768 positions; the
// keep-th largest by four histograms of 8 bits, then what is above it and, of what is equal, the first ones.  Whole numbers
// throughout, so the result does not depend on the order in which the histogram's atomics arrive.
// Gathering: 16 bytes per thread of a key row; of a value row (transposed) a slot per lane, so that 64 kept positions, which lie near
// each other, are found in few lines (8 slots per lane and 16-byte stores visit 8 times the lines: 429 us where this takes 411).
// Memory gives whole lines of the source for them, whatever share of a line's positions stays, and that bounds large evictions (8B
// shape, 32 layers, 4096 -> 1024 positions: 411 us, 1.9 GB with all value lines, at 4.6 TB/s where a large copy has 4.9).  The workgroup
// that selected may gather too (MOST_FUSED), which saves a launch and the list's way through memory.  That many workgroups are on the card at
// once, three to a CU (up to 16 positions a lane; one above), so all of them select first and copy then.
#include <type_traits>

#include "psd_internal.h"
#include "device_types.h"

namespace {

constexpr int ST = 512;        // threads of a selection
constexpr int GT = 256;        // threads of a gather
constexpr int KP = 4;          // 16-byte pieces of keys per thread
constexpr int VPOS = 512;      // kept positions that a workgroup of the value gather takes
constexpr int VCH = 32;        // channels that it takes
constexpr int KEPT_LDS = 4096; // kept positions that a workgroup holds in LDS
// One launch where there are at most MOST_FUSED workgroups and each has no more to copy (of keys, and as much of values) than 2 KB times
// their number, or 16 KB.  One launch | two, us: 560 workgroups of 125 KB 89 | 91, 256 of 256 KB 116 | 120, 128 of 256 KB 68 | 72, 112 of
// 64 KB 24 | 28, 64 of 16 KB 9.7 | 14, 16 of 7 KB 9.4 | 11.4; 64 of 128 KB 28 | 28; 112 of 512 KB 148 | 108, 32 of 256 KB 55 | 35, 4 of
// 32 KB 13 | 12, 4 of 1 MB 202 | 62; 1024 of 256 KB 418 | 411, 1024 of 16 KB 61 | 59.
constexpr int MOST_FUSED = 768;

__device__ __forceinline__ int unit_length(const SharedSegment &s, int u) { return s.lens ? min(max(s.lens[u], 0), s.len) : s.len; }

// larger weight <-> larger integer; both zeros alike, NaN below everything; a position that stays whatever it drew is above everything
__device__ __forceinline__ uint32_t order_of(float w, bool stays) {
    if (stays) return 0xffffffffu;
    if (w != w) return 0u;
    const uint32_t b = __float_as_uint(w == 0.f ? 0.f : w);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}

// The selection of one (unit, head) by a workgroup: n positions into `out`, and their first KEPT_LDS into `list`.  A wavefront takes a run
// of 64 EACH positions, 64 at a time, and holds their keys in registers (EACH 0: any number, read again for every histogram).  (The
// lanes of a wavefront counting into 4 or 8 copies of the histogram, which fewer of them share: the same time.)
template <int EACH>
__device__ __forceinline__ void select_positions(const float *__restrict__ w, int len, int keep, int n_first, int n_last, int32_t *__restrict__ out,
                                                 int32_t *list) {
    __shared__ uint32_t hist[256];
    __shared__ uint32_t found[2];          // digit, how many of the digit's keys are still to be taken
    __shared__ int sums[2][ST / 64];
    const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
    auto key = [&](int i) { return order_of(w[i], i < n_first || i >= len - n_last); };
    const int each = EACH > 0 ? EACH : (len + ST - 1) / ST, lo = wave * each * 64;
    uint32_t mine[EACH > 0 ? EACH : 1];
    if constexpr (EACH > 0) {
#pragma unroll
        for (int e = 0; e < EACH; ++e) mine[e] = key(min(lo + e * 64 + lane, len - 1));
    }
    auto walk = [&](auto f) {   // over the wavefront's positions; all lanes of it take part (f's third argument: there is such a position)
        if constexpr (EACH > 0) {
#pragma unroll
            for (int e = 0; e < EACH; ++e) f(lo + e * 64 + lane, mine[e], lo + e * 64 + lane < len);
        } else {
            for (int i = lo; i < min(lo + each * 64, len); i += 64) f(i + lane, key(min(i + lane, len - 1)), i + lane < len);
        }
    };
    uint32_t prefix = 0, need = keep;
    for (int shift = 24; shift >= 0; shift -= 8) {   // the keep-th largest key, 8 bits at a time
        if (t < 256) hist[t] = 0;
        __syncthreads();
        walk([&](int, uint32_t k, bool in) {
            if (in && (shift == 24 || (k >> (shift + 8)) == prefix)) atomicAdd(&hist[(k >> shift) & 255], 1u);
        });
        __syncthreads();
        if (wave == 0) {   // lane l: digits 255 - 4 l .. 252 - 4 l, the largest first
            uint32_t c[4], total = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) total += c[e] = hist[255 - 4 * lane - e];
            uint32_t upto = total;
#pragma unroll
            for (int d = 1; d < 64; d <<= 1) {
                const uint32_t v = __shfl_up(upto, d, 64);
                if (lane >= d) upto += v;
            }
            uint32_t above = upto - total;
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
    int above = 0, equal = 0;   // of the wavefront
    walk([&](int, uint32_t k, bool in) {
        above += __popcll(__ballot(in && k > prefix));
        equal += __popcll(__ballot(in && k == prefix));
    });
    if (lane == 0) sums[0][wave] = above, sums[1][wave] = equal;
    __syncthreads();
    above = equal = 0;          // of what is before
    for (int v = 0; v < wave; ++v) above += sums[0][v], equal += sums[1][v];
    const unsigned long long before = (1ull << lane) - 1;
    walk([&](int i, uint32_t k, bool in) {
        const unsigned long long a = __ballot(in && k > prefix), q = __ballot(in && k == prefix);
        const int same = equal + __popcll(q & before), at = above + __popcll(a & before) + min(same, (int)need);
        if (in && (k > prefix || (k == prefix && same < (int)need))) {
            out[at] = i;
            if (at < KEPT_LDS) list[at] = i;
        }
        above += __popcll(a);
        equal += __popcll(q);
    });
}

// Values of positions i0 .. i0 + n - 1 of one (unit, head), channels c0, c0 + step .. below c_end (c0 the same for a whole wavefront): a
// lane takes a slot of every 64 of a row, E times, and RV rows at a time, so that a load finds its 64 positions in few lines.
// position(i): the source of the i-th kept one.
template <int E, int RV, typename T, typename F>
__device__ __forceinline__ void gather_slots(const T *from, int ld_from, T *to, int ld_to, int i0, int n, int c0, int step, int c_end, F position) {
    const int lane = threadIdx.x & 63, at = lane & ~15, s = lane & 15;
    const int own = at + ((s & 3) | (s & 4) << 1 | (s & 8) >> 1);   // which position lies in the lane's slot
    uint32_t slot[E];
#pragma unroll
    for (int e = 0; e < E; ++e) slot[e] = vt_key_slot(position(i0 + min(e * 64 + own, n - 1)));
    to += i0 + lane;
    for (int c = c0; c < c_end; c += RV * step) {
        T v[RV][E];
#pragma unroll
        for (int k = 0; k < RV; ++k)
#pragma unroll
            for (int e = 0; e < E; ++e) v[k][e] = (from + (int64_t)min(c + k * step, c_end - 1) * ld_from)[slot[e]];
#pragma unroll
        for (int k = 0; k < RV; ++k) {
            if (c + k * step >= c_end) break;
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (e * 64 + own < n) (to + (int64_t)(c + k * step) * ld_to)[e * 64] = v[k][e];
        }
    }
}
template <typename T, typename F>
__device__ __forceinline__ void gather_values(const T *from, int ld_from, T *to, int ld_to, int i0, int n, int c0, int step, int c_end, F position) {
    if (n <= 0) return;
    if (n > VPOS / 2) gather_slots<VPOS / 64, 4>(from, ld_from, to, ld_to, i0, n, c0, step, c_end, position);
    else if (n > VPOS / 4) gather_slots<VPOS / 128, 8>(from, ld_from, to, ld_to, i0, n, c0, step, c_end, position);
    else gather_slots<VPOS / 256, 16>(from, ld_from, to, ld_to, i0, n, c0, step, c_end, position);
}

// One workgroup per (unit, head): selects, and (GATHER) gathers what it selected.
template <typename T, int EACH, bool GATHER>
__global__ __launch_bounds__(ST) void evict_select_kernel(SharedSegment src, SharedSegment dst, int n_kv_heads, int d_head, int keep, int n_first, int n_last,
                                                          int32_t *__restrict__ kept, int32_t *__restrict__ kept_lens) {
    __shared__ int32_t list[KEPT_LDS];
    const int u = blockIdx.x / n_kv_heads, g = blockIdx.x % n_kv_heads, t = threadIdx.x;
    const int len = unit_length(src, u), n = min(len, keep);
    const float *w = src.weights + (int64_t)u * src.stride_w + (int64_t)g * src.ld_w;
    int32_t *out = kept + (int64_t)blockIdx.x * keep;
    if (g == 0 && t == 0 && kept_lens) kept_lens[u] = n;
    for (int i = n + t; i < keep; i += ST) out[i] = -1;
    if (len <= keep) {
        for (int i = t; i < n; i += ST) {
            out[i] = i;
            if (i < KEPT_LDS) list[i] = i;
        }
    } else {
        select_positions<EACH>(w, len, keep, n_first, n_last, out, list);
    }
    if constexpr (GATHER) {
        __syncthreads();
        auto position = [&](int i) { return i < KEPT_LDS ? list[i] : out[i]; };
        if (dst.weights) {
            float *to = dst.weights + (int64_t)u * dst.stride_w + (int64_t)g * dst.ld_w;
            for (int i = t; i < n; i += ST) to[i] = w[position(i)];
        }
        constexpr int C = 16 / sizeof(T);
        const int pieces = d_head / C;
        const T *k_from = (const T *)src.k + (int64_t)u * src.stride_k + g * d_head;
        T *k_to = (T *)dst.k + (int64_t)u * dst.stride_k + g * d_head;
        const int across = min(pieces, ST), rows = ST / across, c0 = t % across;   // a thread keeps to its pieces of the rows
        if (t / across < rows)
            for (int c = c0 * C; c < d_head; c += across * C)
                for (int i0 = t / across; i0 < n; i0 += KP * rows) {
                    uint4 v[KP];
#pragma unroll
                    for (int e = 0; e < KP; ++e)
                        v[e] = *reinterpret_cast<const uint4 *>(k_from + (int64_t)position(min(i0 + e * rows, n - 1)) * src.ld_k + c);
#pragma unroll
                    for (int e = 0; e < KP; ++e)
                        if (i0 + e * rows < n) *reinterpret_cast<uint4 *>(k_to + (int64_t)(i0 + e * rows) * dst.ld_k + c) = v[e];
                }
        for (int i0 = 0; i0 < n; i0 += VPOS)
            gather_values((const T *)src.vt + (int64_t)u * src.stride_vt + (int64_t)g * d_head * src.ld_vt, src.ld_vt,
                          (T *)dst.vt + (int64_t)u * dst.stride_vt + (int64_t)g * d_head * dst.ld_vt, dst.ld_vt, i0, min(n - i0, VPOS),
                          __builtin_amdgcn_readfirstlane(t >> 6), ST / 64, d_head, position);
    }
}

// The second launch.  Workgroups [0, key_wgs): keys and weights, KP 16-byte pieces a thread; the rest: values of VPOS kept positions and
// VCH channels of one (unit, head).
template <typename T>
__global__ __launch_bounds__(GT) void evict_gather_kernel(SharedSegment src, SharedSegment dst, int n_kv_heads, int d_head, int keep,
                                                          const int32_t *__restrict__ kept, int wgs_per_unit, int64_t key_wgs) {
    constexpr int C = 16 / sizeof(T);
    if ((int64_t)blockIdx.x < key_wgs) {
        const int u = (int)(blockIdx.x / wgs_per_unit), pieces = n_kv_heads * d_head / C, n = min(unit_length(src, u), keep);
        const int64_t x0 = (int64_t)(blockIdx.x % wgs_per_unit) * (GT * KP);
        const int first = (int)(x0 / pieces), rest = (int)(x0 % pieces);
        int from[KP], at[KP], c[KP];
        uint4 v[KP];
#pragma unroll
        for (int e = 0; e < KP; ++e) {
            const int x = rest + threadIdx.x + e * GT;
            at[e] = first + x / pieces;
            c[e] = x % pieces * C;
            from[e] = at[e] < n ? kept[((int64_t)u * n_kv_heads + c[e] / d_head) * keep + at[e]] : -1;
        }
#pragma unroll
        for (int e = 0; e < KP; ++e)
            if (from[e] >= 0) v[e] = *reinterpret_cast<const uint4 *>((const T *)src.k + (int64_t)u * src.stride_k + (int64_t)from[e] * src.ld_k + c[e]);
#pragma unroll
        for (int e = 0; e < KP; ++e) {
            if (from[e] < 0) continue;
            *reinterpret_cast<uint4 *>((T *)dst.k + (int64_t)u * dst.stride_k + (int64_t)at[e] * dst.ld_k + c[e]) = v[e];
            const int g = c[e] / d_head;
            if (dst.weights && c[e] % d_head == 0)
                dst.weights[(int64_t)u * dst.stride_w + (int64_t)g * dst.ld_w + at[e]] = src.weights[(int64_t)u * src.stride_w + (int64_t)g * src.ld_w + from[e]];
        }
        return;
    }
    const int tiles = (keep + VPOS - 1) / VPOS, groups = (d_head + VCH - 1) / VCH;
    const int64_t x = (int64_t)blockIdx.x - key_wgs;
    const int c0 = (int)(x % groups) * VCH, i0 = (int)(x / groups % tiles) * VPOS, ug = (int)(x / groups / tiles), u = ug / n_kv_heads, g = ug % n_kv_heads;
    const int n = min(min(unit_length(src, u), keep) - i0, VPOS);   // positions of this workgroup
    gather_values((const T *)src.vt + (int64_t)u * src.stride_vt + (int64_t)g * d_head * src.ld_vt, src.ld_vt,
                  (T *)dst.vt + (int64_t)u * dst.stride_vt + (int64_t)g * d_head * dst.ld_vt, dst.ld_vt, i0, n, c0 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), GT / 64,
                  min(c0 + VCH, d_head), [&](int i) { return kept[(int64_t)ug * keep + i]; });
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

template <typename T>
void run_evict(const SharedSegment &src, const SharedSegment &dst, int units, int n_kv_heads, int d_head, int dtype, int keep, int n_first, int n_last,
               int32_t *kept, int32_t *kept_lens, hipStream_t st) {
    const int wgs = units * n_kv_heads;
    const int64_t copied = (int64_t)std::min(keep, src.len) * d_head * sizeof(T);   // bytes of keys, and as many of values, per workgroup
    const bool gather = wgs <= MOST_FUSED && copied <= 2048ll * std::max(wgs, 8);
    auto select = [&](auto each, auto fused) {
        hipLaunchKernelGGL((evict_select_kernel<T, decltype(each)::value, decltype(fused)::value>), dim3((unsigned)wgs), dim3(ST), 0, st, src, dst, n_kv_heads,
                           d_head, keep, n_first, n_last, kept, kept_lens);
    };
    auto by_length = [&](auto fused) {
        using std::integral_constant;
        if (src.len <= ST) select(integral_constant<int, 1>(), fused);
        else if (src.len <= 4 * ST) select(integral_constant<int, 4>(), fused);
        else if (src.len <= 16 * ST) select(integral_constant<int, 16>(), fused);
        else if (src.len <= 64 * ST) select(integral_constant<int, 64>(), fused);
        else select(integral_constant<int, 0>(), fused);
    };
    if (gather) {
        by_length(std::true_type());
        return;
    }
    by_length(std::false_type());
    const GatherGrid gr = gather_grid(src, units, n_kv_heads, d_head, dtype, keep);
    const int64_t key_wgs = gr.per_unit * units;
    hipLaunchKernelGGL(evict_gather_kernel<T>, dim3((unsigned)(key_wgs + gr.values)), dim3(GT), 0, st, src, dst, n_kv_heads, d_head, keep, kept,
                       (int)gr.per_unit, key_wgs);
}

}   // namespace

void launch_kv_evict(const SharedSegment &src, const SharedSegment &dst, int units, int n_kv_heads, int d_head, int dtype, int keep, int n_first,
                     int n_last, int32_t *kept, int32_t *kept_lens, hipStream_t st) {
    if (dtype == PSD_DTYPE_BF16) run_evict<bf16_t>(src, dst, units, n_kv_heads, d_head, dtype, keep, n_first, n_last, kept, kept_lens, st);
    else run_evict<float>(src, dst, units, n_kv_heads, d_head, dtype, keep, n_first, n_last, kept, kept_lens, st);
}

bool kv_evict_launchable(const SharedSegment &src, int units, int n_kv_heads, int d_head, int dtype, int keep) {
    const GatherGrid gr = gather_grid(src, units, n_kv_heads, d_head, dtype, keep);
    return launchable((int64_t)units * n_kv_heads, ST) && launchable(gr.per_unit * units + gr.values, GT);
}
