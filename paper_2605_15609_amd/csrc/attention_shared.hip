// Attention of the rows of a batch over keys that its sequences share (psd_attention_shared), and the weight that every key
// draws (psd_attention_weights).
//
// Keys come in segments, coarse to fine.  A unit of a segment is one run of keys that seqs_per_unit consecutive sequences see: a
// prefix of the whole batch (one unit), a cache of a request (its drafts), the rows of a block (one sequence).  For row r and the
// keys j of the units it belongs to
//     x_j = <q_r, k_j> / sqrt(d),   m = max x,   l = sum exp(x_j - m),   o = sum exp(x_j - m) v_j / l,   lse = m + ln l.
// (m, l, sum exp(x_j - m) v_j) over any set of keys can be joined with those over another, so a segment is computed once for all
// rows that see it: the rows of a unit that read one KV head are stacked into tiles, whatever sequence or query head they belong
// to, each tile walks the unit's keys (or, where there are few tiles, a part of them), and a second kernel joins a row's parts.
//
// What bounds it, with bf16 heads of 128: 128 drafts of 64 rows of the 8B shape over 4096 + 1024 + 64 keys take 650 - 670 us, 1.04 -
// 1.07 PFLOP/s (on this card a loop of the same instructions without loads has 1.55, a library product of 8192 cubed 1.22): the matrix
// cores are busy 59 % of a clock that power holds near 1.65 GHz, the rest goes to the exponentials beside them (6 vector instructions a
// product).  32 single rows of the 7B shape over 32768 shared keys take 40 us, 32 of them the attention (67 MB of keys and values): 11
// tiles of keys a workgroup at 2.3 us each, a wait for other wavefronts or for a tile in nearly half of it.  Small calls are one chain
// of round trips: about 8 us.
//
// Per tile the problem is transposed as in attention_mfma.hip: S^T = K Q^T, O^T += V^T P^T.  A lane owns one row; the softmax stays
// in its registers, and the probabilities are the second product's operand as they are.
#include <algorithm>
#include <type_traits>

#include "psd_internal.h"
#include "device_types.h"

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef __attribute__((address_space(3))) void lds_void;

constexpr int TR = 32;    // rows of a tile where there are few
constexpr int MT = 128;   // rows of a tile where there are many
constexpr int BK = 32;    // keys that a wavefront takes at a time
constexpr int KT = 64;    // keys of a tile in LDS
constexpr int NW = 4;     // wavefronts of a workgroup, which deal a tile's keys among themselves
constexpr float SLACK = 8.f;      // (see many_rows)
constexpr float FAR = 0x1p24f;    // (see many_rows)
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

// a Frag out of LDS, chunk by chunk of 16 bytes
template <typename F>
__device__ __forceinline__ void load_chunks(Frag<bf16_t> &f, const unsigned char *lds, F at) {
    f.v = *reinterpret_cast<const uint4 *>(lds + at(0));
}
template <typename F>
__device__ __forceinline__ void load_chunks(Frag<float> &f, const unsigned char *lds, F at) {
    const float4 a = *reinterpret_cast<const float4 *>(lds + at(0)), b = *reinterpret_cast<const float4 *>(lds + at(1));
    f.v[0] = a.x, f.v[1] = a.y, f.v[2] = a.z, f.v[3] = a.w, f.v[4] = b.x, f.v[5] = b.y, f.v[6] = b.z, f.v[7] = b.w;
}

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

// unit u of a launch: which unit of the segment's memory it is, and how many keys that holds (a length outside the unit is cut to it)
__device__ __forceinline__ int cache_of(const SharedSegment &s, int u) {
    return s.rows ? __builtin_amdgcn_readfirstlane(s.rows[(int64_t)u * s.seqs_per_unit]) / s.rows_div : u;
}
__device__ __forceinline__ int unit_keys(const SharedSegment &s, int cache) {
    return s.lens ? __builtin_amdgcn_readfirstlane(min(max(s.lens[cache], 0), s.len)) : s.len;
}
// its keys, as device pointers of one KV head
template <typename T>
struct Keys {
    const T *k, *vt;
    int len;
};
template <typename T>
__device__ __forceinline__ Keys<T> keys_of(const SharedSegment &s, int u, int kvh, int d_head) {
    const int64_t cache = cache_of(s, u);
    Keys<T> r;
    r.k = (const T *)s.k + cache * s.stride_k + kvh * d_head;
    r.vt = (const T *)s.vt + cache * s.stride_vt + (int64_t)kvh * d_head * s.ld_vt;
    r.len = unit_keys(s, cache);
    return r;
}

// A lane's unit: of the job's segment i the j-th from that of sequence s_first on, its place in memory and its keys; none where there is
// no such segment, or the unit starts behind s_last.  One load for all that a workgroup needs: taken one by one, each is a round trip to memory.
__device__ __forceinline__ void unit_of_lane(const SharedLaunch &ln, const SharedJob &jb, int i, int64_t s_first, int j, int64_t s_last, int &cache, int &keys) {
    const SharedSegment *s = &ln.seg[jb.seg];
    const int *lens = s->lens, *rows = s->rows;
    int spu = s->seqs_per_unit, most = s->len, div = s->rows_div;
    for (int n = 1; n < jb.segs; ++n) {
        const SharedSegment &o = ln.seg[jb.seg + n];
        if (i == n) lens = o.lens, rows = o.rows, spu = o.seqs_per_unit, most = o.len, div = o.rows_div;
    }
    const int u = (int)s_first / spu + j;
    cache = keys = 0;
    if (i < jb.segs && (int64_t)u * spu <= s_last) {
        cache = rows ? rows[(int64_t)u * spu] / div : u;
        keys = lens ? min(max(lens[cache], 0), most) : most;
    }
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

// A job's workgroups are dealt to the XCDs in runs of equal length: (unit, KV head, part) by (unit, KV head, part), the tiles of one
// behind one another, so that those that read the same keys meet in one L2.  False: a workgroup of the padding.
struct Place {
    int u, kvh, split, tile;
};
__device__ __forceinline__ bool place_of(const SharedJob &jb, int n_kv_heads, Place &p) {
    const int n = jb.units * n_kv_heads * jb.splits * jb.tiles, run = (n + 7) / 8;
    const int local = blockIdx.x - jb.block0, at = (local & 7) * run + (local >> 3);
    if (at >= n) return false;
    const int grp = at / jb.tiles;
    p = {grp / jb.splits / n_kv_heads, grp / jb.splits % n_kv_heads, grp % jb.splits, at % jb.tiles};
    return true;
}

// Where a row's result over the keys of one workgroup goes: a part that the join reads, or, where it is the only one, the output
template <typename T, int DH>
struct PartOut {
    const SharedLaunch &ln;
    const bool direct;
    int64_t at;      // of the row in [parts][n_rows], or among the rows
    float *o;
    T *out;
    __device__ PartOut(const SharedShape &sh, const SharedLaunch &l, int part, const RowOf &row) : ln(l), direct(l.parts == 0) {
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

// Few rows: a tile of TR rows of a unit of the job's last segment against a part of the keys that they see in the job's segments.  The
// wavefronts deal the keys, BK at a time, operands straight from memory, and merge in LDS in wavefront order.  A job of several segments
// reads the keys of the coarser ones once for every tile, which pays where one launch then does what two would (4 rows of 8 heads of 64
// channels over 256 shared and 61 own keys: 11.4 us with parts and a join, 9.2 so).
// W = 1: the workgroup's wavefronts have a unit each, where there are many units of few keys (184 single rows of the 8B shape, 4510 keys
// shared and one their own: 83 us, 52 so; 300 single rows of 8 heads of 64, 800 shared and 120 own: 30, 24; up to 256 own: no difference).
template <typename T, int DH, int W>
__device__ __forceinline__ void few_rows(const T *__restrict__ q, const SharedShape &sh, const SharedLaunch &ln, const SharedJob &jb, int u, int kvh,
                                         int tile, int split, float sl2, float *part /* [wavefront][max, sum, NF values][64 lanes] */) {
    constexpr int KS = DH / 16, CT = (DH + 31) / 32, NF = CT * 16;   // contraction steps of the scores, channel subtiles, output values per lane
    const int spu = ln.seg[jb.seg + jb.segs - 1].seqs_per_unit;
    const int lane = threadIdx.x & 63, wave = W > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : 0, lrow = lane & 31, half = lane >> 5;
    const int rows = spu * sh.L * (sh.n_heads / sh.n_kv_heads), r = tile * TR + lrow;
    const RowOf row(sh, (int64_t)u * spu, kvh, min(r, rows - 1));   // (rows past the last repeat it and store nothing)
    // lane i: the unit of the job's segment i that holds the rows (see many_rows)
    int lane_cache, lane_keys;
    unit_of_lane(ln, jb, lane, (int64_t)u * spu, 0, (int64_t)u * spu, lane_cache, lane_keys);
    // a step: BK keys of one segment, from k0 on
    struct Step {
        const T *k, *vt;
        int ld_k, ld_vt, k0, keys, seg, end;   // end: the first step behind the segment
    };
    int n_steps = 0;
    for (int i = 0; i < jb.segs; ++i) n_steps += (__builtin_amdgcn_readlane(lane_keys, i) + BK - 1) / BK;
    const int first = (int)((int64_t)n_steps * split / jb.splits), last = (int)((int64_t)n_steps * (split + 1) / jb.splits);
    auto go = [&](Step &s, int st) {   // forward to step st
        if (st >= s.end) {
            int begin;
            do {
                begin = s.end;
                s.keys = __builtin_amdgcn_readlane(lane_keys, ++s.seg);
                s.end += (s.keys + BK - 1) / BK;
            } while (st >= s.end);
            const SharedSegment &seg = ln.seg[jb.seg + s.seg];
            const int64_t cache = __builtin_amdgcn_readlane(lane_cache, s.seg);
            s.k = (const T *)seg.k + cache * seg.stride_k + kvh * DH;
            s.vt = (const T *)seg.vt + cache * seg.stride_vt + (int64_t)kvh * DH * seg.ld_vt;
            s.ld_k = seg.ld_k;
            s.ld_vt = seg.ld_vt;
            s.k0 = (st - begin) * BK;
            return;
        }
        s.k0 += W * BK;
    };
    Frag<T> qf[KS];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qf[ks].load(q + row.token * sh.ld_q + row.head * DH + ks * 16 + half * 8);

    floatx16 acc_o[CT];
#pragma unroll
    for (int ct = 0; ct < CT; ++ct)
#pragma unroll
        for (int v = 0; v < 16; ++v) acc_o[ct][v] = 0.f;
    // bf16: keys of the next step go out when the scores of this one are done, its values before them: a step is one round trip to memory
    // where it would be two (4 rows of 8 heads of 64 channels over 317 keys: 8.4 us, 9.2 without).  fp32 (slower
    // products, twice the registers) gains nothing: 8.8 us and 8.6 without at 48 rows of 8 heads of 64 over 426 keys.
    constexpr bool AHEAD = sizeof(T) == 2;
    float m_run = -INFINITY, neg_m = 0.f, l_run = 0.f;   // (as in many_rows)
    bool far = false;
    Frag<T> kf[KS], vf[BK / 16][CT];
    auto load_keys = [&](const Step &s) {
        const T *krow = s.k + (int64_t)min(s.k0 + lrow, s.keys - 1) * s.ld_k + half * 8;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) kf[ks].load(krow + ks * 16);
    };
    auto load_values = [&](const Step &s, int k0, int kg) {
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
            const int c = CT * 32 > DH ? min(lrow, DH - 1) : ct * 32 + lrow;
            vf[kg][ct].load(s.vt + (int64_t)c * s.ld_vt + k0 + kg * 16 + half * 8);
        }
    };
    Step next = {nullptr, nullptr, 0, 0, 0, 0, -1, 0};
    if (first + wave < last) {
        go(next, first + wave);
        if (AHEAD) load_keys(next);
    }
    for (int st = first + wave; st < last; st += W) {
        const Step here = next;
        const int k0 = here.k0, left = here.keys - k0;
        if constexpr (!AHEAD) load_keys(here);
        if constexpr (AHEAD) {
            load_values(here, k0, 0);
            load_values(here, left > 16 ? k0 : k0 - 16, 1);   // (a value row ends with the group of 16 that its last key is in)
        }
        floatx16 x;
#pragma unroll
        for (int v = 0; v < 16; ++v) x[v] = 0.f;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) product(kf[ks], qf[ks], x);
        if (st + W < last) {
            go(next, st + W);
            if (AHEAD) load_keys(next);
        }
        // x[v] <-> key 8 (v / 4) + 4 half + v % 4 of the step
        if (left < BK) {
#pragma unroll
            for (int v = 0; v < 16; ++v)
                if (8 * (v >> 2) + 4 * half + (v & 3) >= left) x[v] = -INFINITY;
        }
        float mx = x[0];
#pragma unroll
        for (int v = 1; v < 16; ++v) mx = fmaxf(mx, x[v]);
        mx = both_max(mx);
        const float over = (mx - m_run) * sl2;   // (NaN where there is no score yet, which raises nothing)
        if (__any(over > SLACK)) {   // (as in many_rows)
            const bool raised = over > SLACK;
            const float alpha = raised ? __builtin_amdgcn_exp2f(-over) : 1.f;
            l_run *= alpha;
            m_run = raised ? mx : m_run;
            neg_m = raised ? -mx * sl2 : neg_m;
            far = __any(fabsf(neg_m) > FAR);
#pragma unroll
            for (int ct = 0; ct < CT; ++ct)
#pragma unroll
                for (int v = 0; v < 16; ++v) acc_o[ct][v] *= alpha;
        }
        float shift = neg_m;
        if (far) {
            const float ref = fabsf(neg_m) > FAR ? m_run : 0.f;
            if (fabsf(neg_m) > FAR) shift = 0.f;
#pragma unroll
            for (int v = 0; v < 16; ++v) x[v] -= ref;
        }
        float p[16], psum[2] = {0.f, 0.f};
#pragma unroll
        for (int v = 0; v < 16; ++v) {
            p[v] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[v], sl2, shift));
            psum[v & 1] += p[v];
        }
        l_run += psum[0] + psum[1];
#pragma unroll
        for (int kg = 0; kg < BK / 16; ++kg) {
            if (kg * 16 >= left) break;
            Frag<T> pf;
            probabilities(p + 8 * kg, pf);
            if constexpr (!AHEAD) load_values(here, k0, kg);
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) {
                // slots behind the last key hold anything: their probabilities are zero, but 0 x NaN is NaN
                if (left < BK) vf[kg][ct].keep(left - kg * 16 - 4 * half);
                product(vf[kg][ct], pf, acc_o[ct]);
            }
        }
    }
    l_run = both_sum(l_run);   // the halves of a row hold disjoint keys

    if constexpr (W == 1) {
        if (r >= rows) return;
        const PartOut<T, DH> to(sh, ln, jb.part0 + split, row);
        if (half == 0) to.sums(m_run, l_run, sl2);
        const float inv = to.factor(l_run);
        if (inv == 0.f && !to.direct) return;
#pragma unroll
        for (int g = 0; g < NF / 4; ++g) {
            const int c = (g >> 2) * 32 + 8 * (g & 3) + 4 * half;
            const float o[4] = {acc_o[g >> 2][4 * (g & 3)], acc_o[g >> 2][4 * (g & 3) + 1], acc_o[g >> 2][4 * (g & 3) + 2], acc_o[g >> 2][4 * (g & 3) + 3]};
            if (c < DH) to.values(c, o, inv);
        }
        return;
    }
    float *mine = part + wave * (2 + NF) * 64 + lane;
    mine[0] = m_run;
    mine[64] = l_run;
#pragma unroll
    for (int ct = 0; ct < CT; ++ct)
#pragma unroll
        for (int v = 0; v < 16; ++v) mine[(2 + ct * 16 + v) * 64] = acc_o[ct][v];
    __syncthreads();
    float scale[NW], m_all = -INFINITY, l_all = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
        scale[w] = part[w * (2 + NF) * 64 + lane];
        m_all = fmaxf(m_all, scale[w]);
    }
    const float ref = m_all == -INFINITY ? 0.f : m_all;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
        scale[w] = __builtin_amdgcn_exp2f((scale[w] - ref) * sl2);
        l_all += part[(w * (2 + NF) + 1) * 64 + lane] * scale[w];
    }
    if (r >= rows) return;
    const PartOut<T, DH> to(sh, ln, jb.part0 + split, row);
    if (wave == 0 && half == 0) to.sums(m_all, l_all, sl2);
    const float inv = to.factor(l_all);
    if (inv == 0.f && !to.direct) return;   // (no keys: the join reads no values)
#pragma unroll
    for (int g = 0; g < NF / 4; ++g) {   // 4 values of a row: subtile g / 4, channels 8 (g % 4) + 4 half ..
        if (g % NW != wave) continue;
        const int c = (g >> 2) * 32 + 8 * (g & 3) + 4 * half;
        if (c >= DH) continue;
        float o[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < NW; ++w)
#pragma unroll
            for (int v = 0; v < 4; ++v) o[v] += part[(w * (2 + NF) + 2 + g * 4 + v) * 64 + lane] * scale[w];
        to.values(c, o, inv);
    }
}

// Many rows (bf16): a tile of 128 rows, 32 to a wavefront, walks tiles of 64 keys that pass through LDS, fetched a tile ahead by
// loads that go to LDS directly (chunks of 16 bytes swizzled on the way, as in attention_mfma.hip).  The rows of the tile share the unit
// of the job's first segment; of the others the tile walks every unit that one of its rows sees, and hides it from the rows that do not.
// The keys of one unit are a run.  The rows of a wavefront see a run as a whole or not at all (walked_tiles), so a wavefront leaves out the
// tiles that its rows do not see and masks only the last tile of a unit.
// Tried and slower at 128 drafts of the 8B shape (where this took 745 us): 256 rows and 8 wavefronts, in step or half a tile apart 813 and
// more; halves of a tile pipelined, the exponentials of one beside the products of two others, 786; three tiles under way 860.
struct Run {
    const bf16_t *k, *vt;             // at its first tile
    int ld_k, ld_vt, keys, tiles;     // keys from there on, tiles of this workgroup
    int seqs_per_unit, u;
};

template <int DH>
__device__ __forceinline__ void many_rows(const bf16_t *__restrict__ q, const SharedShape &sh, const SharedLaunch &ln, const SharedJob &jb, int u0,
                                          int kvh, int tile, int split, float sl2, unsigned char *lds) {
    constexpr int KROW = DH * 2, VROW = KT * 2, K_BYTES = KT * KROW, STAGE = K_BYTES + DH * VROW, CT = DH / 32, KS = DH / 16;
    constexpr int KRPI = 1024 / KROW, KLPR = 64 / KRPI;      // key rows of a load instruction, lanes to a row
    constexpr int KG = KT / KRPI / NW, VG = DH / 8 / NW;     // load instructions per wavefront and tile
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lrow = lane & 31, half = lane >> 5;
    const int group = sh.n_heads / sh.n_kv_heads, per_seq = sh.L * group;
    const int rows = ln.seg[jb.seg].seqs_per_unit * per_seq, r = tile * MT + wave * 32 + lrow;
    const int s0 = u0 * ln.seg[jb.seg].seqs_per_unit;
    const int s_first = s0 + tile * MT / per_seq, s_last = s0 + (min(tile * MT + MT, rows) - 1) / per_seq;
    const RowOf row(sh, s0, kvh, min(r, rows - 1));   // (rows past the last repeat it and store nothing)
    const int my_seq = s0 + (tile * MT + wave * 32) / per_seq, end_seg = jb.seg + jb.segs;   // (of all rows of the wavefront, where it matters)
    const bool any_rows = tile * MT + wave * 32 < rows;

    int lane_cache, lane_keys;   // lane 16 i + j: of segment i the j-th unit that the tile touches (at most 8, see walked_tiles)
    unit_of_lane(ln, jb, lane >> 4, s_first, lane & 15, s_last, lane_cache, lane_keys);
    // this workgroup's share of the key tiles
    int n_tiles = (lane_keys + KT - 1) / KT;
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) n_tiles += __shfl_xor(n_tiles, d, 64);
    n_tiles = __builtin_amdgcn_readfirstlane(n_tiles);
    int skip = (int)((int64_t)n_tiles * split / jb.splits), budget = (int)((int64_t)n_tiles * (split + 1) / jb.splits) - skip;
    int at_seg = jb.seg, at_u = 0;   // (counted from the first that the tile touches)
    auto next_run = [&](Run &run) {
        while (budget > 0 && at_seg < end_seg) {
            const SharedSegment &s = ln.seg[at_seg];
            const int u0 = s_first / s.seqs_per_unit, u = u0 + at_u, from = (at_seg - jb.seg) * 16 + at_u;
            if (u < s_last / s.seqs_per_unit) ++at_u;
            else ++at_seg, at_u = 0;
            const int64_t cache = __builtin_amdgcn_readlane(lane_cache, from);
            const int keys = __builtin_amdgcn_readlane(lane_keys, from), tiles = (keys + KT - 1) / KT;
            if (skip >= tiles) {
                skip -= tiles;
                continue;
            }
            run.k = (const bf16_t *)s.k + cache * s.stride_k + kvh * DH + (int64_t)skip * KT * s.ld_k;
            run.vt = (const bf16_t *)s.vt + cache * s.stride_vt + (int64_t)kvh * DH * s.ld_vt + skip * KT;
            run.ld_k = s.ld_k;
            run.ld_vt = s.ld_vt;
            run.keys = keys - skip * KT;
            run.tiles = min(tiles - skip, budget);
            run.seqs_per_unit = s.seqs_per_unit;
            run.u = u;
            skip = 0;
            budget -= run.tiles;
            return true;
        }
        return false;
    };

    bf16x8 qf[KS];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
        qf[ks] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const uint4 *>(q + row.token * sh.ld_q + row.head * DH + ks * 16 + half * 8));

    // swizzle keys, as in attention_mfma.hip.  Those of the rows that a lane fetches do not depend on the instruction.
    auto kkey = [](int x) { return DH == 128 ? (x & 15) : ((x >> 1) & 7); };
    const int k_row = lane / KLPR, k_chunk = ((lane % KLPR) ^ kkey(wave * KRPI + k_row)) << 4;
    const int v_row = lane >> 3, v_chunk = ((lane & 7) ^ (((wave * 8 + v_row) >> 1) & 7)) << 4;
    auto fetch = [&](const Run &run, int i, int stage) {   // tile i; what lies behind its keys is rejected by the descriptors or never used
        const int left = min(run.keys - i * KT, KT);
        const __amdgpu_buffer_rsrc_t rk = __builtin_amdgcn_make_buffer_rsrc(const_cast<bf16_t *>(run.k) + (int64_t)i * KT * run.ld_k, 0,
                                                                            ((left - 1) * run.ld_k + DH) * 2, 0x00020000);
        const __amdgpu_buffer_rsrc_t rv = __builtin_amdgcn_make_buffer_rsrc(const_cast<bf16_t *>(run.vt) + i * KT, 0,
                                                                            ((DH - 1) * run.ld_vt + (left + 15) / 16 * 16) * 2, 0x00020000);
        unsigned char *sk = lds + stage * STAGE + wave * 1024, *sv = sk + K_BYTES;
        const int k_off = k_row * run.ld_k * 2 + k_chunk, v_off = v_row * run.ld_vt * 2 + v_chunk;
#pragma unroll
        for (int j = 0; j < KG; ++j)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rk, (lds_void *)(sk + j * (NW * 1024)), 16, k_off, (j * NW + wave) * KRPI * run.ld_k * 2, 0, 0);
#pragma unroll
        for (int j = 0; j < VG; ++j)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rv, (lds_void *)(sv + j * (NW * 1024)), 16, v_off, (j * NW + wave) * 8 * run.ld_vt * 2, 0, 0);
    };

    floatx16 acc_o[CT];
#pragma unroll
    for (int i = 0; i < CT; ++i)
#pragma unroll
        for (int v = 0; v < 16; ++v) acc_o[i][v] = 0.f;
    float m_run = -INFINITY, neg_m = 0.f, l_run = 0.f;   // the reference of the exponentials, and minus it in units of log2 (0: no score yet)
    bool far = false;                                    // a row of the wavefront has a reference beyond FAR

    // the addresses of a lane's fragments within a stage
    int k_at[KS], v_at[4];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) k_at[ks] = lrow * KROW + (((ks * 2 + half) ^ kkey(lrow)) << 4);   // (32 rows further: the same key)
#pragma unroll
    for (int kg = 0; kg < 4; ++kg) v_at[kg] = K_BYTES + lrow * VROW + (((kg * 2 + half) ^ ((lrow >> 1) & 7)) << 4);

    auto scores = [&](const unsigned char *st, floatx16 (&x)[2]) {
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
            for (int v = 0; v < 16; ++v) x[kt][v] = 0.f;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)
#pragma unroll
            for (int kt = 0; kt < 2; ++kt)
                x[kt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*reinterpret_cast<const bf16x8 *>(st + k_at[ks] + kt * 32 * KROW), qf[ks], x[kt], 0, 0, 0);
    };
    // The sums are kept relative to a running reference, raised to the maximum only where that has grown by more than 2^SLACK in a
    // probability: bf16 and fp32 are as exact there, and the outputs are not touched in most tiles.  A row that has not grown keeps its
    // reference when others of the wavefront raise theirs (its factor is 1), so its bits do not depend on what other sequences hold.
    // Returns what the exponentials add to x sl2.  That is minus the reference in units of log2, rounded: off by up to half a unit up to FAR,
    // which is a factor of all of the row's terms, but beyond FAR by more than they span; there x is taken relative to the reference before it
    // is scaled.
    auto reference = [&](floatx16 (&x)[2]) {
        float mx = fmaxf(x[0][0], x[1][0]);
#pragma unroll
        for (int v = 1; v < 16; ++v) mx = fmaxf(fmaxf(mx, x[0][v]), x[1][v]);
        mx = both_max(mx);
        const float over = (mx - m_run) * sl2;   // (NaN where there is no score yet, which raises nothing)
        if (__any(over > SLACK)) {
            const bool raised = over > SLACK;
            const float alpha = raised ? __builtin_amdgcn_exp2f(-over) : 1.f;
            l_run *= alpha;
            m_run = raised ? mx : m_run;
            neg_m = raised ? -mx * sl2 : neg_m;
            far = __any(fabsf(neg_m) > FAR);
#pragma unroll
            for (int ct = 0; ct < CT; ++ct)
#pragma unroll
                for (int v = 0; v < 16; ++v) acc_o[ct][v] *= alpha;
        }
        float shift = neg_m;
        if (far) {
            const float ref = fabsf(neg_m) > FAR ? m_run : 0.f;
            if (fabsf(neg_m) > FAR) shift = 0.f;
#pragma unroll
            for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                for (int v = 0; v < 16; ++v) x[kt][v] -= ref;
        }
        return shift;
    };
    auto exponentials = [&](const floatx16 (&x)[2], float shift, bf16x8 (&pf)[4]) {
        float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                float p[8];
#pragma unroll
                for (int v = 0; v < 8; ++v) {
                    p[v] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[kt][8 * e + v], sl2, shift));
                    sum[v & 3] += p[v];
                }
                pf[kt * 2 + e] = __builtin_bit_cast(bf16x8, make_uint4(pack_bf16x2(p[0], p[1]), pack_bf16x2(p[2], p[3]), pack_bf16x2(p[4], p[5]),
                                                                       pack_bf16x2(p[6], p[7])));
            }
        l_run += (sum[0] + sum[1]) + (sum[2] + sum[3]);
    };

    Run run, next;
    bool more = next_run(run);
    int stage = 0;
    if (more) fetch(run, 0, 0);
    while (more) {
        const bool after = next_run(next);
        const bool seen = any_rows && (jb.segs == 1 || my_seq / run.seqs_per_unit == run.u);
        for (int i = 0; i < run.tiles; ++i, stage ^= 1) {
            // this tile has landed for every wavefront, and every wavefront is done with the stage that the next one goes to
            asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
            if (i + 1 < run.tiles) fetch(run, i + 1, stage ^ 1);
            else if (after) fetch(next, 0, stage ^ 1);
            if (!seen) continue;
            const unsigned char *st = lds + stage * STAGE;
            const int left = run.keys - i * KT;
            floatx16 x[2];
            scores(st, x);
            // the values are under way while the exponentials are computed
            Frag<bf16_t> vf[4][CT];
#pragma unroll
            for (int kg = 0; kg < 4; ++kg)
#pragma unroll
                for (int ct = 0; ct < CT; ++ct) vf[kg][ct].v = *reinterpret_cast<const uint4 *>(st + v_at[kg] + ct * 32 * VROW);
            // 6 fragments under way before the first product, then one for each (16 blocks of 32 rows over 1024 + 288 keys, 8B shape: 39.5 us
            // where every product waits for its own read, 36 so)
            __builtin_amdgcn_sched_group_barrier(0x100, 6, 0);
#pragma unroll
            for (int j = 0; j < 2 * KS; ++j) {
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
            }
            asm volatile("" ::: "memory");
            if (left < KT) {   // the last tile of a unit.  Values behind the last key are cleared too: 0 x NaN is NaN
#pragma unroll
                for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                    for (int v = 0; v < 16; ++v)
                        if (kt * 32 + 8 * (v >> 2) + 4 * half + (v & 3) >= left) x[kt][v] = -INFINITY;
#pragma unroll
                for (int kg = 0; kg < 4; ++kg)
#pragma unroll
                    for (int ct = 0; ct < CT; ++ct) vf[kg][ct].keep(left - kg * 16 - 4 * half);
            }
            const float shift = reference(x);
            bf16x8 pf[4];
            exponentials(x, shift, pf);
#pragma unroll
            for (int kg = 0; kg < 4; ++kg)
#pragma unroll
                for (int ct = 0; ct < CT; ++ct)
                    acc_o[ct] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, vf[kg][ct].v), pf[kg], acc_o[ct], 0, 0, 0);
        }
        run = next;
        more = after;
    }
    l_run = both_sum(l_run);   // the halves of a row hold disjoint keys
    if (r >= rows) return;
    const PartOut<bf16_t, DH> to(sh, ln, jb.part0 + split, row);
    if (half == 0) to.sums(m_run, l_run, sl2);
    const float f = to.factor(l_run);
    if (f == 0.f && !to.direct) return;
#pragma unroll
    for (int ct = 0; ct < CT; ++ct)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const float o[4] = {acc_o[ct][4 * g], acc_o[ct][4 * g + 1], acc_o[ct][4 * g + 2], acc_o[ct][4 * g + 3]};
            to.values(ct * 32 + 8 * g + 4 * half, o, f);
        }
}

template <typename T, int DH>
constexpr int attention_lds() {
    constexpr int merge = NW * (2 + (DH + 31) / 32 * 16) * 64 * 4, ring = sizeof(T) == 2 ? 2 * (KT * DH * 2 + DH * KT * 2) : 0;
    return merge > ring ? merge : ring;
}

template <typename T, int DH>
__global__ __launch_bounds__(NW * 64, 2) void shared_attention_kernel(const T *__restrict__ q, SharedShape sh, SharedLaunch ln, float sl2) {
    extern __shared__ __align__(16) unsigned char lds[];
    int j = 0;
    while (j + 1 < ln.n_jobs && (int)blockIdx.x >= ln.job[j + 1].block0) ++j;
    const SharedJob &jb = ln.job[j];
    if (jb.packed) {
        const int n = jb.units * sh.n_kv_heads, run = ((n + NW - 1) / NW + 7) / 8, local = blockIdx.x - jb.block0;
        const int of = __builtin_amdgcn_readfirstlane(((local & 7) * run + (local >> 3)) * NW + (threadIdx.x >> 6));
        if (local >> 3 < run && of < n) few_rows<T, DH, 1>(q, sh, ln, jb, of / sh.n_kv_heads, of % sh.n_kv_heads, 0, 0, sl2, nullptr);
        return;
    }
    Place at;
    if (!place_of(jb, sh.n_kv_heads, at)) return;
    if constexpr (sizeof(T) == 2) {
        if (jb.tiled) {
            many_rows<DH>(q, sh, ln, jb, at.u, at.kvh, at.tile, at.split, sl2, lds);
            return;
        }
    }
    few_rows<T, DH, NW>(q, sh, ln, jb, at.u, at.kvh, at.tile, at.split, sl2, reinterpret_cast<float *>(lds));
}

// The parts of a row joined: a thread takes 4 channels of every G-th part, and the G sums, each relative to a maximum of its own, are
// joined in order.  G = 8 where there are many parts of few rows: every load is a round trip to memory, so as many as possible are
// under way at a time (896 rows of 60 parts: 21 us with one loop over all maxima in front, 5.8 without).
template <typename T, int DH, int G>
__global__ __launch_bounds__(256) void shared_join_kernel(SharedShape sh, SharedLaunch ln, float sl2) {
    constexpr int TPR = DH / 4, RPW = 256 / (TPR * G);   // threads per part, rows per workgroup
    static_assert(RPW >= 1, "a row's threads are one workgroup");
    __shared__ float4 sums[G > 1 ? 256 : 1];
    __shared__ float2 stats[G > 1 ? 256 : 1];
    const int64_t r = (int64_t)blockIdx.x * RPW + threadIdx.x / (TPR * G);
    const int g = threadIdx.x / TPR % G, c = threadIdx.x % TPR * 4;
    const bool live = r < sh.n_rows;
    const float2 *ml = ln.ml + (live ? r : 0);
    const float *op = ln.o + (live ? r : 0) * DH + c;
    constexpr int B = 8;   // parts at a time
    float m = -INFINITY, l = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
    for (int p0 = g; p0 < ln.parts; p0 += G * B) {
        float2 s[B];
        float4 v[B];
#pragma unroll
        for (int i = 0; i < B; ++i) {
            const int64_t at = (int64_t)min(p0 + i * G, ln.parts - 1) * sh.n_rows;
            s[i] = ml[at];
            v[i] = *reinterpret_cast<const float4 *>(op + at * DH);
            if (p0 + i * G >= ln.parts) s[i] = make_float2(-INFINITY, 0.f);
        }
        float top = m;
#pragma unroll
        for (int i = 0; i < B; ++i) top = fmaxf(top, s[i].x);
        const float ref = top == -INFINITY ? 0.f : top, a = __builtin_amdgcn_exp2f((m - ref) * sl2);
        l *= a, o[0] *= a, o[1] *= a, o[2] *= a, o[3] *= a;
        m = top;
#pragma unroll
        for (int i = 0; i < B; ++i) {
            const bool none = s[i].y == 0.f;   // (values that were never written may be anything)
            const float w = none ? 0.f : __builtin_amdgcn_exp2f((s[i].x - ref) * sl2);
            l += w * s[i].y;
            o[0] += none ? 0.f : w * v[i].x, o[1] += none ? 0.f : w * v[i].y, o[2] += none ? 0.f : w * v[i].z, o[3] += none ? 0.f : w * v[i].w;
        }
    }
    if constexpr (G > 1) {
        sums[threadIdx.x] = make_float4(o[0], o[1], o[2], o[3]);
        stats[threadIdx.x] = make_float2(m, l);
        __syncthreads();
        if (g > 0) return;
#pragma unroll
        for (int i = 1; i < G; ++i) m = fmaxf(m, stats[threadIdx.x + i * TPR].x);
        const float ref = m == -INFINITY ? 0.f : m;
        l = o[0] = o[1] = o[2] = o[3] = 0.f;
#pragma unroll
        for (int i = 0; i < G; ++i) {
            const float2 s = stats[threadIdx.x + i * TPR];
            const float4 v = sums[threadIdx.x + i * TPR];
            const float w = __builtin_amdgcn_exp2f((s.x - ref) * sl2);
            l += w * s.y;
            o[0] += w * v.x, o[1] += w * v.y, o[2] += w * v.z, o[3] += w * v.w;
        }
    }
    if (!live) return;
    const float inv = l == 0.f ? 0.f : 1.0f / l;   // (a row without keys: zeros)
    T *to = (T *)ln.out + r / sh.n_heads * sh.ld_out + r % sh.n_heads * DH + c;
    if constexpr (sizeof(T) == 2) *reinterpret_cast<uint2 *>(to) = make_uint2(pack_bf16x2(o[0] * inv, o[1] * inv), pack_bf16x2(o[2] * inv, o[3] * inv));
    else *reinterpret_cast<float4 *>(to) = make_float4(o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv);
    if (ln.lse && c == 0) ln.lse[r] = PartOut<T, DH>::log_sum(m, l, sl2);
}

// w[j] (+)= sum over the rows of the unit of exp(x_j - lse).  A wavefront keeps 32 NK keys in registers, a workgroup four times as many, and
// walks the rows in tiles of WR that pass through LDS, fetched a tile ahead; a lane adds up what its row of every tile gives, and the
// lanes are added at the end.  Where a unit has few keys and many rows, workgroups take a part of the rows each and a second kernel
// adds the parts.  Every sum has an order that the shapes alone decide.
// 16 x 64 rows of the 7B shape over 2048 shared and up to 4001 own keys take 60 - 64 us, 0.33 PFLOP/s (the attention before it 92 - 96, its
// join 12).  The exponentials, 64 a lane and tile at a quarter of the rate, are some 20 us of that.  The rest is the shape of the launch: of 1280
// workgroups, of which a CU holds two (248 registers), those whose block lies behind a unit's last key leave at once, and each of the others
// loads its 64 KB of keys, with nothing beside it, for some seven tiles of rows.
template <typename T>
constexpr int NKEYS = sizeof(T) == 2 ? 2 : 1;
template <typename T>
constexpr int WROWS = sizeof(T) == 2 ? 64 : 32;

template <typename T, int DH>
__global__ __launch_bounds__(NW * 64, 2) void shared_weights_kernel(const T *__restrict__ q, const float *__restrict__ lse, SharedShape sh, SharedLaunch ln,
                                                                    int accumulate, float sl2) {
    constexpr int NK = NKEYS<T>, WR = WROWS<T>, KS = DH / 16, KPW = 32 * NK, C = 16 / sizeof(T), CH = DH / C, ROW = DH * (int)sizeof(T);
    constexpr int LOADS = (WR * CH + NW * 64 - 1) / (NW * 64), STEP = NW * 64 / CH;   // 16-byte loads per thread and tile, rows from one to the next
    static_assert(WR % STEP == 0 || LOADS == 1, "a thread's loads are of one channel piece");
    __shared__ __align__(16) unsigned char tiles[2][WR * ROW];
    __shared__ float z2[2][WR];
    int j = 0;
    while (j + 1 < ln.n_jobs && (int)blockIdx.x >= ln.job[j + 1].block0) ++j;
    const SharedJob &jb = ln.job[j];
    const SharedSegment &seg = ln.seg[jb.seg];
    Place at;   // (tile: block of keys; all blocks of a unit, KV head and part read the same rows)
    if (!place_of(jb, sh.n_kv_heads, at)) return;
    const int u = at.u, kvh = at.kvh, split = at.split, block = at.tile;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lrow = lane & 31, half = lane >> 5;
    const Keys<T> keys = keys_of<T>(seg, u, kvh, DH);
    if (block * NW * KPW >= keys.len) return;
    const int k0 = (block * NW + wave) * KPW;
    Frag<T> kf[NK][KS];
#pragma unroll
    for (int i = 0; i < NK; ++i)
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) kf[i][ks].load(keys.k + (int64_t)min(k0 + i * 32 + lrow, keys.len - 1) * seg.ld_k + ks * 16 + half * 8);
    const int rows = seg.seqs_per_unit * sh.L * (sh.n_heads / sh.n_kv_heads), n_tiles = (rows + WR - 1) / WR;
    const int first = (int)((int64_t)n_tiles * split / jb.splits), last = (int)((int64_t)n_tiles * (split + 1) / jb.splits);
    const int64_t s0 = (int64_t)u * seg.seqs_per_unit;

    // rows pass global -> registers -> LDS, chunks of 16 bytes swizzled so that 32 rows meet all banks
    auto place = [](int row, int chunk) {
        constexpr int PER = ROW >= 256 ? 1 : 256 / ROW, MASK = CH >= 16 ? 15 : CH - 1;   // rows in 256 bytes of LDS
        return row * ROW + ((chunk ^ ((row / PER) & MASK)) << 4);
    };
    // A thread's rows move on by WR a tile: WR / group tokens and WR % group heads, and a token more where the heads of one are through.
    const int group = sh.n_heads / sh.n_kv_heads, tokens = WR / group, heads = WR % group;
    const bool loads = WR * CH >= NW * 64 || tid < WR * CH;
    const T *from[LOADS];
    int head[LOADS];
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
        const int r = first * WR + tid / CH + i * STEP;
        head[i] = r % group;
        from[i] = q + (s0 * sh.L + r / group) * sh.ld_q + (kvh * group + head[i]) * DH + tid % CH * C;
    }
    // (rows past the last one: the unit's first, whose weight is taken away by an infinite z; zeros would make NaN of infinite keys)
    const T *spare = q + s0 * sh.L * sh.ld_q + kvh * group * DH + tid % CH * C;
    int z_head = (first * WR + tid) % group;
    const float *z_from = lse + (s0 * sh.L + (first * WR + tid) / group) * sh.n_heads + kvh * group + z_head;
    uint4 held[LOADS];
    float held_z = 0.f;
    auto fetch = [&](int t) {
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const T *p = from[i];
            if (t * WR + tid / CH + i * STEP >= rows) p = spare;
            held[i] = make_uint4(0, 0, 0, 0);
            if (loads) held[i] = *reinterpret_cast<const uint4 *>(p);
            from[i] += tokens * sh.ld_q + heads * DH;
            head[i] += heads;
            if (head[i] >= group) {
                head[i] -= group;
                from[i] += sh.ld_q - group * DH;
            }
        }
        held_z = INFINITY;   // (rows past the last one give nothing)
        if (tid < WR && t * WR + tid < rows) held_z = *z_from;
        z_from += tokens * sh.n_heads + heads;
        z_head += heads;
        if (z_head >= group) {
            z_head -= group;
            z_from += sh.n_heads - group;
        }
    };
    auto store = [&](int stage) {
#pragma unroll
        for (int i = 0; i < LOADS; ++i)
            if (loads) *reinterpret_cast<uint4 *>(tiles[stage] + place(tid / CH + i * STEP, tid % CH)) = held[i];
        // (a row without a score above -inf gives nothing either)
        if (tid < WR) z2[stage][tid] = held_z == -INFINITY ? INFINITY : held_z * LOG2E;
    };
    float w[NK][16];
#pragma unroll
    for (int i = 0; i < NK; ++i)
#pragma unroll
        for (int v = 0; v < 16; ++v) w[i][v] = 0.f;
    if (first < last) {
        fetch(first);
        store(0);
    }
    for (int t = first; t < last; ++t) {
        const int stage = (t - first) & 1;
        if (t + 1 < last) fetch(t + 1);
        __syncthreads();
#pragma unroll
        for (int rt = 0; rt < WR / 32; ++rt) {
            floatx16 x[NK];
#pragma unroll
            for (int i = 0; i < NK; ++i)
#pragma unroll
                for (int v = 0; v < 16; ++v) x[i][v] = 0.f;
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                Frag<T> qf;
                load_chunks(qf, tiles[stage], [&](int e) { return place(rt * 32 + lrow, (ks * 16 + half * 8) / C + e); });
#pragma unroll
                for (int i = 0; i < NK; ++i) product(kf[i][ks], qf, x[i]);
            }
            const float z = z2[stage][rt * 32 + lrow];
            // Beyond FAR the rounding of lse is more than an exponential spans: what would exceed a probability of 1 counts as 1
            if (__any(fabsf(z) > FAR && fabsf(z) < INFINITY)) {
#pragma unroll
                for (int i = 0; i < NK; ++i)
#pragma unroll
                    for (int v = 0; v < 16; ++v) {
                        const float e = __builtin_fmaf(x[i][v], sl2, -z);
                        w[i][v] += __builtin_amdgcn_exp2f(fabsf(z) > FAR && e > 0.f ? 0.f : e);
                    }
                continue;
            }
#pragma unroll
            for (int i = 0; i < NK; ++i)
#pragma unroll
                for (int v = 0; v < 16; ++v) w[i][v] += __builtin_amdgcn_exp2f(__builtin_fmaf(x[i][v], sl2, -z));
        }
        if (t + 1 < last) store(stage ^ 1);   // (every wavefront has left that stage: it passed the barrier above)
    }
    const int64_t cache = cache_of(seg, u);
    float *to = seg.weights + cache * seg.stride_w + (int64_t)kvh * seg.ld_w;
    float *part = ln.o + jb.part0 * 64ll + ((int64_t)split * jb.units * sh.n_kv_heads + (int64_t)u * sh.n_kv_heads + kvh) * seg.len;
    const bool shift = jb.splits == 1 && accumulate;   // (else the join adds)
    if (jb.splits > 1) to = part;
    // The lanes of a half are added up: each step a lane hands one half of its keys to its partner and takes the partner's share of the
    // others, so that lane x ends with the key of number x (with 16 keys, one step adds without handing over).
    float a[NK * 16];
#pragma unroll
    for (int i = 0; i < NK; ++i)
#pragma unroll
        for (int v = 0; v < 16; ++v) a[i * 16 + v] = w[i][v];
#pragma unroll
    for (int n = NK * 16, d = NK * 8; d > 0; d >>= 1, n >>= 1)
#pragma unroll
        for (int x = 0; x < n / 2; ++x) {
            const bool upper = lane & d;
            const float give = upper ? a[x] : a[x + n / 2], keep = upper ? a[x + n / 2] : a[x];
            a[x] = keep + __shfl_xor(give, d, 64);
        }
    if constexpr (NK == 1) a[0] += __shfl_xor(a[0], 16, 64);
    const int x = lrow % (NK * 16), key = k0 + (x >> 4) * 32 + 8 * ((x & 15) >> 2) + 4 * half + (x & 3);
    if (lrow < NK * 16 && key < keys.len) to[key] = shift ? to[key] + a[0] : a[0];
}

// the parts of weights whose rows were taken by several workgroups, added in order
__global__ __launch_bounds__(256) void weights_join_kernel(SharedShape sh, SharedLaunch ln, int accumulate) {
    int j = 0;
    while (j + 1 < ln.n_jobs && (int)blockIdx.x >= ln.join0[j + 1]) ++j;
    const SharedJob &jb = ln.job[j];
    const SharedSegment &seg = ln.seg[jb.seg];
    const int64_t local = blockIdx.x - ln.join0[j], blocks = (seg.len + 255) / 256;
    const int64_t ug = local / blocks;
    const int u = (int)(ug / sh.n_kv_heads), kvh = (int)(ug % sh.n_kv_heads), key = (int)(local % blocks) * 256 + threadIdx.x;
    const int64_t cache = cache_of(seg, u);
    if (key >= unit_keys(seg, cache)) return;
    const float *part = ln.o + jb.part0 * 64ll + ug * seg.len + key;
    float w = 0.f;
#pragma unroll 4
    for (int s = 0; s < jb.splits; ++s) w += part[(int64_t)s * jb.units * sh.n_kv_heads * seg.len];
    float *to = seg.weights + cache * seg.stride_w + (int64_t)kvh * seg.ld_w + key;
    *to = accumulate ? *to + w : w;
}

__global__ __launch_bounds__(256) void block_values_kernel(const float *__restrict__ qkv, int ld_qkv, int v_col, int L, int width, float *__restrict__ vT,
                                                           int ld_vt) {
    const int64_t s = blockIdx.x / L;
    const int i = blockIdx.x % L;
    for (int c = threadIdx.x; c < width; c += 256) vT[(s * width + c) * ld_vt + vt_key_slot(i)] = qkv[(int64_t)blockIdx.x * ld_qkv + v_col + c];
}

// the join of a launch: lanes of parts to a row (G of its kernel), workgroups
constexpr int MANY_PARTS = 8;
bool many_parts(const SharedLaunch &ln) { return ln.parts >= 16; }
int64_t join_workgroups(const SharedShape &sh, const SharedLaunch &ln) {
    const int rows = 256 / (sh.d_head / 4 * (many_parts(ln) ? MANY_PARTS : 1));
    return (sh.n_rows + rows - 1) / rows;
}

bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

template <typename T, int DH>
void run_attention(const T *q, const SharedShape &sh, const SharedLaunch &ln, hipStream_t st) {
    constexpr int smem = attention_lds<T, DH>();
    const float sl2 = LOG2E / sqrtf((float)DH);
    auto kern = shared_attention_kernel<T, DH>;
    static std::atomic<uint64_t> lds_raised{0};   // one per instantiation
    ensure_dynamic_lds(reinterpret_cast<const void *>(kern), smem, lds_raised);
    if (ln.blocks > 0) hipLaunchKernelGGL(kern, dim3((unsigned)ln.blocks), dim3(NW * 64), smem, st, q, sh, ln, sl2);
    if (ln.blocks > 0 && ln.parts == 0) return;
    const dim3 grid((unsigned)join_workgroups(sh, ln));
    if (many_parts(ln)) hipLaunchKernelGGL((shared_join_kernel<T, DH, MANY_PARTS>), grid, dim3(256), 0, st, sh, ln, sl2);
    else hipLaunchKernelGGL((shared_join_kernel<T, DH, 1>), grid, dim3(256), 0, st, sh, ln, sl2);
}

template <typename T, int DH>
void run_weights(const T *q, const float *lse, const SharedShape &sh, const SharedLaunch &ln, int accumulate, hipStream_t st) {
    if (ln.blocks > 0)
        hipLaunchKernelGGL((shared_weights_kernel<T, DH>), dim3((unsigned)ln.blocks), dim3(NW * 64), 0, st, q, lse, sh, ln, accumulate,
                           LOG2E / sqrtf((float)DH));
    if (ln.join_blocks > 0)
        hipLaunchKernelGGL(weights_join_kernel, dim3((unsigned)ln.join_blocks), dim3(256), 0, st, sh, ln, accumulate);
}

// The work of one launch.  Segments with keys, in order, are cut into jobs: those that a job takes together need no parts, but its
// tiles walk the keys of every finer unit that they touch.  Then the keys of every job are cut so that the workgroups have about as
// much to do each.  Times are in steps of a tile of MT rows against 64 keys with two workgroups on a CU (2.3 us with heads of 128):
// ALONE where a workgroup has the CU to itself, FEW for TR rows against NW * BK keys of
// 256 bytes (what a CU takes of them out of L2 bounds it; fp32: the products too), WG_FIXED what a workgroup costs besides, and what
// the join costs, its launch and the parts' way through memory.
constexpr double ALONE = 0.65, FEW = 1.5, FEW_FP32 = 2.0, WG_FIXED = 2.0, JOIN_FIXED = 1.5, STEP_SECONDS = 2.3e-6, PART_RATE = 6e12;
constexpr int SLOTS = 512;
constexpr int PACKED_STEPS = 4;   // of BK keys: up to there a wavefront takes a unit by itself where there are more of them than SLOTS
constexpr int MOST_TOUCHED = 8;   // units of a finer segment that the tiles of a walk may touch
constexpr int64_t MOST_PART_ROWS = 1 << 17;   // rows times parts, where segments are cut: 1024 tiles of 128 rows
int rows_per_unit(const SharedShape &sh, const SharedSegment &s) { return s.seqs_per_unit * sh.L * (sh.n_heads / sh.n_kv_heads); }

int64_t workgroups(const SharedJob &jb, int n_kv_heads, int splits) {
    const int64_t n = (int64_t)jb.units * n_kv_heads;
    return jb.packed ? (n + NW - 1) / NW : n * jb.tiles * splits;
}

// key tiles of 64 that a tile of MT rows of segments [a, b] walks at most (0: not possible), and as a share of that on average: units of
// lengths of their own are taken to be half full
int walked_tiles(const SharedShape &sh, const SharedSegment *seg, int a, int b, double *full) {
    const int64_t rows = rows_per_unit(sh, seg[a]);
    int64_t keys = 0, half = 0;
    for (int i = a; i <= b; ++i) {
        if (sh.dtype != PSD_DTYPE_BF16 || seg[i].ld_k >= 1 << 23 || seg[i].ld_vt >= 1 << 22) return 0;   // (32-bit offsets within a tile)
        const int64_t fine = rows_per_unit(sh, seg[i]);
        if (i > a && fine % 32) return 0;   // (see many_rows)
        const int64_t touched = i == a ? 1 : std::min<int64_t>((std::min<int64_t>(rows, MT) + fine - 1) / fine + (MT % fine && fine % MT ? 1 : 0), rows / fine);
        if (touched > MOST_TOUCHED) return 0;
        keys += touched * ((seg[i].len + KT - 1) / KT);
        if (seg[i].lens) half += touched * ((seg[i].len + KT - 1) / KT);
    }
    *full = 1.0 - 0.5 * half / std::max<int64_t>(keys, 1);
    return keys > 1 << 30 ? 0 : (int)keys;
}

SharedLaunch plan_attention(const SharedShape &sh, const SharedSegment *given, int n_given) {
    SharedLaunch ln;
    for (int i = 0; i < n_given; ++i)
        if (given[i].len > 0) ln.seg[ln.n_segs++] = given[i];
    const int n = ln.n_segs;
    if (n == 0) return ln;
    const double few = sh.dtype == PSD_DTYPE_BF16 ? FEW * sh.d_head / 128 : FEW_FP32 * sh.d_head / 64;
    double best = -1.0, each_of[kMaxSegments] = {};
    // bit i of a cut: a job ends with segment i.  Jobs of more than one segment: tiles of MT rows of the first one's units, or (the second
    // half of the choices, where the cut has such a job) of TR rows of the last one's, which read the keys of the coarser ones each for itself
    for (int choice = 0; choice < 1 << n; ++choice) {
        const int cut = choice & ((1 << (n - 1)) - 1);
        const bool narrow = choice >> (n - 1);
        if (narrow && cut == (1 << (n - 1)) - 1) continue;
        SharedJob job[kMaxSegments] = {};
        int keys[kMaxSegments], jobs = 0, most = 1;
        double full[kMaxSegments];
        int64_t rows[kMaxSegments];
        bool possible = true;
        for (int a = 0, b = 0; a < n && possible; a = b + 1, ++jobs) {
            b = a;
            while (b < n - 1 && !(cut >> b & 1)) ++b;
            SharedJob &jb = job[jobs];
            const int of = narrow ? b : a, per_unit = rows_per_unit(sh, ln.seg[of]);   // (whose units the job's tiles are cut from)
            jb.tiled = a == b ? per_unit > TR : !narrow;
            keys[jobs] = jb.tiled ? walked_tiles(sh, ln.seg, a, b, full + jobs) : 0;
            if (keys[jobs] == 0 && a == b) jb.tiled = false;
            if (!jb.tiled) {
                int64_t steps = 0, half = 0;
                for (int i = a; i <= b; ++i) {
                    steps += (ln.seg[i].len + BK - 1) / BK;
                    if (ln.seg[i].lens) half += (ln.seg[i].len + BK - 1) / BK;
                }
                full[jobs] = 1.0 - 0.5 * half / steps;
                jb.packed = steps <= PACKED_STEPS && per_unit <= TR && (int64_t)(sh.S / ln.seg[of].seqs_per_unit) * sh.n_kv_heads > SLOTS;
                if (!jb.packed) steps = (steps + NW - 1) / NW;
                keys[jobs] = steps > 1 << 30 ? 0 : (int)steps;
            }
            if (keys[jobs] == 0) possible = false;
            jb.seg = a;
            jb.segs = b - a + 1;
            jb.units = sh.S / ln.seg[of].seqs_per_unit;
            jb.tiles = (per_unit + (jb.tiled ? MT : TR) - 1) / (jb.tiled ? MT : TR);
            rows[jobs] = workgroups(jb, sh.n_kv_heads, 1);
            most = std::max(most, keys[jobs]);
        }
        if (!possible) continue;
        for (int pieces = 1; pieces <= most; pieces += std::max(1, pieces / 8)) {   // of the longest job
            const double share = (double)most / pieces;
            int64_t wgs = 0, parts = 0;
            double longest = 0.0, work = 0.0, each[kMaxSegments];
            int splits[kMaxSegments];
            for (int j = 0; j < jobs; ++j) {
                splits[j] = job[j].packed ? 1 : std::min(keys[j], std::max(1, (int)(keys[j] * (job[j].tiled ? 1.0 : few) / share + 0.999)));
                parts += splits[j];
            }
            if (parts > jobs && parts * sh.n_rows > MOST_PART_ROWS) {   // (a part of every row and job is the least that there is)
                for (int j = 0; j < jobs; ++j) splits[j] = 1;
                parts = jobs;
            }
            for (int j = 0; j < jobs; ++j) {
                const double step = job[j].tiled ? 1.0 : few;
                each[j] = (keys[j] + splits[j] - 1) / splits[j] * step + WG_FIXED;
                longest = std::max(longest, each[j]);
                work += (each[j] - (1.0 - full[j]) * keys[j] / splits[j] * step) * rows[j] * splits[j];
                wgs += rows[j] * splits[j];
            }
            // one round lasts as long as its longest workgroup, many as long as the work
            double cost = wgs <= SLOTS / 2 ? longest * ALONE : std::max(longest, work / SLOTS + (wgs > SLOTS ? longest / 2 : 0.0));
            if (parts > 1) cost += JOIN_FIXED + parts * (double)sh.n_rows * sh.d_head * 8 / PART_RATE / STEP_SECONDS;
            if (best >= 0 && cost >= best) continue;
            best = cost;
            ln.n_jobs = jobs;
            ln.parts = 0;
            ln.blocks = 0;
            for (int j = 0; j < jobs; ++j) {
                SharedJob &jb = ln.job[j];
                jb = job[j];
                jb.splits = splits[j];
                each_of[j] = each[j];
                jb.part0 = ln.parts;
                ln.parts += jb.splits;
                ln.blocks += align_up(rows[j] * jb.splits, 8);
            }
        }
    }
    // long workgroups first, short ones fill what they leave (16 x 64 rows of the 7B shape over 2048 shared and up to 4001 own keys, with
    // weights: 183 us in the order of the segments, 177 so)
    for (int j = 1; j < ln.n_jobs; ++j)
        for (int i = j; i > 0 && each_of[i] > each_of[i - 1]; --i) {
            std::swap(each_of[i], each_of[i - 1]);
            std::swap(ln.job[i], ln.job[i - 1]);
        }
    int64_t block = 0;
    for (int j = 0; j < ln.n_jobs; ++j) {
        SharedJob &jb = ln.job[j];
        jb.block0 = (int)block;   // (grids of 2^24 workgroups and more are refused)
        block += align_up(workgroups(jb, sh.n_kv_heads, jb.splits), 8);
    }
    if (ln.parts == 1) ln.parts = 0;
    return ln;
}

// Weights: a job per segment that collects them; tiles = blocks of keys, splits = parts of the rows.  part0 and parts in units of 64 floats.
SharedLaunch plan_weights(const SharedShape &sh, const SharedSegment *given, int n) {
    SharedLaunch ln;
    const bool bf16 = sh.dtype == PSD_DTYPE_BF16;
    const int per_block = NW * 32 * (bf16 ? NKEYS<bf16_t> : NKEYS<float>), WR = bf16 ? WROWS<bf16_t> : WROWS<float>;
    double total = 0.0;
    for (int i = 0; i < n; ++i) {
        if (!given[i].weights || given[i].len == 0) continue;
        SharedJob &jb = ln.job[ln.n_jobs];
        jb.seg = ln.n_segs;
        ln.seg[ln.n_segs++] = given[i];
        jb.units = sh.S / given[i].seqs_per_unit;
        jb.tiles = (given[i].len + per_block - 1) / per_block;
        total += (double)jb.units * sh.n_kv_heads * jb.tiles * ((rows_per_unit(sh, given[i]) + WR - 1) / WR);
        ++ln.n_jobs;
    }
    // About 768 workgroups with as many tiles of rows each, if every unit is full: one and a half rounds of the two that a CU holds.  A part costs
    // a round trip, so at least 4 tiles.
    const int share = (int)std::max(4.0, std::min(total / 768.0 + 0.999, 1e9));
    int64_t blocks = 0, joins = 0, parts = 0;
    for (int j = 0; j < ln.n_jobs; ++j) {
        SharedJob &jb = ln.job[j];
        const SharedSegment &s = ln.seg[jb.seg];
        jb.splits = ((rows_per_unit(sh, s) + WR - 1) / WR + share - 1) / share;
        jb.block0 = (int)blocks;
        ln.join0[j] = (int)joins;
        jb.part0 = (int)parts;
        const int64_t ug = (int64_t)jb.units * sh.n_kv_heads;
        blocks += align_up(ug * jb.splits * jb.tiles, 8);
        if (jb.splits > 1) {
            joins += ug * ((s.len + 255) / 256);
            parts += (ug * jb.splits * s.len + 63) / 64;
        }
    }
    ln.blocks = blocks;
    ln.join_blocks = joins;
    ln.parts = (int)parts;
    return ln;
}

}   // namespace

bool shared_attention_takes(int dtype, int d_head) {
    return dtype == PSD_DTYPE_BF16 ? d_head == 64 || d_head == 128 : d_head == 16 || d_head == 32 || d_head == 64 || d_head == 128;
}

// why a segment cannot be read (NULL: it can)
const char *shared_segment_fault(int dtype, const SharedSegment &s) {
    const int chunk = dtype == PSD_DTYPE_BF16 ? 8 : 4;   // elements of 16 bytes
    if (s.len == 0) return nullptr;
    if (!s.k || !s.vt) return "keys or values are NULL";
    if (!aligned16(s.k) || !aligned16(s.vt) || s.ld_k % chunk || s.stride_k % chunk || s.stride_vt % chunk)
        return "keys and values need 16-byte aligned rows";
    if (s.ld_vt % 16 || s.ld_vt < (s.len + 15) / 16 * 16) return "rows of values hold whole groups of 16 positions";
    return nullptr;
}

bool plan_attention_shared(const SharedShape &sh, const SharedSegment *seg, int n, SharedLaunch *out) {
    for (int i = 0; i < n; ++i)   // (counts that the plans keep in 32 bits)
        if ((double)sh.n_rows * seg[i].len > 1e15) return false;
    *out = plan_attention(sh, seg, n);
    return launchable(out->blocks, NW * 64) && ((out->blocks > 0 && out->parts == 0) || launchable(join_workgroups(sh, *out), 256));
}
int64_t shared_attention_bytes(const SharedShape &sh, const SharedLaunch &ln) {
    return align_up((int64_t)ln.parts * sh.n_rows * sh.d_head * 4, 256) + align_up((int64_t)ln.parts * sh.n_rows * 8, 256);
}
// the most that any batch of 1 .. sh.S sequences over these segments needs, however they share them
int64_t shared_attention_most(const SharedShape &sh, const SharedSegment *seg, int n) {
    // No job has more parts than key tiles: those of a segment, or, of a finer segment in a walk, of every unit that a tile touches,
    // of which there are no more than sequences.
    int64_t steps = 0;
    for (int i = 0; i < n; ++i) {
        const int64_t walked = (int64_t)(i == 0 ? 1 : std::min(sh.S, MOST_TOUCHED)) * ((seg[i].len + KT - 1) / KT);
        steps += std::max<int64_t>((seg[i].len + BK - 1) / BK, walked);
    }
    const int64_t rows = std::max(n * sh.n_rows, std::min(MOST_PART_ROWS, steps * sh.n_rows));
    return align_up(rows * sh.d_head * 4, 256) + align_up(rows * 8, 256);
}
bool plan_attention_weights(const SharedShape &sh, const SharedSegment *seg, int n, SharedLaunch *out) {
    for (int i = 0; i < n; ++i)
        if ((double)sh.n_rows * seg[i].len > 1e15) return false;
    *out = plan_weights(sh, seg, n);
    return launchable(out->blocks, NW * 64) && launchable(out->join_blocks, 256);
}
int64_t shared_weights_bytes(const SharedLaunch &ln) { return ln.parts * 256ll; }

// (parts cost one more than the workgroups that plan_weights asks for, and those are at most a quarter of the tiles of rows; seqs_per_unit 1
// is the most units that a segment can have)
int64_t shared_weights_most(const SharedShape &sh, const SharedSegment *seg, int n) {
    const bool bf16 = sh.dtype == PSD_DTYPE_BF16;
    const int64_t per_block = NW * 32 * (bf16 ? NKEYS<bf16_t> : NKEYS<float>), WR = bf16 ? WROWS<bf16_t> : WROWS<float>;
    int64_t floats = 0;
    for (int i = 0; i < n; ++i) {
        if (!seg[i].weights || seg[i].len == 0) continue;
        const int64_t ug = (int64_t)(sh.S / seg[i].seqs_per_unit) * sh.n_kv_heads;
        const int64_t tiles = ug * ((seg[i].len + per_block - 1) / per_block) * ((rows_per_unit(sh, seg[i]) + WR - 1) / WR);
        floats += per_block * std::min<int64_t>(tiles / 4 + 1, 800) + ug * seg[i].len + 64;
    }
    return floats * 4;
}

#define PSD_SHARED_DISPATCH(CALL)                                             \
    if (sh.dtype == PSD_DTYPE_BF16) {                                         \
        using T = bf16_t;                                                     \
        if (sh.d_head == 128) { constexpr int DH = 128; CALL; }               \
        else { constexpr int DH = 64; CALL; }                                 \
    } else {                                                                  \
        using T = float;                                                      \
        if (sh.d_head == 128) { constexpr int DH = 128; CALL; }               \
        else if (sh.d_head == 64) { constexpr int DH = 64; CALL; }            \
        else if (sh.d_head == 32) { constexpr int DH = 32; CALL; }            \
        else { constexpr int DH = 16; CALL; }                                 \
    }

void launch_attention_shared(const void *q, const SharedShape &sh, SharedLaunch &ln, void *out, float *lse, void *ws, hipStream_t st) {
    ln.o = (float *)ws;
    ln.ml = (float2 *)((char *)ws + align_up((int64_t)ln.parts * sh.n_rows * sh.d_head * 4, 256));
    ln.out = out;
    ln.lse = lse;
    PSD_SHARED_DISPATCH((run_attention<T, DH>((const T *)q, sh, ln, st)))
}

void launch_block_values(const float *qkv, int ld_qkv, int v_col, int S, int L, int width, float *vT, int ld_vt, hipStream_t st) {
    hipLaunchKernelGGL(block_values_kernel, dim3((unsigned)(S * L)), dim3(256), 0, st, qkv, ld_qkv, v_col, L, width, vT, ld_vt);
}

void launch_attention_weights(const void *q, const SharedShape &sh, SharedLaunch &ln, const float *lse, int accumulate, void *ws, hipStream_t st) {
    ln.o = (float *)ws;
    PSD_SHARED_DISPATCH((run_weights<T, DH>((const T *)q, lse, sh, ln, accumulate, st)))
}
