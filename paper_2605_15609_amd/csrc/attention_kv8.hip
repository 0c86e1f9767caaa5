// Attention over a cache of 8-bit codes (psd_attention_kv8) and, behind it, over the rows of the sequences' own blocks.
//
// For a row q and the positions j of its unit, with codes c, C and scales s, t of their blocks,
//     x_j = <q, c_j> s_j / sqrt(d),   p_j = exp(x_j - m),   o = sum p_j t_j C_j / sum p_j,   lse = m + ln sum p_j.
// A code is exact in bf16, so the products take codes as they are: a key's scale multiplies its score (one factor for 16 positions, in the
// multiply-add that the exponential needs anyway), a value's scale the probability before that is rounded to bf16.
//
// Per tile the problem is transposed as in the other attention kernels: S^T = K Q^T, O^T += V^T P^T.  A lane owns one row; the cache holds
// codes in the order of the products' fragments (kv8_device.h), so a lane's 16 bytes are two fragments once they are converted.
#include <algorithm>

#include "psd_internal.h"
#include "kv8_device.h"
#include "attention_parts.h"

namespace {

constexpr int TR = 32;    // rows of a tile where there are few
constexpr int MT = 128;   // rows of a tile where there are many
constexpr int KT = 64;    // keys of a stage in LDS
constexpr int NW = 4;     // wavefronts of a workgroup
constexpr float SLACK = 8.f;      // the reference of a row's exponentials is raised where its maximum has grown by more (in units of log 2)
constexpr float FAR = 0x1p24f;    // references beyond it (see Softmax)

// 16 codes: the first 8 into a, the last 8 into b
template <int FORMAT>
__device__ __forceinline__ void convert(const uint4 c, Frag<bf16_t> &a, Frag<bf16_t> &b) {
    const uint32_t w[4] = {c.x, c.y, c.z, c.w};
    uint32_t r[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (FORMAT == PSD_KV8_INT8) {
            r[2 * i] = pack_bf16x2((float)(int8_t)w[i], (float)(int8_t)(w[i] >> 8));
            r[2 * i + 1] = pack_bf16x2((float)(int8_t)(w[i] >> 16), (float)((int32_t)w[i] >> 24));
        } else {
            r[2 * i] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[i], 1.0f, false));
            r[2 * i + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[i], 1.0f, true));
        }
    }
    a.v = make_uint4(r[0], r[1], r[2], r[3]);
    b.v = make_uint4(r[4], r[5], r[6], r[7]);
}
template <int FORMAT>
__device__ __forceinline__ void convert(const uint4 c, Frag<float> &a, Frag<float> &b) {
    const uint32_t w[4] = {c.x, c.y, c.z, c.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float *to = i < 2 ? a.v + 4 * i : b.v + 4 * (i - 2);
        if constexpr (FORMAT == PSD_KV8_INT8) {
            to[0] = (float)(int8_t)w[i], to[1] = (float)(int8_t)(w[i] >> 8), to[2] = (float)(int8_t)(w[i] >> 16), to[3] = (float)((int32_t)w[i] >> 24);
        } else {
            to[0] = __builtin_amdgcn_cvt_f32_fp8((int)w[i], 0), to[1] = __builtin_amdgcn_cvt_f32_fp8((int)w[i], 1);
            to[2] = __builtin_amdgcn_cvt_f32_fp8((int)w[i], 2), to[3] = __builtin_amdgcn_cvt_f32_fp8((int)w[i], 3);
        }
    }
}
// keeps the value codes of positions before `left` (of a half whose first position that is counted from): 0 x NaN is NaN
__device__ __forceinline__ uint4 keep(uint4 c, int left) {
    uint32_t *w = &c.x;
#pragma unroll
    for (int b = 0; b < 4; ++b) {
        const int n = left - 8 * b;
        w[b] &= n >= 4 ? ~0u : n <= 0 ? 0u : (1u << (8 * n)) - 1;
    }
    return c;
}

// 16 positions of a head's scales: key scale times 1 / sqrt(d) in units of log 2, value scale
struct Scale {
    float k, v;
};

// The softmax of a lane's row, kept relative to a running reference that is raised only where the maximum has grown by more than 2^SLACK in a
// probability: bf16 and fp32 are as exact there, and the outputs are not touched in most tiles.  A row that has not grown keeps its reference
// when others of the wavefront raise theirs, so its bits do not depend on what other sequences hold.
// All in units of log 2.  The reference is rounded: off by up to half a unit up to FAR, which is a factor of all of the row's terms, but
// beyond by more than they span; there scores are scaled before the reference is taken away.
struct Softmax {
    float m = -INFINITY, neg = 0.f, l = 0.f;   // reference (-inf: no score yet), what is added to scores, sum
    bool far = false;                          // a row of the wavefront has a reference beyond FAR

    // Scores of NT groups of 32 positions (x[t][v] <-> position 32 t + 8 (v / 4) + 4 half + v % 4) into probabilities times value scales, 8 at a time as
    // the second product takes them.
    template <typename T, int NT, int CT>
    __device__ __forceinline__ void step(floatx16 (&x)[NT], const Scale (&s)[2 * NT], floatx16 (&acc)[CT], Frag<T> (&p)[2 * NT]) {
        float mx = -INFINITY;
#pragma unroll
        for (int g = 0; g < 2 * NT; ++g) {
            const floatx16 &y = x[g >> 1];
            float top = y[8 * (g & 1)];
#pragma unroll
            for (int v = 1; v < 8; ++v) top = fmaxf(top, y[8 * (g & 1) + v]);
            mx = fmaxf(mx, top * s[g].k);
        }
        mx = both_max(mx);
        const float over = mx - m;   // (NaN where there is no score yet, which raises nothing)
        if (__any(over > SLACK)) {
            const bool raised = over > SLACK;
            const float alpha = raised ? __builtin_amdgcn_exp2f(-over) : 1.f;
            l *= alpha;
            m = raised ? mx : m;
            neg = raised ? -mx : neg;
            far = __any(fabsf(neg) > FAR);
#pragma unroll
            for (int ct = 0; ct < CT; ++ct)
#pragma unroll
                for (int v = 0; v < 16; ++v) acc[ct][v] *= alpha;
        }
        float sum[2] = {0.f, 0.f};
#pragma unroll
        for (int g = 0; g < 2 * NT; ++g) {
            float by = s[g].k;
            if (far) {
#pragma unroll
                for (int v = 0; v < 8; ++v) {
                    float scaled = x[g >> 1][8 * (g & 1) + v] * by;
                    asm volatile("" : "+v"(scaled));   // (rounded: contracted into what follows it would not be)
                    x[g >> 1][8 * (g & 1) + v] = scaled;
                }
                by = 1.f;
            }
            float e[8];
#pragma unroll
            for (int v = 0; v < 8; ++v) {
                e[v] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[g >> 1][8 * (g & 1) + v], by, neg));
                sum[v & 1] += e[v];
                e[v] *= s[g].v;
            }
            probabilities(e, p[g]);
        }
        l += sum[0] + sum[1];
    }
};

// the last tile of a unit: positions from `left` on are hidden, whatever codes and scales they have
template <int NT>
__device__ __forceinline__ void hide(floatx16 (&x)[NT], Scale (&s)[2 * NT], int left, int half) {
#pragma unroll
    for (int g = 0; g < 2 * NT; ++g) {
        if (g * 16 >= left) s[g] = {1.f, 0.f};
        const bool zero = s[g].k == 0.f;   // (0 x -inf is NaN)
        if (zero) s[g].k = 1.f;
#pragma unroll
        for (int v = 0; v < 8; ++v) {
            const float y = zero ? 0.f : x[g >> 1][8 * (g & 1) + v];
            x[g >> 1][8 * (g & 1) + v] = 16 * g + 8 * (v >> 2) + 4 * half + (v & 3) >= left ? -INFINITY : y;
        }
    }
}

// Codes and scales of one unit and KV head
struct Head {
    const uint8_t *codes;
    const float2 *scales;
    int keys, shift;
    __device__ Head(const Kv8 &c, int u, int kvh) {
        codes = c.codes + u * c.stride_codes + (int64_t)kvh * (c.capacity / KV8_TILE) * (64 * c.d_head);
        scales = c.scales + u * c.stride_scales + (int64_t)kvh * (c.capacity >> c.block_shift);
        keys = __builtin_amdgcn_readfirstlane(kv8_keys(c, u));
        shift = c.block_shift;
    }
    // of the g-th 16 positions from tile t on (those behind the cache's last key: of that one)
    __device__ __forceinline__ float2 scale(int t, int g) const { return scales[min(t * KV8_TILE + 16 * g, keys - 1) >> shift]; }
};

// channels that the first product's step ks takes from a lane's half
template <int DH>
__device__ __forceinline__ int channel_of(int ks, int half) {
    return DH < 32 ? half * 8 : (ks >> 1) * 32 + half * 16 + (ks & 1) * 8;
}

// 32 rows at most of a sequence's own block, from row k0 of sequence s on: keys and values as the projection leaves them.  mixed: the wavefront
// has rows of other sequences, which see nothing of it.
template <typename T, int DH, int CT>
__device__ __forceinline__ void own_step(const SharedShape &sh, const Kv8Launch &ln, int kvh, int64_t s, int k0, bool mixed, bool sees, float sl2, const Frag<T> (&qf)[DH / 16],
                                         Softmax &soft, floatx16 (&acc)[CT]) {
    const int lane = threadIdx.x & 63, lrow = lane & 31, half = lane >> 5, left = min(sh.L - k0, 32);
    const T *k = (const T *)ln.k + (s * sh.L + k0 + min(lrow, left - 1)) * ln.ld_k + kvh * DH;
    const T *v = (const T *)ln.v + (s * sh.L + k0) * ln.ld_v + kvh * DH;
    floatx16 x[1];
#pragma unroll
    for (int i = 0; i < 16; ++i) x[0][i] = 0.f;
#pragma unroll
    for (int ks = 0; ks < DH / 16; ++ks) {
        Frag<T> kf;
        kf.load(k + channel_of<DH>(ks, half));
        product(kf, qf[ks], x[0]);
    }
    // a lane's channel of 8 positions, one by one: they lie in rows of their own
    Frag<T> vf[2][CT];
#pragma unroll
    for (int kg = 0; kg < 2; ++kg)
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
            const T *at = v + (CT * 32 > DH ? min(lrow, DH - 1) : ct * 32 + lrow);
            T e[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int j = kg * 16 + 8 * (i >> 2) + 4 * half + (i & 3);
                e[i] = at[(int64_t)min(j, left - 1) * ln.ld_v];
                if (j >= left) e[i] = from_float<T>(0.f);
            }
            if constexpr (sizeof(T) == 2) {
                vf[kg][ct].v = make_uint4(e[0].bits | (uint32_t)e[1].bits << 16, e[2].bits | (uint32_t)e[3].bits << 16, e[4].bits | (uint32_t)e[5].bits << 16,
                                          e[6].bits | (uint32_t)e[7].bits << 16);
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) vf[kg][ct].v[i] = e[i];
            }
        }
#pragma unroll
    for (int i = 0; i < 16; ++i)
        if (8 * (i >> 2) + 4 * half + (i & 3) >= left || !sees) x[0][i] = -INFINITY;
    const Scale scale[2] = {{sl2, 1.f}, {sl2, 1.f}};
    Frag<T> p[2];
    soft.step(x, scale, acc, p);
#pragma unroll
    for (int kg = 0; kg < 2; ++kg)
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
            if (!mixed) {
                product(vf[kg][ct], p[kg], acc[ct]);
            } else {   // (rows that do not see the block: their probabilities are 0, but its values may be anything)
                floatx16 sum = acc[ct];
                product(vf[kg][ct], p[kg], sum);
#pragma unroll
                for (int i = 0; i < 16; ++i) acc[ct][i] = sees ? sum[i] : acc[ct][i];
            }
        }
}

// A tile of up to 32 rows of a unit and KV head (r_first ..) against the own blocks of their sequences, every W-th step from `first` on
template <typename T, int DH, int CT>
__device__ __forceinline__ void own_blocks(const SharedShape &sh, const Kv8Launch &ln, int u, int kvh, int r_first, int rows, int64_t token, int first, int W, float sl2,
                                           const Frag<T> (&qf)[DH / 16], Softmax &soft, floatx16 (&acc)[CT]) {
    const int per_seq = sh.L * (sh.n_heads / sh.n_kv_heads), n = (sh.L + 31) / 32;
    const int a = r_first / per_seq, b = (min(r_first + 32, rows) - 1) / per_seq;
    const int mine = (int)(token / sh.L);
    for (int i = first; i < (b - a + 1) * n; i += W) {
        const int s = u * ln.cache.seqs_per_unit + a + i / n;
        own_step<T, DH, CT>(sh, ln, kvh, s, i % n * 32, a != b, mine == s, sl2, qf, soft, acc);
    }
}

// Few rows: a tile of TR rows against a part of its unit's keys, and the last part against their own blocks too.  The wavefronts deal the keys, 32 at
// a time, codes straight from memory a step ahead, and merge in LDS in wavefront order.
template <typename T, int DH, int FORMAT>
__device__ __forceinline__ void few_rows(const T *__restrict__ q, const SharedShape &sh, const Kv8Launch &ln, int u, int kvh, int tile, int split, float sl2,
                                         float *part /* [wavefront][max, sum, NF values][64 lanes] */) {
    constexpr int KS = DH / 16, CT = (DH + 31) / 32, NF = CT * 16, KL = DH < 32 ? 1 : DH / 32;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lrow = lane & 31, half = lane >> 5;
    const int spu = ln.cache.seqs_per_unit, rows = spu * sh.L * (sh.n_heads / sh.n_kv_heads), r = tile * TR + lrow;
    const RowOf row(sh, (int64_t)u * spu, kvh, min(r, rows - 1));   // (rows past the last repeat it and store nothing)
    const Head head(ln.cache, u, kvh);
    const int begin = (int)min((int64_t)split * ln.chunk, (int64_t)head.keys), end = (int)min((int64_t)begin + ln.chunk, (int64_t)head.keys);
    const int t0 = begin / KV8_TILE, steps = (end - begin + KV8_TILE - 1) / KV8_TILE;
    Frag<T> qf[KS];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qf[ks].load(q + row.token * sh.ld_q + row.head * DH + channel_of<DH>(ks, half));
    floatx16 acc[CT];
#pragma unroll
    for (int ct = 0; ct < CT; ++ct)
#pragma unroll
        for (int v = 0; v < 16; ++v) acc[ct][v] = 0.f;
    Softmax soft;
    uint4 kc[KL], vc[CT];
    float2 sc[2];
    auto load = [&](int t) {
        const uint8_t *at = head.codes + (int64_t)t * (64 * DH);
        if constexpr (DH < 32) {
            kc[0] = *reinterpret_cast<const uint4 *>(at + lrow * 16);
            vc[0] = *reinterpret_cast<const uint4 *>(at + 32 * DH + half * (16 * DH) + min(lrow, DH - 1) * 16);
        } else {
#pragma unroll
            for (int l = 0; l < KL; ++l) kc[l] = *reinterpret_cast<const uint4 *>(at + l * 1024 + lane * 16);
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) vc[ct] = *reinterpret_cast<const uint4 *>(at + 32 * DH + ct * 1024 + lane * 16);
        }
#pragma unroll
        for (int g = 0; g < 2; ++g) sc[g] = head.scale(t, g);
    };
    if (wave < steps) load(t0 + wave);
    for (int st = wave; st < steps; st += NW) {
        const int left = end - begin - st * KV8_TILE;
        uint4 k[KL], v[CT];
        Scale scale[2];
#pragma unroll
        for (int l = 0; l < KL; ++l) k[l] = kc[l];
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) v[ct] = vc[ct];
#pragma unroll
        for (int g = 0; g < 2; ++g) scale[g] = {sc[g].x * sl2, sc[g].y};
        if (st + NW < steps) load(t0 + st + NW);
        floatx16 x[1];
#pragma unroll
        for (int i = 0; i < 16; ++i) x[0][i] = 0.f;
#pragma unroll
        for (int l = 0; l < KL; ++l) {
            Frag<T> a, b;
            convert<FORMAT>(k[l], a, b);
            if constexpr (DH < 32) {
                if constexpr (sizeof(T) == 4) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) a.v[e] = half ? b.v[e] : a.v[e];
                }
                product(a, qf[0], x[0]);
            } else {
                product(a, qf[2 * l], x[0]);
                product(b, qf[2 * l + 1], x[0]);
            }
        }
        if (left < KV8_TILE) {
            hide(x, scale, left, half);
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) v[ct] = keep(v[ct], left - 4 * half);
        }
        Frag<T> p[2];
        soft.step(x, scale, acc, p);
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
            Frag<T> a, b;
            convert<FORMAT>(v[ct], a, b);
            product(a, p[0], acc[ct]);
            product(b, p[1], acc[ct]);
        }
    }
    if (ln.k && split == ln.splits - 1) own_blocks<T, DH, CT>(sh, ln, u, kvh, tile * TR, rows, row.token, (wave - steps) & (NW - 1), NW, sl2, qf, soft, acc);
    const float l_run = both_sum(soft.l);   // the halves of a row hold disjoint keys

    float *mine = part + wave * (2 + NF) * 64 + lane;
    mine[0] = soft.m;
    mine[64] = l_run;
#pragma unroll
    for (int ct = 0; ct < CT; ++ct)
#pragma unroll
        for (int v = 0; v < 16; ++v) mine[(2 + ct * 16 + v) * 64] = acc[ct][v];
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
        scale[w] = __builtin_amdgcn_exp2f(scale[w] - ref);
        l_all += part[(w * (2 + NF) + 1) * 64 + lane] * scale[w];
    }
    if (r >= rows) return;
    const PartOut<T, DH> to(sh, ln, split, row);
    if (wave == 0 && half == 0) to.sums(m_all, l_all, 1.f);
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

// Many rows (bf16): a tile of 128 rows, 32 to a wavefront, walks stages of 64 keys.  Each wavefront fetches a quarter of a stage's codes a stage ahead,
// converts them once for all four and puts them into LDS as the fragments that they are: lane by lane, so neither side has a bank conflict.
template <int DH, int FORMAT>
__device__ __forceinline__ void many_rows(const bf16_t *__restrict__ q, const SharedShape &sh, const Kv8Launch &ln, int u, int kvh, int tile, int split, float sl2,
                                          unsigned char *lds) {
    constexpr int KS = DH / 16, CT = DH / 32, LOADS = 2 * CT / NW, STAGE = KT * DH * 4;   // loads of keys, and of values, a wavefront; bytes of a stage
    static_assert(2 * CT % NW == 0, "the wavefronts take equal shares of a stage");
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lrow = lane & 31, half = lane >> 5;
    const int spu = ln.cache.seqs_per_unit, rows = spu * sh.L * (sh.n_heads / sh.n_kv_heads), r_first = tile * MT + wave * 32, r = r_first + lrow;
    const RowOf row(sh, (int64_t)u * spu, kvh, min(r, rows - 1));
    const bool any_rows = r_first < rows;
    const Head head(ln.cache, u, kvh);
    const int begin = (int)min((int64_t)split * ln.chunk, (int64_t)head.keys), end = (int)min((int64_t)begin + ln.chunk, (int64_t)head.keys);
    const int t0 = begin / KV8_TILE, stages = (end - begin + KT - 1) / KT, t_last = (end - 1) / KV8_TILE;
    Frag<bf16_t> qf[KS];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qf[ks].load(q + row.token * sh.ld_q + row.head * DH + channel_of<DH>(ks, half));
    floatx16 acc[CT];
#pragma unroll
    for (int ct = 0; ct < CT; ++ct)
#pragma unroll
        for (int v = 0; v < 16; ++v) acc[ct][v] = 0.f;
    Softmax soft;
    uint4 kc[LOADS], vc[LOADS];
    float2 sc;
    auto load = [&](int st) {   // (a tile behind the part's last is that one again: its positions are hidden)
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int n = wave * LOADS + i;
            const uint8_t *at = head.codes + (int64_t)min(t0 + 2 * st + n / CT, t_last) * (64 * DH) + n % CT * 1024 + lane * 16;
            kc[i] = *reinterpret_cast<const uint4 *>(at);
            vc[i] = *reinterpret_cast<const uint4 *>(at + 32 * DH);
        }
        sc = head.scale(t0 + 2 * st, lane & 3);
    };
    if (stages > 0) load(0);
    for (int st = 0; st < stages; ++st) {
        unsigned char *at = lds + (st & 1) * STAGE + lane * 16;
        const int left = end - begin - st * KT;
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int n = wave * LOADS + i;   // keys: fragment (tile, step) at tile * KS + step, two a load; values: (tile, channels, 16 positions) behind them
            Frag<bf16_t> a, b;
            convert<FORMAT>(kc[i], a, b);
            *reinterpret_cast<uint4 *>(at + (2 * n) * 1024) = a.v;
            *reinterpret_cast<uint4 *>(at + (2 * n + 1) * 1024) = b.v;
            convert<FORMAT>(left < KT ? keep(vc[i], left - n / CT * 32 - 4 * half) : vc[i], a, b);
            *reinterpret_cast<uint4 *>(at + (2 * KS + 2 * n) * 1024) = a.v;
            *reinterpret_cast<uint4 *>(at + (2 * KS + 2 * n + 1) * 1024) = b.v;
        }
        Scale scale[4];
#pragma unroll
        for (int g = 0; g < 4; ++g)
            scale[g] = {__int_as_float(__builtin_amdgcn_readlane(__float_as_int(sc.x), g)) * sl2, __int_as_float(__builtin_amdgcn_readlane(__float_as_int(sc.y), g))};
        if (st + 1 < stages) load(st + 1);
        // The stage is whole.  (The one before it is read until this point, the next goes to where that was.)
        __syncthreads();
        if (!any_rows) continue;
        floatx16 x[2];
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
            for (int v = 0; v < 16; ++v) x[kt][v] = 0.f;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)
#pragma unroll
            for (int kt = 0; kt < 2; ++kt) {
                Frag<bf16_t> kf;
                kf.v = *reinterpret_cast<const uint4 *>(at + (kt * KS + ks) * 1024);
                product(kf, qf[ks], x[kt]);
            }
        if (left < KT) hide(x, scale, left, half);
        Frag<bf16_t> p[4];
        soft.step(x, scale, acc, p);
#pragma unroll
        for (int g = 0; g < 4; ++g)
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) {
                Frag<bf16_t> vf;
                vf.v = *reinterpret_cast<const uint4 *>(at + (2 * KS + ((g >> 1) * CT + ct) * 2 + (g & 1)) * 1024);
                product(vf, p[g], acc[ct]);
            }
    }
    if (ln.k && split == ln.splits - 1 && any_rows) own_blocks<bf16_t, DH, CT>(sh, ln, u, kvh, r_first, rows, row.token, 0, 1, sl2, qf, soft, acc);
    const float l_run = both_sum(soft.l);
    if (r >= rows) return;
    const PartOut<bf16_t, DH> to(sh, ln, split, row);
    if (half == 0) to.sums(soft.m, l_run, 1.f);
    const float f = to.factor(l_run);
    if (f == 0.f && !to.direct) return;
#pragma unroll
    for (int ct = 0; ct < CT; ++ct)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const float o[4] = {acc[ct][4 * g], acc[ct][4 * g + 1], acc[ct][4 * g + 2], acc[ct][4 * g + 3]};
            to.values(ct * 32 + 8 * g + 4 * half, o, f);
        }
}

template <typename T, int DH>
constexpr int attention_lds() {
    constexpr int merge = NW * (2 + (DH + 31) / 32 * 16) * 64 * 4, stages = sizeof(T) == 2 ? 2 * KT * DH * 4 : 0;
    return merge > stages ? merge : stages;
}

// Workgroups are dealt to the XCDs in runs of equal length, the tiles of one unit, KV head and part behind one another, so that those that read the same
// keys meet in one L2.
template <typename T, int DH, int FORMAT>
__global__ __launch_bounds__(NW * 64, 2) void attention_kv8_kernel(const T *__restrict__ q, SharedShape sh, Kv8Launch ln, float sl2) {
    extern __shared__ __align__(16) unsigned char lds[];
    const int n = ln.units * sh.n_kv_heads * ln.splits * ln.tiles, run = (n + 7) / 8;
    const int at = (blockIdx.x & 7) * run + (blockIdx.x >> 3);
    if (at >= n) return;
    const int tile = at % ln.tiles, split = at / ln.tiles % ln.splits, kvh = at / ln.tiles / ln.splits % sh.n_kv_heads, u = at / ln.tiles / ln.splits / sh.n_kv_heads;
    if constexpr (sizeof(T) == 2) {
        if (ln.tiled) {
            many_rows<DH, FORMAT>(q, sh, ln, u, kvh, tile, split, sl2, lds);
            return;
        }
    }
    few_rows<T, DH, FORMAT>(q, sh, ln, u, kvh, tile, split, sl2, reinterpret_cast<float *>(lds));
}

int64_t workgroups(const SharedShape &sh, const Kv8Launch &ln) { return (int64_t)ln.units * sh.n_kv_heads * ln.splits * ln.tiles; }

template <typename T, int DH, int FORMAT>
void run(const T *q, const SharedShape &sh, const Kv8Launch &ln, hipStream_t st) {
    constexpr int smem = attention_lds<T, DH>();
    auto kern = attention_kv8_kernel<T, DH, FORMAT>;
    static std::atomic<uint64_t> lds_raised{0};   // one per instantiation
    ensure_dynamic_lds(reinterpret_cast<const void *>(kern), smem, lds_raised);
    hipLaunchKernelGGL(kern, dim3((unsigned)align_up(workgroups(sh, ln), 8)), dim3(NW * 64), smem, st, q, sh, ln, LOG2E / sqrtf((float)DH));
}
template <typename T, int DH>
void run(const T *q, const SharedShape &sh, const Kv8Launch &ln, hipStream_t st) {
    if (ln.cache.format == PSD_KV8_INT8) run<T, DH, PSD_KV8_INT8>(q, sh, ln, st);
    else run<T, DH, PSD_KV8_E4M3>(q, sh, ln, st);
}

}   // namespace

bool plan_attention_kv8(const SharedShape &sh, const Kv8 &cache, bool own_rows, Kv8Launch *out) {
    Kv8Launch ln;
    ln.cache = cache;
    ln.units = sh.S / cache.seqs_per_unit;
    const int64_t rows = (int64_t)cache.seqs_per_unit * sh.L * (sh.n_heads / sh.n_kv_heads);
    ln.tiled = sh.dtype == PSD_DTYPE_BF16 && rows >= 64;
    const int rows_of_tile = ln.tiled ? MT : TR, step = ln.tiled ? KT : KV8_TILE * NW;
    ln.tiles = (int)((rows + rows_of_tile - 1) / rows_of_tile);
    const double base = (double)ln.units * sh.n_kv_heads * ln.tiles;
    const int steps = (cache.len + step - 1) / step;
    const int want = (int)std::max(1.0, std::min(std::ceil(512.0 / base), steps / 4.0));
    const int each = std::max(1, (steps + want - 1) / want);
    ln.chunk = each * step;
    ln.splits = std::max(1, (steps + each - 1) / each);
    ln.parts = ln.splits > 1 ? ln.splits : 0;
    *out = ln;
    return base * ln.splits < 0x1p31 && launchable(align_up(workgroups(sh, ln), 8), NW * 64) && (ln.parts == 0 || attention_join_launchable(sh, ln));
}

void launch_attention_kv8(const void *q, const SharedShape &sh, const Kv8Launch &ln, hipStream_t st) {
    if (sh.dtype == PSD_DTYPE_BF16) {
        if (sh.d_head == 64) run<bf16_t, 64>((const bf16_t *)q, sh, ln, st);
        else run<bf16_t, 128>((const bf16_t *)q, sh, ln, st);
    } else {
        if (sh.d_head == 16) run<float, 16>((const float *)q, sh, ln, st);
        else if (sh.d_head == 32) run<float, 32>((const float *)q, sh, ln, st);
        else if (sh.d_head == 64) run<float, 64>((const float *)q, sh, ln, st);
        else run<float, 128>((const float *)q, sh, ln, st);
    }
    if (ln.parts > 0) launch_attention_join(sh, ln, 1.f, st);
}
