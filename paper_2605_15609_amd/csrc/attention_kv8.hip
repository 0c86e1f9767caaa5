// Attention over a cache of 8-bit codes (psd_attention_kv8) and, behind it, over the rows of the sequences' own blocks.
//
// For a row q and the positions j of its unit, with codes c, C and scales s, t of their blocks,
//     x_j = <q, c_j> s_j / sqrt(d),   p_j = exp(x_j - m),   o = sum p_j t_j C_j / sum p_j,   lse = m + ln sum p_j.
// A code is exact in bf16, so the products take codes as they are: a key's scale multiplies its score (one factor for 16 positions, in the
// multiply-add that the exponential needs anyway), a value's scale the probability before that is rounded to bf16.
//
// Per tile the problem is transposed as in the other attention kernels: S^T = K Q^T, O^T += V^T P^T.  A lane owns one row; the cache holds
// codes in the order of the products' fragments (kv8_device.h), so a lane's 16 bytes are two fragments once they are converted.
//
// What bounds it, with bf16 heads of 128: single rows memory (32 requests of the 7B shape over 16384 positions each take 94 us, 5.7 TB/s of codes; of
// lengths even over 1 .. 16384 60 - 73 us, where a part's last workgroups run alone); blocks of 16 requests over 1312 positions (8B shape) 40 us, of
// which 32 are memory.  Drafts are bound by vector instructions: a tile of 32 keys and 32 rows has 16 products and, in int8, 192 instructions that convert
// its codes (e4m3: 64) and some 150 of softmax.  128 drafts of 64 rows over 5120 + 64 keys (8B shape) take 783 - 845 us, 0.82 - 0.89 PFLOP/s: vector units busy 70 %
// of the cycles, matrix cores 44 %, at a clock that power holds near 1.8 GHz.  Small calls are one chain of round trips: 6.5 us, 7.5 with the host's call.
// Tried and slower: queries in LDS for three workgroups a CU, with one tile of codes under way a wavefront in place of two (32 requests, ragged: 58 -> 66);
// 16x16 products for up to 16 rows, a third workgroup a CU (level with these, 64 us); value scales in the exponent and no maximum in front of the exponentials
// (many rows: 776 -> 760, but 92 -> 101 at 32 drafts over 2000 keys: two ways through a stage, of which the careful one spills).
#include <math.h>

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

// 8 codes, and 16: the first 8 into a, the last 8 into b
template <int FORMAT>
__device__ __forceinline__ uint4 convert(uint32_t c0, uint32_t c1) {
    const uint32_t w[2] = {c0, c1};
    uint32_t r[4];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        if constexpr (FORMAT == PSD_KV8_INT8) {
            r[2 * i] = pack_bf16x2((float)(int8_t)w[i], (float)(int8_t)(w[i] >> 8));
            r[2 * i + 1] = pack_bf16x2((float)(int8_t)(w[i] >> 16), (float)((int32_t)w[i] >> 24));
        } else {
            r[2 * i] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[i], 1.0f, false));
            r[2 * i + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[i], 1.0f, true));
        }
    }
    return make_uint4(r[0], r[1], r[2], r[3]);
}
template <int FORMAT>
__device__ __forceinline__ void convert(const uint4 c, Frag<bf16_t> &a, Frag<bf16_t> &b) {
    a.v = convert<FORMAT>(c.x, c.y);
    b.v = convert<FORMAT>(c.z, c.w);
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

// 16 positions of a head's scales, the same in all lanes: key scale times 1 / sqrt(d) in units of log 2, value scale
struct Scale {
    float k, v;
    float inv;   // what products are multiplied by that tell what probabilities were rounded to (see weigh)
    bool told;
    __device__ Scale() {}
    __device__ Scale(float key, float value, float reciprocal) : k(key), v(value), inv(reciprocal), told(tells(value)) {}
    // the reciprocal of a value scale holds what it has to: 2^-126 .. 2^126
    static __device__ __forceinline__ bool tells(float value) { return __float_as_uint(value) - 0x00800000u < 0x7e000000u; }
    static __device__ __forceinline__ float reciprocal(float value) { return tells(value) ? __builtin_amdgcn_rcpf(value) : 1.f; }
};

// The softmax of a lane's row, kept relative to a running reference that is raised only where the maximum has grown by more than 2^SLACK in a
// probability: bf16 and fp32 are as exact there, and the outputs are not touched in most tiles.  A row that has not grown keeps its reference
// when others of the wavefront raise theirs, so its bits do not depend on what other sequences hold.
// All in units of log 2.  The reference is rounded: off by up to half a unit up to FAR, which is a factor of all of the row's terms, but
// beyond by more than they span; there scores are scaled before the reference is taken away.
struct Softmax {
    float m = -INFINITY, neg = 0.f, l = 0.f;   // reference (-inf: no score yet), what is added to scores, sum
    float given = 0.f;                         // the sum as the second product has it (see correction)
    bool far = false;                          // a row of the wavefront has a reference beyond FAR

    // x: scores of NT groups of 32 positions (x[t][v] <-> position 32 t + 8 (v / 4) + 4 half + v % 4), as sums over the codes.  Raises the reference.
    template <int NT, int CT>
    __device__ __forceinline__ void reference(floatx16 (&x)[NT], const Scale (&s)[2 * NT], floatx16 (&acc)[CT]) {
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
            given *= alpha;
            m = raised ? mx : m;
            neg = raised ? -mx : neg;
            far = __any(fabsf(neg) > FAR);
#pragma unroll
            for (int ct = 0; ct < CT; ++ct)
#pragma unroll
                for (int v = 0; v < 16; ++v) acc[ct][v] *= alpha;
        }
    }
    // (the last words of reference(): of a row that is far, scores scaled and rounded, scales of 1)
    template <int NT>
    __device__ __forceinline__ void scale_far(floatx16 (&x)[NT], Scale (&s)[2 * NT]) const {
        if (!far) return;
        const bool row = fabsf(neg) > FAR;
#pragma unroll
        for (int g = 0; g < 2 * NT; ++g) {
#pragma unroll
            for (int v = 0; v < 8; ++v) {
                float scaled = x[g >> 1][8 * (g & 1) + v] * s[g].k;
                asm volatile("" : "+v"(scaled));   // (rounded: contracted into what follows it would not be)
                x[g >> 1][8 * (g & 1) + v] = row ? scaled : x[g >> 1][8 * (g & 1) + v];
            }
            s[g].k = row ? 1.f : s[g].k;
        }
    }
    // 8 probabilities, whose sum is l8, times value scales as the second product takes them.  The products over their scale say what the probabilities were
    // rounded to; where a scale does not (a block of zeros has 0) these count as they are, so that what the products of others say stays.
    template <typename T>
    __device__ __forceinline__ void weigh(float (&e)[8], float l8, const Scale &s, Frag<T> &p) {
#pragma unroll
        for (int v = 0; v < 8; ++v) e[v] *= s.v;
        probabilities(e, p);
        if constexpr (sizeof(T) == 2) {
            typedef __bf16 pair __attribute__((ext_vector_type(2)));
            const pair ones = __builtin_bit_cast(pair, 0x3f803f80u);
            float sum = 0.f;
#pragma unroll
            for (int i = 0; i < 4; ++i) sum = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(pair, (&p.v.x)[i]), ones, sum, false);
            given = __builtin_fmaf(s.told ? sum : l8, s.inv, given);
        }
    }
    template <typename T, int NT>
    __device__ __forceinline__ void weights(const floatx16 (&x)[NT], const Scale (&s)[2 * NT], Frag<T> (&p)[2 * NT]) {
#pragma unroll
        for (int g = 0; g < 2 * NT; ++g) {
            float e[8], sum[2] = {0.f, 0.f};
#pragma unroll
            for (int v = 0; v < 8; ++v) {
                e[v] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[g >> 1][8 * (g & 1) + v], s[g].k, neg));
                sum[v & 1] = v < 2 ? e[v] : sum[v & 1] + e[v];
            }
            l += sum[0] + sum[1];
            weigh(e, sum[0] + sum[1], s[g], p[g]);
        }
    }
    // What the outputs of a row are multiplied by.  A probability times its value scale is rounded to bf16, and where one key has nearly all of a row that
    // is a factor of the whole row, half a step like the result's own rounding.  The sum of the rounded products over their scales has the same factor, so
    // it goes away, for 4 % of the time where vector instructions bound it (128 drafts 799 -> 829 us, drafts of 4 requests 47 -> 48.8) and 1 % where memory
    // does.  It is within half a step; anything else comes from rows without a number or products below the normal numbers, and corrects nothing.
    // (Blocks of scale 0 looked for in front of the exponentials instead, in a branch that is hardly ever taken: 128 drafts 830 -> 840 us.)
    template <typename T>
    __device__ __forceinline__ float correction() const {
        if constexpr (sizeof(T) == 4) return 1.f;
        const float f = both_sum(l) / both_sum(given);
        return fabsf(f - 1.f) < 0x1.02p-8f ? f : 1.f;
    }
    template <typename T, int NT, int CT>
    __device__ __forceinline__ void step(floatx16 (&x)[NT], Scale (&s)[2 * NT], floatx16 (&acc)[CT], Frag<T> (&p)[2 * NT]) {
        reference(x, s, acc);
        scale_far(x, s);
        weights(x, s, p);
    }
};

// the last tile of a unit: positions from `left` on are hidden, whatever codes and scales they have
template <int NT>
__device__ __forceinline__ void hide(floatx16 (&x)[NT], Scale (&s)[2 * NT], int left, int half) {
#pragma unroll
    for (int g = 0; g < 2 * NT; ++g) {
        if (g * 16 >= left) s[g] = Scale(1.f, 1.f, 1.f);
        const bool zero = s[g].k == 0.f;   // (0 x -inf is NaN: the scores are scaled here)
        if (zero) s[g].k = 1.f;
#pragma unroll
        for (int v = 0; v < 8; ++v) {
            const float y = zero ? 0.f * x[g >> 1][8 * (g & 1) + v] : x[g >> 1][8 * (g & 1) + v];
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

// Value rows of a sequence's own block lie position by position, and the second product wants 4 positions of a channel together.  bf16: 32 rows pass
// through LDS, 64 bytes apart more than they are long (the four positions of a read meet all banks), and come back transposed; fp32: element by element.
template <typename T, int DH>
constexpr int own_lds() {
    return sizeof(T) == 2 ? 32 * (DH * 2 + 64) : 0;
}
template <int DH>
struct OwnValues {
    static constexpr int ROW = DH * 2 + 64, LPR = DH / 8, RPI = 64 / LPR, N = 32 / RPI;   // bytes of a row, lanes to a row, rows a load
    uint4 v[N];
    __device__ __forceinline__ void load(const bf16_t *at, int64_t ld, int left) {
        const int lane = threadIdx.x & 63;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int j = i * RPI + lane / LPR;
            v[i] = *reinterpret_cast<const uint4 *>(at + min(j, left - 1) * ld + lane % LPR * 8);
            if (j >= left) v[i] = make_uint4(0, 0, 0, 0);   // (their probabilities are 0, but 0 x NaN is NaN)
        }
    }
    __device__ __forceinline__ void put(unsigned char *lds) const {
        const int lane = threadIdx.x & 63;
#pragma unroll
        for (int i = 0; i < N; ++i) *reinterpret_cast<uint4 *>(lds + (i * RPI + lane / LPR) * ROW + lane % LPR * 16) = v[i];
    }
    // positions 16 kg + 8 b + 4 half + (0 .. 3), channel 32 ct + lane % 32: every 16 lanes read 4 rows of 16 channels
    static __device__ __forceinline__ void read(const unsigned char *lds, int kg, int ct, Frag<bf16_t> &f) {
        typedef short short4_t __attribute__((ext_vector_type(4)));
        typedef __attribute__((address_space(3))) short4_t lds_short4;
        const int lane = threadIdx.x & 63, row = 16 * kg + 4 * (lane >> 5) + (lane >> 2 & 3), c = 32 * ct + (lane & 16) + 4 * (lane & 3);
        const unsigned char *at = lds + row * ROW + c * 2;
        const uint2 a = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_short4 *)at));
        const uint2 b = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_short4 *)(at + 8 * ROW)));
        f.v = make_uint4(a.x, a.y, b.x, b.y);
    }
};

// 32 rows at most of a sequence's own block, from row k0 of sequence s on: keys and values as the projection leaves them.  mixed: the wavefront
// has rows of other sequences, which see nothing of it.  lds: own_lds bytes of the wavefront's.
template <typename T, int DH, int CT, typename Q>
__device__ __forceinline__ void own_step(const SharedShape &sh, const Kv8Launch &ln, int kvh, int64_t s, int k0, bool mixed, bool sees, float sl2, const Q &query,
                                         Softmax &soft, floatx16 (&acc)[CT], unsigned char *lds) {
    const int lane = threadIdx.x & 63, lrow = lane & 31, half = lane >> 5, left = min(sh.L - k0, 32);
    const T *k = (const T *)ln.k + (s * sh.L + k0 + min(lrow, left - 1)) * ln.ld_k + kvh * DH;
    const T *v = (const T *)ln.v + (s * sh.L + k0) * ln.ld_v + kvh * DH;
    if constexpr (sizeof(T) == 2) {
        OwnValues<DH> rows;
        rows.load(v, ln.ld_v, left);
        rows.put(lds);
    }
    floatx16 x[1];
#pragma unroll
    for (int i = 0; i < 16; ++i) x[0][i] = 0.f;
#pragma unroll
    for (int ks = 0; ks < DH / 16; ++ks) {
        Frag<T> kf;
        kf.load(k + channel_of<DH>(ks, half));
        product(kf, query(ks), x[0]);
    }
#pragma unroll
    for (int i = 0; i < 16; ++i)
        if (8 * (i >> 2) + 4 * half + (i & 3) >= left || !sees) x[0][i] = -INFINITY;
    Scale scale[2] = {{sl2, 1.f, 1.f}, {sl2, 1.f, 1.f}};
    Frag<T> p[2];
    soft.step(x, scale, acc, p);
    asm volatile("" ::: "memory");
#pragma unroll
    for (int kg = 0; kg < 2; ++kg)
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
            Frag<T> vf;
            if constexpr (sizeof(T) == 2) {
                OwnValues<DH>::read(lds, kg, ct, vf);
            } else {
                const T *at = v + (CT * 32 > DH ? min(lrow, DH - 1) : ct * 32 + lrow);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int j = kg * 16 + 8 * (i >> 2) + 4 * half + (i & 3);
                    vf.v[i] = at[(int64_t)min(j, left - 1) * ln.ld_v];
                    if (j >= left) vf.v[i] = 0.f;
                }
            }
            if (!mixed) {
                product(vf, p[kg], acc[ct]);
            } else {   // (rows that do not see the block: their probabilities are 0, but its values may be anything)
                floatx16 sum = acc[ct];
                product(vf, p[kg], sum);
#pragma unroll
                for (int i = 0; i < 16; ++i) acc[ct][i] = sees ? sum[i] : acc[ct][i];
            }
        }
    asm volatile("" ::: "memory");
}

// A tile of up to 32 rows of a unit and KV head (r_first ..) against the own blocks of their sequences, every W-th step from `first` on.  A step is of one
// sequence, so many drafts of one row take 3 - 6 us of their call (8 requests of 8 drafts over 2000 positions, 8B shape: 30 us, 24 without own rows).
template <typename T, int DH, int CT, typename Q>
__device__ __forceinline__ void own_blocks(const SharedShape &sh, const Kv8Launch &ln, int u, int kvh, int r_first, int rows, int64_t token, int first, int W, float sl2,
                                           const Q &query, Softmax &soft, floatx16 (&acc)[CT], unsigned char *lds) {
    const int per_seq = sh.L * (sh.n_heads / sh.n_kv_heads), n = (sh.L + 31) / 32;
    const int a = r_first / per_seq, b = (min(r_first + 32, rows) - 1) / per_seq;
    const int mine = (int)(token / sh.L);
    for (int i = first; i < (b - a + 1) * n; i += W) {
        const int s = u * ln.cache.seqs_per_unit + a + i / n;
        own_step<T, DH, CT>(sh, ln, kvh, s, i % n * 32, a != b, mine == s, sl2, query, soft, acc, lds);
    }
}

// Few rows: a tile of TR rows against a part of its unit's keys, and the last part against their own blocks too.  The wavefronts deal the keys, 32 at
// a time, codes straight from memory a step ahead (into two sets of registers in turn: copying one to the other took 36 of 210 instructions), and merge in
// LDS in wavefront order.  No barrier in the loop, so a batch of tiles that fills the CUs little more than once is faster so than in tiles of MT
// rows, although every wavefront converts its codes alone: 6 drafts of 4 requests over 2596 keys (7B shape) 46 - 50 us against 57, 8 drafts over 2000 (8B) 36
// against 42; 32 drafts over 2000 it is 92 in tiles of MT rows against 130.
template <typename T, int DH>
constexpr int few_rows_lds() {
    constexpr int merge = NW * (2 + (DH + 31) / 32 * 16) * 64 * 4, own = NW * own_lds<T, DH>();
    return merge > own ? merge : own;
}
template <typename T, int DH, int FORMAT>
__device__ __forceinline__ void few_rows(const T *__restrict__ q, const SharedShape &sh, const Kv8Launch &ln, int u, int kvh, int tile, int split, float sl2,
                                         unsigned char *lds /* own values of every wavefront, then [wavefront][max, sum, NF values][64 lanes] */) {
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
    struct Codes {
        uint4 k[KL], v[CT];
        float2 scale[2];
    } here, ahead;
    auto load = [&](Codes &c, int t) {
        const uint8_t *at = head.codes + (int64_t)t * (64 * DH);
        if constexpr (DH < 32) {
            c.k[0] = *reinterpret_cast<const uint4 *>(at + lrow * 16);
            c.v[0] = *reinterpret_cast<const uint4 *>(at + 32 * DH + half * (16 * DH) + min(lrow, DH - 1) * 16);
        } else {
#pragma unroll
            for (int l = 0; l < KL; ++l) c.k[l] = *reinterpret_cast<const uint4 *>(at + l * 1024 + lane * 16);
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) c.v[ct] = *reinterpret_cast<const uint4 *>(at + 32 * DH + ct * 1024 + lane * 16);
        }
#pragma unroll
        for (int g = 0; g < 2; ++g) c.scale[g] = head.scale(t, g);
    };
    auto step = [&](Codes &c, Codes &next, int st) {
        const int left = end - begin - st * KV8_TILE;
        Scale scale[2];
#pragma unroll
        for (int g = 0; g < 2; ++g) scale[g] = Scale(c.scale[g].x * sl2, c.scale[g].y, Scale::reciprocal(c.scale[g].y));
        if (st + NW < steps) load(next, t0 + st + NW);
        floatx16 x[1];
#pragma unroll
        for (int i = 0; i < 16; ++i) x[0][i] = 0.f;
#pragma unroll
        for (int l = 0; l < KL; ++l) {
            Frag<T> a, b;
            convert<FORMAT>(c.k[l], a, b);
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
            for (int ct = 0; ct < CT; ++ct) c.v[ct] = keep(c.v[ct], left - 4 * half);
        }
        Frag<T> p[2];
        soft.step(x, scale, acc, p);
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
            Frag<T> a, b;
            convert<FORMAT>(c.v[ct], a, b);
            product(a, p[0], acc[ct]);
            product(b, p[1], acc[ct]);
        }
    };
    if (wave < steps) load(here, t0 + wave);
    for (int st = wave; st < steps; st += 2 * NW) {
        step(here, ahead, st);
        if (st + NW < steps) step(ahead, here, st + NW);
    }
    if (ln.k && split == ln.splits - 1)
        own_blocks<T, DH, CT>(sh, ln, u, kvh, tile * TR, rows, row.token, (wave - steps) & (NW - 1), NW, sl2, [&](int ks) { return qf[ks]; }, soft, acc,
                              lds + wave * own_lds<T, DH>());
    const float l_run = both_sum(soft.l), fix = soft.correction<T>();   // the halves of a row hold disjoint keys

    __syncthreads();
    float *part = reinterpret_cast<float *>(lds);
    float *mine = part + wave * (2 + NF) * 64 + lane;
    mine[0] = soft.m;
    mine[64] = l_run;
#pragma unroll
    for (int ct = 0; ct < CT; ++ct)
#pragma unroll
        for (int v = 0; v < 16; ++v) mine[(2 + ct * 16 + v) * 64] = acc[ct][v] * fix;
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

// Many rows (bf16): a tile of 128 rows, 32 to a wavefront, walks stages of 64 keys.  Each wavefront fetches a quarter of a stage's codes, converts it once
// for all four and puts it into LDS as the fragments that it is: lane by lane, so neither side has a bank conflict.
// Vector instructions (exponentials, conversions) take longer than the matrix instructions beside them, so the two are kept apart by a stage: the scores of
// the next stage are computed beside the exponentials of this one, and its codes converted beside this one's second product.
template <int DH, int FORMAT>
__device__ __forceinline__ void many_rows(const bf16_t *__restrict__ q, const SharedShape &sh, const Kv8Launch &ln, int u, int kvh, int tile, int split, float sl2,
                                          unsigned char *lds) {
    constexpr int KS = DH / 16, CT = DH / 32, LOADS = 2 * CT / NW, HALF = KT * DH * 2;   // loads of keys, and of values, a wavefront; bytes of a stage's keys
    static_assert(2 * CT % NW == 0, "the wavefronts take equal shares of a stage");
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lrow = lane & 31, half = lane >> 5;
    const int spu = ln.cache.seqs_per_unit, rows = spu * sh.L * (sh.n_heads / sh.n_kv_heads), r_first = tile * MT + wave * 32, r = r_first + lrow;
    const RowOf row(sh, (int64_t)u * spu, kvh, min(r, rows - 1));   // (rows past the last repeat it and store nothing)
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
    unsigned char *mine = lds + lane * 16;
    // (a tile behind the part's last is that one again: its positions are hidden, and stages behind the last are never used)
    auto load = [&](uint4 (&to)[LOADS], int st, int which) {
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int n = wave * LOADS + i;
            to[i] = *reinterpret_cast<const uint4 *>(head.codes + (int64_t)min(t0 + 2 * st + n / CT, t_last) * (64 * DH) + which * (32 * DH) + n % CT * 1024 + lane * 16);
        }
    };
    // keys: fragment (tile, step) at tile * KS + step, two a load; values: (tile, channels, 16 positions), likewise
    auto put = [&](const uint4 (&from)[LOADS], int st, int which) {
        unsigned char *at = mine + which * (2 * HALF) + (st & 1) * HALF;
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int n = wave * LOADS + i;
            Frag<bf16_t> a, b;
            convert<FORMAT>(from[i], a, b);
            *reinterpret_cast<uint4 *>(at + (2 * n) * 1024) = a.v;
            *reinterpret_cast<uint4 *>(at + (2 * n + 1) * 1024) = b.v;
        }
    };
    auto hide_values = [&](int st) {   // in the codes that have been loaded for stage st
        const int left = end - begin - st * KT;
        if (FORMAT == PSD_KV8_E4M3 && left < KT) {   // (whole numbers are no NaN)
#pragma unroll
            for (int i = 0; i < LOADS; ++i) vc[i] = keep(vc[i], left - (wave * LOADS + i) / CT * 32 - 4 * half);
        }
    };
    auto scores = [&](floatx16 (&x)[2], int st) {
        const unsigned char *at = mine + (st & 1) * HALF;
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
    };
    // what the wavefront put into LDS has arrived, and so has everybody's
    auto meet = [&]() {
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    // Stage st, whose scores are in x.  In LDS: keys of st + 1 and values of st; in registers: codes of the keys of st + 2 and of the values of st + 1.  They go
    // where the keys of st and the values of st - 1 were, which all wavefronts have read in front of the last meeting.
    // The order is laid out by hand, in pieces that the compiler keeps apart: two products each, whose fragments were read a piece ahead, beside a part of
    // the exponentials or the conversion of one fragment.
    auto stage = [&](int st, floatx16 (&x)[2], floatx16 (&next)[2]) {
        const unsigned char *ak = mine + ((st + 1) & 1) * HALF, *av = mine + 2 * HALF + (st & 1) * HALF;
        unsigned char *pk = mine + (st & 1) * HALF, *pv = mine + 2 * HALF + ((st + 1) & 1) * HALF;
        Frag<bf16_t> f[2][2];
        auto read = [&](Frag<bf16_t> (&to)[2], const unsigned char *at, int a, int b) {
            to[0].v = *reinterpret_cast<const uint4 *>(at + a * 1024);
            to[1].v = *reinterpret_cast<const uint4 *>(at + b * 1024);
        };
        read(f[0], ak, 0, KS);
        Scale scale[4];
        const float inv = Scale::reciprocal(sc.y);   // of lane g: group g
        auto of_lane = [](float x, int g) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), g)); };
#pragma unroll
        for (int g = 0; g < 4; ++g) scale[g] = Scale(of_lane(sc.x, g) * sl2, of_lane(sc.y, g), of_lane(inv, g));
        sc = head.scale(t0 + 2 * (st + 1), lane & 3);
        const int left = end - begin - st * KT;
        if (left < KT) hide(x, scale, left, half);
        hide_values(st + 1);
        soft.reference(x, scale, acc);
        soft.scale_far(x, scale);
        Frag<bf16_t> p[4];
        float e[4][8], sum[2] = {0.f, 0.f};
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
            for (int v = 0; v < 16; ++v) next[kt][v] = 0.f;
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            if (ks + 1 < KS) read(f[(ks + 1) & 1], ak, ks + 1, KS + ks + 1);
            else read(f[(ks + 1) & 1], av, 0, 2);   // (value_at(0), value_at(1))
            product(f[ks & 1][0], qf[ks], next[0]);
            product(f[ks & 1][1], qf[ks], next[1]);
            constexpr int N = 32 / KS;
#pragma unroll
            for (int i = ks * N; i < ks * N + N; ++i) {
                e[i >> 3][i & 7] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[i >> 4][i & 15], scale[i >> 3].k, soft.neg));
                sum[i & 1] = (i & 7) < 2 ? e[i >> 3][i & 7] : sum[i & 1] + e[i >> 3][i & 7];
                if ((i & 7) == 7) {
                    soft.l += sum[0] + sum[1];
                    soft.weigh(e[i >> 3], sum[0] + sum[1], scale[i >> 3], p[i >> 3]);
                }
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        // product j of the values: 16 positions g = j / CT, channels j % CT, whose fragment is the one at 2 (g / 2 CT + j % CT) + g % 2
        auto value_at = [](int j) { return ((j / CT >> 1) * CT + j % CT) * 2 + (j / CT & 1); };
#pragma unroll
        for (int j = 0; j < 4 * CT; j += 2) {
            const int i = j / 2, of = i / 2 % LOADS, n = wave * LOADS + of;   // fragment i of the next stages': keys first
            Frag<bf16_t>(&now)[2] = f[(KS + i) & 1];
            if (j + 2 < 4 * CT) read(f[(KS + i + 1) & 1], av, value_at(j + 2), value_at(j + 3));
            product(now[0], p[j / CT], acc[j % CT]);
            product(now[1], p[(j + 1) / CT], acc[(j + 1) % CT]);
            const bool keys = i < 2 * LOADS;
            const uint4 c = keys ? kc[of] : vc[of];
            *reinterpret_cast<uint4 *>((keys ? pk : pv) + (2 * n + (i & 1)) * 1024) = i & 1 ? convert<FORMAT>(c.z, c.w) : convert<FORMAT>(c.x, c.y);
            if (i == 2 * LOADS - 1) load(kc, st + 3, 0);
            if (i == 4 * LOADS - 1) load(vc, st + 2, 1);
            __builtin_amdgcn_sched_barrier(0);
        }
        meet();
    };
    if (stages > 0) {
        floatx16 x[2], y[2];
        load(kc, 0, 0);
        load(vc, 0, 1);
        sc = head.scale(t0, lane & 3);
        put(kc, 0, 0);
        load(kc, 1, 0);
        hide_values(0);
        put(vc, 0, 1);
        load(vc, 1, 1);
        put(kc, 1, 0);
        load(kc, 2, 0);
        meet();
        scores(x, 0);
        meet();
        for (int st = 0; st < stages; st += 2) {
            stage(st, x, y);
            if (st + 1 < stages) stage(st + 1, y, x);
        }
    }
    if (ln.k && split == ln.splits - 1 && r_first < rows) 
        own_blocks<bf16_t, DH, CT>(sh, ln, u, kvh, r_first, rows, row.token, 0, 1, sl2, [&](int ks) { return qf[ks]; }, soft, acc, lds + wave * own_lds<bf16_t, DH>());
    const float l_run = both_sum(soft.l), fix = soft.correction<bf16_t>();
    if (r >= rows) return;
    const PartOut<bf16_t, DH> to(sh, ln, split, row);
    if (half == 0) to.sums(soft.m, l_run, 1.f);
    const float f = to.factor(l_run);
    if (f == 0.f && !to.direct) return;
#pragma unroll
    for (int ct = 0; ct < CT; ++ct)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const float o[4] = {acc[ct][4 * g] * fix, acc[ct][4 * g + 1] * fix, acc[ct][4 * g + 2] * fix, acc[ct][4 * g + 3] * fix};
            to.values(ct * 32 + 8 * g + 4 * half, o, f);
        }
}

template <typename T, int DH, bool MANY>
constexpr int attention_lds() {
    return MANY ? 2 * KT * DH * 4 : few_rows_lds<T, DH>();
}

// Every (unit, KV head, part) is dealt to an XCD, one after the other, with all of its tiles: those that read the same keys meet in one L2.  Parts are turned by
// one from one unit and head to the next, so that no XCD has only first parts, which every unit fills, and another only last ones (32 caches of up to 16384
// positions: 71 us dealt in order, 64 so).
template <typename T, int DH, int FORMAT, bool MANY>
__global__ __launch_bounds__(NW * 64, 2) void attention_kv8_kernel(const T *__restrict__ q, SharedShape sh, Kv8Launch ln, float sl2) {
    extern __shared__ __align__(16) unsigned char lds[];
    const int tile = (int)(blockIdx.x >> 3) % ln.tiles, of = (int)(blockIdx.x >> 3) / ln.tiles * 8 + (int)(blockIdx.x & 7);
    if (of >= ln.units * sh.n_kv_heads * ln.splits) return;
    const int head = of / ln.splits, split = (of % ln.splits + head % ln.splits) % ln.splits, kvh = head % sh.n_kv_heads, u = head / sh.n_kv_heads;
    if constexpr (MANY) many_rows<DH, FORMAT>(q, sh, ln, u, kvh, tile, split, sl2, lds);
    else few_rows<T, DH, FORMAT>(q, sh, ln, u, kvh, tile, split, sl2, lds);
}

int64_t workgroups(const SharedShape &sh, const Kv8Launch &ln) { return align_up((int64_t)ln.units * sh.n_kv_heads * ln.splits, 8) * ln.tiles; }

template <typename T, int DH, int FORMAT, bool MANY>
void run(const T *q, const SharedShape &sh, const Kv8Launch &ln, hipStream_t st) {
    constexpr int smem = attention_lds<T, DH, MANY>();
    auto kern = attention_kv8_kernel<T, DH, FORMAT, MANY>;
    static std::atomic<uint64_t> lds_raised{0};   // one per instantiation
    ensure_dynamic_lds(reinterpret_cast<const void *>(kern), smem, lds_raised);
    hipLaunchKernelGGL(kern, dim3((unsigned)workgroups(sh, ln)), dim3(NW * 64), smem, st, q, sh, ln, LOG2E / sqrtf((float)DH));
}
template <typename T, int DH>
void run(const T *q, const SharedShape &sh, const Kv8Launch &ln, hipStream_t st) {
    const bool int8 = ln.cache.format == PSD_KV8_INT8;
    if constexpr (sizeof(T) == 2) {
        if (ln.tiled) {
            if (int8) run<T, DH, PSD_KV8_INT8, true>(q, sh, ln, st);
            else run<T, DH, PSD_KV8_E4M3, true>(q, sh, ln, st);
            return;
        }
    }
    if (int8) run<T, DH, PSD_KV8_INT8, false>(q, sh, ln, st);
    else run<T, DH, PSD_KV8_E4M3, false>(q, sh, ln, st);
}

// Both forms and every number of parts priced, in us (what the sizes below took on this card, heads of 128 unless it says otherwise):
//   a workgroup alone on a CU  few rows: 0.93 for 128 keys (32768 keys of 4 requests, 16 workgroups), 0.55 with heads of 64, 2.7 in fp32 with heads of 64;
//                              many rows: 1.36 for 64 keys (2000 keys, 8 drafts of 64 rows)
//   two and more               few rows: 0.88 a workgroup, 0.75 with e4m3, whose conversion is shorter (one unit of 512 rows a KV head; 4 of 1344); many rows: 1.25
//                              (fp32 in proportion from heads of 64: of 128 it is 32 us against 18 for 4 blocks of 16 rows of 8 heads over 4000 keys)
//   fixed                      4.5 for the call, 2 or 5 for a workgroup, 4 for the join
//   memory                     5.7 TB/s (32 caches of 16384 keys: 94 us)
// and units of lengths of their own, which are taken to be about half full, by how long the last of them runs.
std::atomic<int> forced_form{-1}, forced_parts{0};

struct Price {
    double us;
    int tiles, splits, each;
};
Price price(const SharedShape &sh, const Kv8 &c, bool own_rows, bool many, int units) {
    const bool fp32 = sh.dtype == PSD_DTYPE_FP32;
    const int64_t rows = (int64_t)c.seqs_per_unit * sh.L * (sh.n_heads / sh.n_kv_heads);
    const int rows_of_tile = many ? MT : TR, keys = many ? KT : KV8_TILE * NW, steps = (int)((c.len + (int64_t)keys - 1) / keys);
    const double size = sh.d_head / 128.0, power = sqrt(size) * sqrt(sqrt(size)), step = fp32 ? 5.4 * size : many ? 1.36 * size : 0.93 * power;
    const double shared = fp32 ? step : many ? 1.25 * size : (c.format == PSD_KV8_E4M3 ? 0.75 : 0.88) * power;
    const double fixed = many ? 5.0 : 2.0, full = c.lens ? 0.55 : 1.0;
    const double own = own_rows ? (sh.L + 31) / 32 * (many ? 0.7 : 0.35) * step : 0.0;
    const double memory = (double)units * sh.n_kv_heads * c.len * sh.d_head * 2 * full / 5.7e6, join_part = (double)sh.n_rows * sh.d_head * 8 / 4e6;
    Price best = {-1.0, (int)((rows + rows_of_tile - 1) / rows_of_tile), 1, std::max(steps, 1)};
    const double base = (double)units * sh.n_kv_heads * best.tiles;
    // (up to as many parts as give the CUs eight workgroups each, no more than 256 MB of them but for one, every eighth of many: this is host time of every call)
    if (const int parts = std::min(forced_parts.load(), std::max(steps, 1))) {
        best.each = (steps + parts - 1) / parts;
        best.splits = std::max(1, (steps + std::max(best.each, 1) - 1) / std::max(best.each, 1));
        best.us = 0.0;
        return best;
    }
    for (int n = 1; n <= std::max(1, steps) && (n == 1 || (base * n <= 2048.0 && (double)n * sh.n_rows * sh.d_head * 4 <= 256e6)); n += 1 + n / 8) {
        const int each = std::max((steps + n - 1) / n, 1), splits = std::max((steps + each - 1) / each, 1);
        // (a CU with one workgroup more than the others is the last; units of lengths of their own even that out)
        const double wgs = c.lens ? base * splits / 256.0 : ceil(base * splits / 256.0);
        const double work = wgs * (each * shared * full + fixed * 0.8), alone = each * step + fixed;
        const double us = 4.5 + std::max(std::max(alone, work), memory) + (c.lens ? 0.3 * each * step : 0.0) + own + (splits > 1 ? 4.0 + splits * join_part : 0.0);
        if (best.us < 0.0 || us < best.us) best.us = us, best.splits = splits, best.each = each;
        if (steps * step < 4.0 + step) break;   // (less than a join takes)
    }
    return best;
}

}   // namespace

void force_attention_kv8(int form, int parts) {
    forced_form = form;
    forced_parts = parts;
}

bool plan_attention_kv8(const SharedShape &sh, const Kv8 &cache, bool own_rows, Kv8Launch *out) {
    Kv8Launch ln;
    ln.cache = cache;
    ln.units = sh.S / cache.seqs_per_unit;
    Price p = price(sh, cache, own_rows, false, ln.units);
    const int form = forced_form;
    if (sh.dtype == PSD_DTYPE_BF16 && (form == 1 || (form < 0 && (int64_t)cache.seqs_per_unit * sh.L * (sh.n_heads / sh.n_kv_heads) > MT / 2))) {
        const Price many = price(sh, cache, own_rows, true, ln.units);
        if (form == 1 || many.us < p.us) p = many, ln.tiled = 1;
    }
    ln.tiles = p.tiles;
    ln.splits = p.splits;
    ln.chunk = std::max(p.each, 1) * (ln.tiled ? KT : KV8_TILE * NW);
    ln.parts = ln.splits > 1 ? ln.splits : 0;
    *out = ln;
    return (double)ln.units * sh.n_kv_heads * ln.tiles * ln.splits < 0x1p31 && launchable(workgroups(sh, ln), NW * 64) &&
           (ln.parts == 0 || attention_join_launchable(sh, ln));
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
