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
// Per tile the problem is transposed as in attention_mfma.hip: S^T = K Q^T, O^T += V^T P^T.  A lane owns one row; the softmax stays
// in its registers, and the probabilities are the second product's operand as they are.
#include "psd_internal.h"
#include "device_types.h"

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float floatx16 __attribute__((ext_vector_type(16)));

constexpr int TR = 32;    // rows per tile
constexpr int BK = 32;    // keys that a wavefront takes at a time
constexpr int NW = 4;     // wavefronts of a workgroup, which deal a tile's keys among themselves
constexpr float LOG2E = 1.4426950408889634f;

// A row of 8 slots of T, as a lane of a 32x32 product holds it: bf16 in one 16-byte load, fp32 in two.
template <typename T>
struct Frag;
template <>
struct Frag<bf16_t> {
    uint4 v;
    __device__ void load(const bf16_t *p) { v = *reinterpret_cast<const uint4 *>(p); }
    __device__ void zero() { v = make_uint4(0, 0, 0, 0); }
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
    __device__ void zero() {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = 0.f;
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

// the keys that unit u (of the launch) sees, as device pointers of one KV head
template <typename T>
struct Keys {
    const T *k, *vt;
    int len;
};
template <typename T>
__device__ __forceinline__ Keys<T> keys_of(const SharedSegment &s, int u, int kvh, int d_head) {
    const int64_t cache = s.rows ? s.rows[(int64_t)u * s.seqs_per_unit] / s.rows_div : u;
    Keys<T> r;
    r.k = (const T *)s.k + cache * s.stride_k + kvh * d_head;
    r.vt = (const T *)s.vt + cache * s.stride_vt + (int64_t)kvh * d_head * s.ld_vt;
    r.len = s.lens ? min(max(s.lens[cache], 0), s.len) : s.len;   // (a length outside the unit is cut to it)
    return r;
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

// One workgroup: a tile of TR rows of a unit against a part of the unit's keys.  The wavefronts deal the keys, BK at a time, operands
// straight from memory, and merge in LDS in wavefront order.
template <typename T, int DH>
__global__ __launch_bounds__(NW * 64, 2) void shared_attention_kernel(const T *__restrict__ q, SharedShape sh, SharedLaunch ln, float sl2) {
    constexpr int KS = DH / 16, CT = (DH + 31) / 32, NF = CT * 16;   // contraction steps of the scores, channel subtiles, output values per lane
    extern __shared__ __align__(16) float part[];                   // [wavefront][max, sum, NF values][64 lanes]
    int j = 0;
    while (j + 1 < ln.n_jobs && (int)blockIdx.x >= ln.job[j + 1].block0) ++j;
    const SharedJob &jb = ln.job[j];
    const SharedSegment &seg = ln.seg[j];
    // (unit, KV head, part) groups are dealt to the XCDs, all tiles of a group to one: they read the same keys
    const int local = blockIdx.x - jb.block0, slot = local >> 3;
    const int grp = slot / jb.tiles * 8 + (local & 7), tile = slot % jb.tiles;
    if (grp >= jb.units * sh.n_kv_heads * jb.splits) return;
    const int split = grp % jb.splits, kvh = grp / jb.splits % sh.n_kv_heads, u = grp / jb.splits / sh.n_kv_heads;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lrow = lane & 31, half = lane >> 5;
    const Keys<T> keys = keys_of<T>(seg, u, kvh, DH);
    const int n_steps = (keys.len + BK - 1) / BK;
    const int first = (int)((int64_t)n_steps * split / jb.splits), last = (int)((int64_t)n_steps * (split + 1) / jb.splits);

    const int rows = seg.seqs_per_unit * sh.L * (sh.n_heads / sh.n_kv_heads), r = tile * TR + lrow;
    const RowOf row(sh, (int64_t)u * seg.seqs_per_unit, kvh, min(r, rows - 1));   // (rows past the last repeat it and store nothing)
    Frag<T> qf[KS];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qf[ks].load(q + row.token * sh.ld_q + row.head * DH + ks * 16 + half * 8);

    floatx16 acc_o[CT];
#pragma unroll
    for (int ct = 0; ct < CT; ++ct)
#pragma unroll
        for (int v = 0; v < 16; ++v) acc_o[ct][v] = 0.f;
    float m_run = -INFINITY, l_run = 0.f;
    for (int st = first + wave; st < last; st += NW) {
        const int k0 = st * BK, left = keys.len - k0;
        floatx16 x;
#pragma unroll
        for (int v = 0; v < 16; ++v) x[v] = 0.f;
        const T *krow = keys.k + (int64_t)min(k0 + lrow, keys.len - 1) * seg.ld_k + half * 8;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            Frag<T> kf;
            kf.load(krow + ks * 16);
            product(kf, qf[ks], x);
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
        mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
        const float m_new = fmaxf(m_run, mx);
        const float m_s = m_new == -INFINITY ? 0.f : m_new * sl2;   // (scores of -inf alone: infinite keys)
        const float alpha = __builtin_amdgcn_exp2f(__builtin_fmaf(m_run, sl2, -m_s));
        float p[16], psum = 0.f;
#pragma unroll
        for (int v = 0; v < 16; ++v) {
            p[v] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[v], sl2, -m_s));
            psum += p[v];
        }
        l_run = l_run * alpha + psum;
        m_run = m_new;
#pragma unroll
        for (int ct = 0; ct < CT; ++ct)
#pragma unroll
            for (int v = 0; v < 16; ++v) acc_o[ct][v] *= alpha;
#pragma unroll
        for (int kg = 0; kg < BK / 16; ++kg) {
            if (kg * 16 >= left) break;   // (a value row ends with the group of 16 that its last key is in)
            Frag<T> pf;
            probabilities(p + 8 * kg, pf);
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) {
                const int c = CT * 32 > DH ? min(lrow, DH - 1) : ct * 32 + lrow;
                Frag<T> vf;
                vf.load(keys.vt + (int64_t)c * seg.ld_vt + k0 + kg * 16 + half * 8);
                // slots behind the last key hold anything: their probabilities are zero, but 0 x NaN is NaN
                if (left < BK) vf.keep(left - kg * 16 - 4 * half);
                product(vf, pf, acc_o[ct]);
            }
        }
    }
    l_run += __shfl_xor(l_run, 32, 64);   // the halves of a row hold disjoint keys

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
    const float m_s = m_all == -INFINITY ? 0.f : m_all * sl2;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
        scale[w] = __builtin_amdgcn_exp2f(__builtin_fmaf(scale[w], sl2, -m_s));
        l_all += part[(w * (2 + NF) + 1) * 64 + lane] * scale[w];
    }
    if (r >= rows) return;
    const int64_t at = (int64_t)(jb.part0 + split) * sh.n_rows + row.token * sh.n_heads + row.head;
    if (wave == 0 && half == 0) ln.ml[at] = make_float2(l_all > 0.f || l_all != l_all ? m_all : -INFINITY, l_all);
    if (l_all == 0.f) return;   // (no keys: the join reads no values)
    float *op = ln.o + at * DH;
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
        *reinterpret_cast<float4 *>(op + c) = make_float4(o[0], o[1], o[2], o[3]);
    }
}

// The parts of a row joined, in their order: a thread takes 4 channels.
template <typename T, int DH>
__global__ __launch_bounds__(256) void shared_join_kernel(SharedShape sh, SharedLaunch ln, T *__restrict__ out, float *__restrict__ lse, float sl2) {
    constexpr int TPR = DH / 4;   // threads per row
    const int64_t r = (int64_t)blockIdx.x * (256 / TPR) + threadIdx.x / TPR;
    if (r >= sh.n_rows) return;
    const int c = threadIdx.x % TPR * 4;
    float m = -INFINITY;
    for (int p = 0; p < ln.parts; ++p) m = fmaxf(m, ln.ml[(int64_t)p * sh.n_rows + r].x);
    const float m_s = m == -INFINITY ? 0.f : m * sl2;
    float l = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
    for (int p = 0; p < ln.parts; ++p) {
        const float2 ml = ln.ml[(int64_t)p * sh.n_rows + r];
        if (ml.y == 0.f) continue;
        const float w = __builtin_amdgcn_exp2f(__builtin_fmaf(ml.x, sl2, -m_s));
        const float4 v = *reinterpret_cast<const float4 *>(ln.o + ((int64_t)p * sh.n_rows + r) * DH + c);
        l += w * ml.y;
        o[0] += w * v.x, o[1] += w * v.y, o[2] += w * v.z, o[3] += w * v.w;
    }
    const float inv = l == 0.f ? 0.f : 1.0f / l;   // (a row without keys: zeros)
    T *op = out + r / sh.n_heads * sh.ld_out + r % sh.n_heads * DH + c;
#pragma unroll
    for (int v = 0; v < 4; ++v) op[v] = from_float<T>(o[v] * inv);
    if (lse && c == 0) lse[r] = l == 0.f ? -INFINITY : m_s / LOG2E + logf(l);
}

// w[j] (+)= sum over the rows of the unit of exp(x_j - lse).  A wavefront keeps 32 keys in registers and walks all rows; a lane adds
// up what its row of every tile gives, and the lanes are added at the end, in one order whatever the launch.
template <typename T, int DH>
__global__ __launch_bounds__(NW * 64) void shared_weights_kernel(const T *__restrict__ q, const float *__restrict__ lse, SharedShape sh, SharedLaunch ln,
                                                                 int accumulate, float sl2) {
    constexpr int KS = DH / 16;
    int j = 0;
    while (j + 1 < ln.n_jobs && (int)blockIdx.x >= ln.job[j + 1].block0) ++j;
    const SharedJob &jb = ln.job[j];
    const SharedSegment &seg = ln.seg[j];
    const int local = blockIdx.x - jb.block0;
    const int u = local / (jb.splits * sh.n_kv_heads), kvh = local / jb.splits % sh.n_kv_heads, part = local % jb.splits;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lrow = lane & 31, half = lane >> 5;
    const Keys<T> keys = keys_of<T>(seg, u, kvh, DH);
    const int k0 = (part * NW + wave) * BK;
    if (k0 >= keys.len) return;
    Frag<T> kf[KS];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) kf[ks].load(keys.k + (int64_t)min(k0 + lrow, keys.len - 1) * seg.ld_k + ks * 16 + half * 8);
    const int rows = seg.seqs_per_unit * sh.L * (sh.n_heads / sh.n_kv_heads);
    float w[16];
#pragma unroll
    for (int v = 0; v < 16; ++v) w[v] = 0.f;
    for (int r0 = 0; r0 < rows; r0 += TR) {
        const RowOf row(sh, (int64_t)u * seg.seqs_per_unit, kvh, min(r0 + lrow, rows - 1));
        const float z = r0 + lrow < rows ? lse[row.token * sh.n_heads + row.head] * LOG2E : INFINITY;   // (rows past the last one give nothing)
        floatx16 x;
#pragma unroll
        for (int v = 0; v < 16; ++v) x[v] = 0.f;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            Frag<T> qf;
            qf.load(q + row.token * sh.ld_q + row.head * DH + ks * 16 + half * 8);
            product(kf[ks], qf, x);
        }
#pragma unroll
        for (int v = 0; v < 16; ++v) w[v] += __builtin_amdgcn_exp2f(__builtin_fmaf(x[v], sl2, -z));
    }
    const int64_t cache = seg.rows ? seg.rows[(int64_t)u * seg.seqs_per_unit] / seg.rows_div : u;
    float *to = seg.weights + cache * seg.stride_w + (int64_t)kvh * seg.ld_w;
#pragma unroll
    for (int v = 0; v < 16; ++v) {
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) w[v] += __shfl_xor(w[v], d, 64);
        const int key = k0 + 8 * (v >> 2) + 4 * half + (v & 3);
        if (lrow == 0 && key < keys.len) to[key] = accumulate ? to[key] + w[v] : w[v];
    }
}

__global__ __launch_bounds__(256) void block_values_kernel(const float *__restrict__ qkv, int ld_qkv, int v_col, int L, int width, float *__restrict__ vT,
                                                           int ld_vt) {
    const int64_t s = blockIdx.x / L;
    const int i = blockIdx.x % L;
    for (int c = threadIdx.x; c < width; c += 256) vT[(s * width + c) * ld_vt + vt_key_slot(i)] = qkv[(int64_t)blockIdx.x * ld_qkv + v_col + c];
}

bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

template <typename T, int DH>
void run_attention(const T *q, const SharedShape &sh, const SharedLaunch &ln, T *out, float *lse, hipStream_t st) {
    constexpr int smem = NW * (2 + (DH + 31) / 32 * 16) * 64 * 4;
    const float sl2 = LOG2E / sqrtf((float)DH);
    auto kern = shared_attention_kernel<T, DH>;
    static std::atomic<uint64_t> lds_raised{0};   // one per instantiation
    ensure_dynamic_lds(reinterpret_cast<const void *>(kern), smem, lds_raised);
    if (ln.blocks > 0) hipLaunchKernelGGL(kern, dim3((unsigned)ln.blocks), dim3(NW * 64), smem, st, q, sh, ln, sl2);
    constexpr int rows = 256 / (DH / 4);
    hipLaunchKernelGGL((shared_join_kernel<T, DH>), dim3((unsigned)((sh.n_rows + rows - 1) / rows)), dim3(256), 0, st, sh, ln, out, lse, sl2);
}

template <typename T, int DH>
void run_weights(const T *q, const float *lse, const SharedShape &sh, const SharedLaunch &ln, int accumulate, hipStream_t st) {
    if (ln.blocks > 0)
        hipLaunchKernelGGL((shared_weights_kernel<T, DH>), dim3((unsigned)ln.blocks), dim3(NW * 64), 0, st, q, lse, sh, ln, accumulate,
                           LOG2E / sqrtf((float)DH));
}

// the work of one launch: a job per segment, its workgroups behind those of the one before
SharedLaunch plan_attention(const SharedShape &sh, const SharedSegment *seg, int n) {
    SharedLaunch ln;
    int64_t blocks = 0;
    for (int i = 0; i < n; ++i) {
        if (seg[i].len == 0) continue;
        SharedJob &jb = ln.job[ln.n_jobs];
        ln.seg[ln.n_jobs++] = seg[i];
        const int rows = seg[i].seqs_per_unit * sh.L * (sh.n_heads / sh.n_kv_heads);
        jb.units = sh.S / seg[i].seqs_per_unit;
        jb.tiles = (rows + TR - 1) / TR;
        jb.block0 = (int)blocks;
        jb.part0 = ln.parts;
        const int64_t base = (int64_t)jb.units * sh.n_kv_heads * jb.tiles;
        const int most = (seg[i].len + NW * BK - 1) / (NW * BK);   // every wavefront has a step
        jb.splits = (int)std::min<int64_t>(most, std::max<int64_t>(1, 1024 / base));
        ln.parts += jb.splits;
        blocks += align_up((int64_t)jb.units * sh.n_kv_heads * jb.splits, 8) * jb.tiles;
    }
    ln.blocks = blocks;
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

int64_t shared_attention_bytes(const SharedShape &sh, const SharedSegment *seg, int n) {
    const SharedLaunch ln = plan_attention(sh, seg, n);
    return align_up((int64_t)ln.parts * sh.n_rows * sh.d_head * 4, 256) + align_up((int64_t)ln.parts * sh.n_rows * 8, 256);
}

bool shared_attention_fits(const SharedShape &sh, const SharedSegment *seg, int n) { return plan_attention(sh, seg, n).blocks < (1ll << 31); }

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

void launch_attention_shared(const void *q, const SharedShape &sh, const SharedSegment *seg, int n, void *out, float *lse, void *ws, hipStream_t st) {
    SharedLaunch ln = plan_attention(sh, seg, n);
    ln.o = (float *)ws;
    ln.ml = (float2 *)((char *)ws + align_up((int64_t)ln.parts * sh.n_rows * sh.d_head * 4, 256));
    PSD_SHARED_DISPATCH((run_attention<T, DH>((const T *)q, sh, ln, (T *)out, lse, st)))
}

void launch_block_values(const float *qkv, int ld_qkv, int v_col, int S, int L, int width, float *vT, int ld_vt, hipStream_t st) {
    hipLaunchKernelGGL(block_values_kernel, dim3((unsigned)(S * L)), dim3(256), 0, st, qkv, ld_qkv, v_col, L, width, vT, ld_vt);
}

int64_t shared_weights_bytes(const SharedShape &, const SharedSegment *, int) { return 0; }

void launch_attention_weights(const void *q, const SharedShape &sh, const SharedSegment *seg, int n, const float *lse, int accumulate, void *,
                              hipStream_t st) {
    SharedLaunch ln;
    int64_t blocks = 0;
    for (int i = 0; i < n; ++i) {
        if (!seg[i].weights || seg[i].len == 0) continue;
        SharedJob &jb = ln.job[ln.n_jobs];
        ln.seg[ln.n_jobs++] = seg[i];
        jb.units = sh.S / seg[i].seqs_per_unit;
        jb.splits = (seg[i].len + NW * BK - 1) / (NW * BK);
        jb.block0 = (int)blocks;
        blocks += (int64_t)jb.units * sh.n_kv_heads * jb.splits;
    }
    ln.blocks = blocks;
    PSD_SHARED_DISPATCH((run_weights<T, DH>((const T *)q, lse, sh, ln, accumulate, st)))
}
