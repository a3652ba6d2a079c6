// Attention over the tokens of channel-first maps, forward and backward.
//
// Forward, for each query: one pass over the keys with the running maximum m and
// sum l of the softmax; o = sum_j exp(s_j - m) v_j / l.  Backward, with the
// logarithm of the sum (lse) and D_i = do_i . o_i:
//   P = exp(S - lse), dV = P^T dO, dS = P (dO V^T - D), dQ = scale dS K,
//   dK = scale dS^T Q,
// in two kernels, one that keeps keys and walks the queries (dK, dV), one that
// keeps queries and walks the keys (dQ): S is formed three times in a training
// step, and no sum is shared between workgroups, so nothing is atomic and every
// result has the same bits each time.
//
// All products run on 32x32 matrix instructions (bfloat16 x16, float32 x2).  The
// accumulator of a product has one column (lane & 31) and 16 rows a lane, so the
// scores are formed with the kept tokens as columns and the walked ones as rows:
// a softmax row lies in two lanes, and the probabilities are, register for
// register, the second operand of the products that follow.  What this needs of
// the other operand is an order of its contraction index, which the packing gives.
//
// Packing: operands are laid out once per call, in the workspace, in the order in
// which lanes hold them (a 16-byte unit a lane, 1 KB a fragment), in two forms:
//   R: rows are 32 tokens, the contraction runs over the head's channels;
//   T: rows are 32 channels, the contraction runs over 32 tokens, in the order of
//      the accumulator's rows.
// Head sizes are filled up with zeros to a multiple of 32, token counts to one of
// 64.  Masked keys are left out: the live ones move up (an index list, made from
// the mask), so masked voxels cost nothing and what they hold is never read.
#include <math.h>

#include "kernels.hpp"
#include "prof.hpp"

namespace rat3d {

typedef __attribute__((ext_vector_type(16))) float f32x16;

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

// One operand fragment: 16 bytes a lane.  R covers kR channels, T covers kT tokens.
template <typename T> struct Mm;
template <> struct Mm<bf16> {
    typedef bf16x8 frag;
    static constexpr int kR = 16, kT = 16, kPer = 8;
    __device__ __forceinline__ static f32x16 mul(frag a, frag b, f32x16 c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
    }
};
template <> struct Mm<float> {
    typedef f32x4 frag;
    static constexpr int kR = 8, kT = 8, kPer = 4;
    __device__ __forceinline__ static f32x16 mul(frag a, frag b, f32x16 c) {
        c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[0], b[0], c, 0, 0, 0);
        c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[1], b[1], c, 0, 0, 0);
        c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[2], b[2], c, 0, 0, 0);
        c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[3], b[3], c, 0, 0, 0);
        return c;
    }
};

// Accumulator register i of a lane is row 8 (i / 4) + 4 (lane / 32) + i % 4.
// Registers i .. i + kPer - 1 as an operand of contraction kT.  Probabilities and
// score gradients are rounded to the storage type here, as the matrix instruction
// takes them; the sums over them stay in float32.
template <typename T>
__device__ __forceinline__ typename Mm<T>::frag to_frag(const f32x16& p, int u);
template <>
__device__ __forceinline__ bf16x8 to_frag<bf16>(const f32x16& p, int u) {
    u32x4 w;
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = pack_bf16x2(p[8 * u + 2 * i], p[8 * u + 2 * i + 1]);
    return __builtin_bit_cast(bf16x8, w);
}
template <>
__device__ __forceinline__ f32x4 to_frag<float>(const f32x16& p, int u) {
    return f32x4{p[4 * u], p[4 * u + 1], p[4 * u + 2], p[4 * u + 3]};
}

// x of this lane and of the lane 32 away.
__device__ __forceinline__ void halves(float x, float& a, float& b) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false,
                                                    false);
    a = __uint_as_float(r[0]);
    b = __uint_as_float(r[1]);
}

// ------------------------------------------------------------------ live keys
// idx[n][j] = the j-th token whose mask byte is not 0, count[n] = how many.
// One workgroup a volume: each turn a thread looks at four tokens.
__global__ __launch_bounds__(1024) void live_keys_k(const uint8_t* __restrict__ mask, int64_t T,
                                                    int64_t Tp, int* __restrict__ idx,
                                                    int* __restrict__ count) {
    __shared__ int wsum[16];
    const uint8_t* m = mask + blockIdx.x * T;
    int* to = idx + blockIdx.x * Tp;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int base = 0;
    for (int64_t t0 = 0; t0 < T; t0 += 4096) {
        const int64_t t = t0 + threadIdx.x * 4;
        int on[4], mine = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            on[j] = t + j < T && m[t + j] != 0;
            mine += on[j];
        }
        int incl = mine;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int o = __shfl_up(incl, d);
            if (lane >= d) incl += o;
        }
        if (lane == 63) wsum[wave] = incl;
        __syncthreads();
        int before = base, all = 0;
#pragma unroll
        for (int w = 0; w < 16; ++w) {
            if (w < wave) before += wsum[w];
            all += wsum[w];
        }
        int at = before + incl - mine;
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (on[j]) to[at++] = (int)(t + j);
        base += all;
        __syncthreads();
    }
    if (threadIdx.x == 0) count[blockIdx.x] = base;
}

// ------------------------------------------------------------------ packing
struct PackJob {
    const void* src;     // [n][heads * D][tokens], volumes `stride` apart
    const void* other;   // o, where src is dout: D = sum over channels of src * other
    const float* lse;
    void* r;             // form R, or null
    void* t;             // form T, or null
    float* lse2;         // lse in units of log 2, padded with +infinity
    float* delta;        // D, padded with 0
    const int* idx;      // live tokens, or null
    const int* count;
    int64_t stride, tokens;
    int heads, tiles;    // tiles of 64 tokens
    int first;           // first workgroup of the job
};
struct PackArgs {
    PackJob job[4];
    int jobs, D, DB;
};

constexpr int kPackTok = 64;

// One workgroup: 64 tokens of one head of one volume, through LDS.
template <typename T>
__global__ __launch_bounds__(256) void attn_pack_k(PackArgs a) {
    typedef Mm<T> M;
    constexpr int ROW = kPackTok + (sizeof(T) == 2 ? 2 : 1);  // odd in banks: columns spread
    __shared__ T tile[128 * ROW];
    __shared__ float part[4][kPackTok];
    int ji = 0;
    while (ji + 1 < a.jobs && (int)blockIdx.x >= a.job[ji + 1].first) ++ji;
    const PackJob& J = a.job[ji];
    const int b = (int)blockIdx.x - J.first;
    const int tl = b % J.tiles, nh = b / J.tiles;
    const int vol = nh / J.heads, h = nh - vol * J.heads;
    const int64_t live = J.count ? J.count[vol] : J.tokens;
    const int64_t t0 = (int64_t)tl * kPackTok;
    if (J.count && t0 >= live) return;  // never read: kernels stop at the live keys
    const int col = threadIdx.x & 63, sub = threadIdx.x >> 6;
    const bool in = t0 + col < live;
    const int64_t tok = in ? (J.idx ? J.idx[vol * (int64_t)J.tiles * kPackTok + t0 + col]
                                    : t0 + col)
                           : 0;
    const int64_t base = vol * J.stride + (int64_t)h * a.D * J.tokens + tok;
    const T* src = (const T*)J.src + base;
    const T* oth = J.other ? (const T*)J.other + base : nullptr;
    const int Dp = 32 * a.DB;
    float d = 0.f;
    for (int c = sub; c < Dp; c += 4) {
        T v = Elt<T>::to_bits(0.f);
        if (in && c < a.D) {
            v = src[(int64_t)c * J.tokens];
            if (oth) d += Elt<T>::cvt(v) * Elt<T>::ld(oth + (int64_t)c * J.tokens);
        }
        tile[c * ROW + col] = v;
    }
    part[sub][col] = d;
    __syncthreads();
    if (J.delta && threadIdx.x < kPackTok) {
        const int64_t at = (int64_t)nh * J.tiles * kPackTok + t0 + threadIdx.x;
        J.delta[at] = (part[0][threadIdx.x] + part[1][threadIdx.x]) +
                      (part[2][threadIdx.x] + part[3][threadIdx.x]);
        // without any key lse is -infinity and no key reads it; behind the last
        // query +infinity makes every probability 0
        J.lse2[at] = in ? J.lse[(int64_t)nh * J.tokens + t0 + threadIdx.x] * kLog2e : INFINITY;
    }
    // fragments: 2 blocks of 32 tokens x Dp, 16 bytes a lane
    const int units = 2 * 32 * Dp / M::kPer;  // 16-byte units of one form
    const int64_t out0 = ((int64_t)nh * J.tiles + tl) * units;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int frags = units / 64;
    for (int f = wave; f < frags; f += 4) {
        typedef __attribute__((ext_vector_type(4))) uint32_t unit_t;
        if (J.r) {
            const int per = Dp / M::kR;  // fragments of one block
            const int tk = (f / per) * 32 + (lane & 31);
            const int ch = (f % per) * M::kR + (lane >> 5) * M::kPer;
            T v[M::kPer];
#pragma unroll
            for (int j = 0; j < M::kPer; ++j) v[j] = tile[(ch + j) * ROW + tk];
            unit_t u;
            __builtin_memcpy(&u, v, 16);
            ((unit_t*)J.r)[out0 + f * 64 + lane] = u;
        }
        if (J.t) {
            const int per = 32 / M::kT * a.DB;
            const int blk = f / per, w = f % per / a.DB, e = f % a.DB;
            const int ch = e * 32 + (lane & 31);
            T v[M::kPer];
#pragma unroll
            for (int j = 0; j < M::kPer; ++j)
                v[j] = tile[ch * ROW + blk * 32 + w * M::kT + 8 * (j / 4) + 4 * (lane >> 5) + j % 4];
            unit_t u;
            __builtin_memcpy(&u, v, 16);
            ((unit_t*)J.t)[out0 + f * 64 + lane] = u;
        }
    }
}

// ------------------------------------------------------------------ shared pieces
struct AttnArgs {
    const void* q;  // forward only: queries as given
    void* o;
    float* lse;
    const uint4 *kr, *kt, *vr, *vt, *qr, *qt, *or_, *ot;  // packed operands
    const float *lse2, *delta;
    const int *idx, *count;
    void *dq, *dk, *dv;
    float* part;   // split sums: [nh][split][D][tokens padded]
    float* stat;   // split forward: [nh][split][2][tqp]
    int64_t tq, tk, tqp, tkp;
    int64_t q_stride, k_stride, v_stride, o_stride;
    int heads, kv, D, tiles, splits;
    float scale, c;  // c = scale * log2 e
};

// U 16-byte units, copied by 256 threads from global memory into registers and from
// there into LDS: the loads of the next tile are in flight while this one is
// multiplied.
template <int U> struct Stage {
    static constexpr int N = (U + 255) / 256;
    uint4 v[N];
    __device__ __forceinline__ static bool mine(int i) {
        return (i + 1) * 256 <= U || i * 256 + (int)threadIdx.x < U;
    }
    __device__ __forceinline__ void load(const uint4* __restrict__ p) {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (mine(i)) v[i] = p[i * 256 + threadIdx.x];
    }
    __device__ __forceinline__ void store(uint4* s) const {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (mine(i)) s[i * 256 + threadIdx.x] = v[i];
    }
};

template <typename T>
__device__ __forceinline__ typename Mm<T>::frag frag_of(const uint4* s, int f) {
    return __builtin_bit_cast(typename Mm<T>::frag, s[f * 64 + (threadIdx.x & 63)]);
}

// 32 tokens of a channel-first tensor as fragments of form R (second operand).
template <typename T, int NF>
__device__ __forceinline__ void load_cols(const T* __restrict__ p, int64_t row, int D, bool in,
                                          typename Mm<T>::frag (&f)[NF]) {
    typedef Mm<T> M;
    const int half = (threadIdx.x & 63) >> 5;
#pragma unroll
    for (int i = 0; i < NF; ++i) {
        T v[M::kPer];
#pragma unroll
        for (int j = 0; j < M::kPer; ++j) {
            const int ch = i * M::kR + half * M::kPer + j;
            v[j] = in && ch < D ? p[ch * row] : Elt<T>::to_bits(0.f);
        }
        __builtin_memcpy(&f[i], v, 16);
    }
}

// The keys of a split: blocks of `step` tokens [b0, b1) of those that `live` fill.
__device__ __forceinline__ void split_range(int64_t live, int step, int splits, int s, int& b0,
                                            int& b1) {
    const int nb = (int)((live + step - 1) / step);
    const int per = (nb + splits - 1) / splits;
    b0 = s * per < nb ? s * per : nb;
    b1 = b0 + per < nb ? b0 + per : nb;
}

// ------------------------------------------------------------------ forward
// A workgroup: 128 queries of one head, 32 a wave as columns; KB x 32 keys a turn.
template <typename T, int DB, int KB, bool SPLIT>
__global__ __launch_bounds__(256, 2) void attn_fwd_k(AttnArgs a) {
    typedef Mm<T> M;
    typedef typename M::frag frag;
    constexpr int NR = 32 * DB / M::kR;      // fragments of 32 tokens, form R
    constexpr int NT = 32 / M::kT;           // contraction steps of 32 tokens, form T
    constexpr int NF = 32 * DB / M::kPer * 32 / 64;  // fragments of 32 tokens (either form)
    constexpr int U = KB * NF * 64;          // units of one operand's tile
    __shared__ uint4 lds[2][2][U];
    int bid = xcd_remap(blockIdx.x, gridDim.x);
    const int tile = bid % a.tiles;
    bid /= a.tiles;
    const int sp = SPLIT ? bid % a.splits : 0;
    const int nh = SPLIT ? bid / a.splits : bid;
    const int vol = nh / a.heads, h = nh - vol * a.heads;
    const int kvh = vol * a.kv + h / (a.heads / a.kv);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t live = a.count ? a.count[vol] : a.tk;
    const int64_t qt = (int64_t)tile * 128 + wave * 32 + (lane & 31);
    const bool in = qt < a.tq;

    frag qf[NR];
    load_cols<T, NR>((const T*)a.q + vol * a.q_stride + (int64_t)h * a.D * a.tq + qt, a.tq, a.D,
                     in, qf);

    f32x16 acc[DB];
#pragma unroll
    for (int e = 0; e < DB; ++e)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[e][i] = 0.f;
    float m = -INFINITY, l = 0.f;

    int b0, b1;
    split_range(live, 32 * KB, SPLIT ? a.splits : 1, sp, b0, b1);
    const uint4* kp = a.kr + ((int64_t)kvh * (a.tkp / 32) + (int64_t)b0 * KB) * NF * 64;
    const uint4* vp = a.vt + ((int64_t)kvh * (a.tkp / 32) + (int64_t)b0 * KB) * NF * 64;
    Stage<U> ks, vs;
    if (b0 < b1) {
        ks.load(kp);
        vs.load(vp);
        ks.store(lds[0][0]);
        vs.store(lds[0][1]);
    }
    __syncthreads();
    for (int b = b0; b < b1; ++b) {
        const int buf = (b - b0) & 1;
        if (b + 1 < b1) {
            kp += U;
            vp += U;
            ks.load(kp);
            vs.load(vp);
        }
        f32x16 s[KB];
#pragma unroll
        for (int k = 0; k < KB; ++k) {
#pragma unroll
            for (int i = 0; i < 16; ++i) s[k][i] = 0.f;
#pragma unroll
            for (int f = 0; f < NR; ++f) s[k] = M::mul(frag_of<T>(lds[buf][0], k * NR + f), qf[f], s[k]);
        }
        if ((int64_t)(b + 1) * 32 * KB > live) {  // the last tile: rows behind the last key
            const int left = (int)(live - (int64_t)b * 32 * KB);
#pragma unroll
            for (int k = 0; k < KB; ++k)
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (k * 32 + 8 * (i / 4) + 4 * (lane >> 5) + i % 4 >= left) s[k][i] = -INFINITY;
        }
        float t = s[0][0];
#pragma unroll
        for (int k = 0; k < KB; ++k)
#pragma unroll
            for (int i = 0; i < 16; ++i) t = fmaxf(t, s[k][i]);
        float ta, tb;
        halves(t, ta, tb);
        t = fmaxf(ta, tb) * a.c;
        // The reference of the exponentials follows the maximum only where it grew by
        // more than 8 (in log 2): probabilities then stay below 2^8, which neither
        // bfloat16 nor the float32 sums mind, and the sums are rescaled rarely.
        if (__any(t > m + 8.f)) {
            const float to = t > m + 8.f ? t : m;
            const float f = to == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - to);
            m = to;
            l *= f;
#pragma unroll
            for (int e = 0; e < DB; ++e)
#pragma unroll
                for (int i = 0; i < 16; ++i) acc[e][i] *= f;
        }
        const float ref = m == -INFINITY ? 0.f : m;
#pragma unroll
        for (int k = 0; k < KB; ++k) {
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                s[k][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[k][i], a.c, -ref));
                l += s[k][i];
            }
#pragma unroll
            for (int w = 0; w < NT; ++w) {
                const frag p = to_frag<T>(s[k], w);
#pragma unroll
                for (int e = 0; e < DB; ++e)
                    acc[e] = M::mul(frag_of<T>(lds[buf][1], (k * NT + w) * DB + e), p, acc[e]);
            }
        }
        if (b + 1 < b1) {
            ks.store(lds[buf ^ 1][0]);
            vs.store(lds[buf ^ 1][1]);
        }
        __syncthreads();
    }
    float la, lb;
    halves(l, la, lb);
    l = la + lb;
    if (!in) return;
    const int half = lane >> 5;
    if (SPLIT) {
        float* st = a.stat + ((int64_t)nh * a.splits + sp) * 2 * a.tqp + qt;
        if (half == 0) {
            st[0] = m;
            st[a.tqp] = l;
        }
        float* to = a.part + ((int64_t)nh * a.splits + sp) * a.D * a.tqp + qt;
#pragma unroll
        for (int e = 0; e < DB; ++e)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int ch = e * 32 + 8 * (i / 4) + 4 * half + i % 4;
                if (ch < a.D) to[ch * a.tqp] = acc[e][i];
            }
    } else {
        const float inv = l == 0.f ? 0.f : 1.f / l;
        T* to = (T*)a.o + vol * a.o_stride + (int64_t)h * a.D * a.tq + qt;
#pragma unroll
        for (int e = 0; e < DB; ++e)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int ch = e * 32 + 8 * (i / 4) + 4 * half + i % 4;
                if (ch < a.D) Elt<T>::st(to + ch * a.tq, acc[e][i] * inv);
            }
        if (a.lse && half == 0)
            a.lse[(int64_t)nh * a.tq + qt] =
                l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * kLn2;
    }
}

// Joins the splits of the forward: thread = query, a slice of the channels each.
template <typename T>
__global__ __launch_bounds__(256) void attn_join_k(AttnArgs a) {
    const int lane = threadIdx.x & 63, sub = threadIdx.x >> 6;
    const int tiles = (int)((a.tq + 63) / 64);
    const int nh = blockIdx.x / tiles;
    const int64_t qt = (int64_t)(blockIdx.x - nh * tiles) * 64 + lane;
    if (qt >= a.tq) return;
    const float* st = a.stat + (int64_t)nh * a.splits * 2 * a.tqp + qt;
    float m = -INFINITY;
    for (int s = 0; s < a.splits; ++s) m = fmaxf(m, st[(int64_t)s * 2 * a.tqp]);
    const float ref = m == -INFINITY ? 0.f : m;
    float l = 0.f;
    for (int s = 0; s < a.splits; ++s)
        l += st[((int64_t)s * 2 + 1) * a.tqp] *
             __builtin_amdgcn_exp2f(st[(int64_t)s * 2 * a.tqp] - ref);
    const float inv = l == 0.f ? 0.f : 1.f / l;
    const int vol = nh / a.heads, h = nh - vol * a.heads;
    T* to = (T*)a.o + vol * a.o_stride + (int64_t)h * a.D * a.tq + qt;
    const float* p = a.part + (int64_t)nh * a.splits * a.D * a.tqp + qt;
    for (int c = sub; c < a.D; c += 4) {
        float v = 0.f;
        for (int s = 0; s < a.splits; ++s)
            v += p[((int64_t)s * a.D + c) * a.tqp] *
                 __builtin_amdgcn_exp2f(st[(int64_t)s * 2 * a.tqp] - ref);
        Elt<T>::st(to + c * a.tq, v * inv);
    }
    if (a.lse && sub == 0)
        a.lse[(int64_t)nh * a.tq + qt] =
            l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * kLn2;
}

// ------------------------------------------------------------------ backward
// dK, dV: a workgroup keeps 128 live keys of one key head, 32 a wave as columns, and
// walks the queries of every head of the group, 32 a turn as rows.
template <typename T, int DB, bool SPLIT>
__global__ __launch_bounds__(256, (DB <= 2 ? 2 : 1)) void attn_dkv_k(AttnArgs a) {
    typedef Mm<T> M;
    typedef typename M::frag frag;
    constexpr int NR = 32 * DB / M::kR, NT = 32 / M::kT, NF = 32 * DB / M::kPer * 32 / 64;
    constexpr int U = NF * 64;
    __shared__ uint4 lds[2][4][U];
    int bid = xcd_remap(blockIdx.x, gridDim.x);
    const int tile = bid % a.tiles;
    bid /= a.tiles;
    const int sp = SPLIT ? bid % a.splits : 0;
    const int kvh = SPLIT ? bid / a.splits : bid;
    const int vol = kvh / a.kv, hk = kvh - vol * a.kv;
    const int grp = a.heads / a.kv;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t live = a.count ? a.count[vol] : a.tk;
    if ((int64_t)tile * 128 >= live) return;
    const int64_t kb = (int64_t)tile * 4 + wave;  // block of 32 keys
    const bool have = kb * 32 < live;             // else packed blocks need not exist

    frag kf[NR], vf[NR];
#pragma unroll
    for (int f = 0; f < NR; ++f) {
        kf[f] = frag{};
        vf[f] = frag{};
        if (have) {
            kf[f] = frag_of<T>(a.kr + ((int64_t)kvh * (a.tkp / 32) + kb) * U, f);
            vf[f] = frag_of<T>(a.vr + ((int64_t)kvh * (a.tkp / 32) + kb) * U, f);
        }
    }
    f32x16 dk[DB], dv[DB];
#pragma unroll
    for (int e = 0; e < DB; ++e)
#pragma unroll
        for (int i = 0; i < 16; ++i) dk[e][i] = dv[e][i] = 0.f;

    // turns: the query blocks of the group's heads one after another
    const int nqb = (int)((a.tq + 31) / 32);
    const int turns = nqb * grp;
    const int per = SPLIT ? (turns + a.splits - 1) / a.splits : turns;
    const int i0 = SPLIT ? (sp * per < turns ? sp * per : turns) : 0;
    const int i1 = i0 + per < turns ? i0 + per : turns;
    Stage<U> s0, s1, s2, s3;
    auto fetch = [&](int i) {
        const int g = i / nqb, b = i - g * nqb;
        const int64_t at = ((int64_t)(vol * a.heads + hk * grp + g) * (a.tqp / 32) + b) * U;
        s0.load(a.qr + at);
        s1.load(a.qt + at);
        s2.load(a.or_ + at);
        s3.load(a.ot + at);
    };
    auto put = [&](int buf) {
        s0.store(lds[buf][0]);
        s1.store(lds[buf][1]);
        s2.store(lds[buf][2]);
        s3.store(lds[buf][3]);
    };
    if (i0 < i1) {
        fetch(i0);
        put(0);
    }
    __syncthreads();
    for (int i = i0; i < i1; ++i) {
        const int buf = (i - i0) & 1;
        const int g = i / nqb, b = i - g * nqb;
        const int64_t row = (int64_t)(vol * a.heads + hk * grp + g) * a.tqp + b * 32 + 4 * (lane >> 5);
        f32x4 ls[4], de[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            ls[r] = *reinterpret_cast<const f32x4*>(a.lse2 + row + 8 * r);
            de[r] = *reinterpret_cast<const f32x4*>(a.delta + row + 8 * r);
        }
        if (i + 1 < i1) fetch(i + 1);
        f32x16 s, dp;
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] = dp[r] = 0.f;
#pragma unroll
        for (int f = 0; f < NR; ++f) {
            s = M::mul(frag_of<T>(lds[buf][0], f), kf[f], s);
            dp = M::mul(frag_of<T>(lds[buf][2], f), vf[f], dp);
        }
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            s[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r], a.c, -ls[r / 4][r % 4]));
            dp[r] = s[r] * (dp[r] - de[r / 4][r % 4]);
        }
#pragma unroll
        for (int w = 0; w < NT; ++w) {
            const frag p = to_frag<T>(s, w), d = to_frag<T>(dp, w);
#pragma unroll
            for (int e = 0; e < DB; ++e) {
                dv[e] = M::mul(frag_of<T>(lds[buf][3], w * DB + e), p, dv[e]);
                dk[e] = M::mul(frag_of<T>(lds[buf][1], w * DB + e), d, dk[e]);
            }
        }
        if (i + 1 < i1) put(buf ^ 1);
        __syncthreads();
    }
    const int64_t j = kb * 32 + (lane & 31);
    if (j >= live) return;
    const int half = lane >> 5;
    if (SPLIT) {
        float* to = a.part + ((int64_t)kvh * a.splits + sp) * 2 * a.D * a.tkp + j;
#pragma unroll
        for (int e = 0; e < DB; ++e)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int ch = e * 32 + 8 * (i / 4) + 4 * half + i % 4;
                if (ch < a.D) {
                    to[ch * a.tkp] = dk[e][i] * a.scale;
                    to[(a.D + ch) * a.tkp] = dv[e][i];
                }
            }
    } else {
        const int64_t tok = a.idx ? a.idx[vol * a.tkp + j] : j;
        T* tk = (T*)a.dk + vol * a.k_stride + (int64_t)hk * a.D * a.tk + tok;
        T* tv = (T*)a.dv + vol * a.v_stride + (int64_t)hk * a.D * a.tk + tok;
#pragma unroll
        for (int e = 0; e < DB; ++e)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int ch = e * 32 + 8 * (i / 4) + 4 * half + i % 4;
                if (ch < a.D) {
                    Elt<T>::st(tk + ch * a.tk, dk[e][i] * a.scale);
                    Elt<T>::st(tv + ch * a.tk, dv[e][i]);
                }
            }
    }
}

// dQ: a workgroup keeps 128 queries of one head, 32 a wave as columns, and walks the
// live keys, 32 a turn as rows.
template <typename T, int DB, bool SPLIT>
__global__ __launch_bounds__(256, (DB <= 2 ? 2 : 1)) void attn_dq_k(AttnArgs a) {
    typedef Mm<T> M;
    typedef typename M::frag frag;
    constexpr int NR = 32 * DB / M::kR, NT = 32 / M::kT, NF = 32 * DB / M::kPer * 32 / 64;
    constexpr int U = NF * 64;
    __shared__ uint4 lds[2][3][U];
    int bid = xcd_remap(blockIdx.x, gridDim.x);
    const int tile = bid % a.tiles;
    bid /= a.tiles;
    const int sp = SPLIT ? bid % a.splits : 0;
    const int nh = SPLIT ? bid / a.splits : bid;
    const int vol = nh / a.heads, h = nh - vol * a.heads;
    const int kvh = vol * a.kv + h / (a.heads / a.kv);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t live = a.count ? a.count[vol] : a.tk;
    const int64_t qb = (int64_t)tile * 4 + wave;
    const bool have = qb * 32 < a.tqp;
    frag qf[NR], of[NR];
#pragma unroll
    for (int f = 0; f < NR; ++f) {
        qf[f] = frag{};
        of[f] = frag{};
        if (have) {
            qf[f] = frag_of<T>(a.qr + ((int64_t)nh * (a.tqp / 32) + qb) * U, f);
            of[f] = frag_of<T>(a.or_ + ((int64_t)nh * (a.tqp / 32) + qb) * U, f);
        }
    }
    const int64_t qt = qb * 32 + (lane & 31);
    const float ls = have ? a.lse2[(int64_t)nh * a.tqp + qt] : INFINITY;
    const float de = have ? a.delta[(int64_t)nh * a.tqp + qt] : 0.f;
    f32x16 dq[DB];
#pragma unroll
    for (int e = 0; e < DB; ++e)
#pragma unroll
        for (int i = 0; i < 16; ++i) dq[e][i] = 0.f;
    int b0, b1;
    split_range(live, 32, SPLIT ? a.splits : 1, sp, b0, b1);
    Stage<U> s0, s1, s2;
    auto fetch = [&](int b) {
        const int64_t at = ((int64_t)kvh * (a.tkp / 32) + b) * U;
        s0.load(a.kr + at);
        s1.load(a.kt + at);
        s2.load(a.vr + at);
    };
    auto put = [&](int buf) {
        s0.store(lds[buf][0]);
        s1.store(lds[buf][1]);
        s2.store(lds[buf][2]);
    };
    if (b0 < b1) {
        fetch(b0);
        put(0);
    }
    __syncthreads();
    for (int b = b0; b < b1; ++b) {
        const int buf = (b - b0) & 1;
        if (b + 1 < b1) fetch(b + 1);
        f32x16 s, dp;
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] = dp[r] = 0.f;
#pragma unroll
        for (int f = 0; f < NR; ++f) {
            s = M::mul(frag_of<T>(lds[buf][0], f), qf[f], s);
            dp = M::mul(frag_of<T>(lds[buf][2], f), of[f], dp);
        }
        // rows behind the last key have K = V = 0 and so give nothing to dq, as
        // long as their P stays finite, which exp(-lse) might not
        const int left = live - (int64_t)b * 32 < 32 ? (int)(live - (int64_t)b * 32) : 32;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            s[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r], a.c, -ls));
            dp[r] = s[r] * (dp[r] - de);
        }
        if (left < 32) {
#pragma unroll
            for (int r = 0; r < 16; ++r)
                if (8 * (r / 4) + 4 * (lane >> 5) + r % 4 >= left) dp[r] = 0.f;
        }
#pragma unroll
        for (int w = 0; w < NT; ++w) {
            const frag d = to_frag<T>(dp, w);
#pragma unroll
            for (int e = 0; e < DB; ++e)
                dq[e] = M::mul(frag_of<T>(lds[buf][1], w * DB + e), d, dq[e]);
        }
        if (b + 1 < b1) put(buf ^ 1);
        __syncthreads();
    }
    if (qt >= a.tq) return;
    const int half = lane >> 5;
    float* tp = SPLIT ? a.part + ((int64_t)nh * a.splits + sp) * a.D * a.tqp + qt : nullptr;
    T* to = (T*)a.dq + vol * a.q_stride + (int64_t)h * a.D * a.tq + qt;
#pragma unroll
    for (int e = 0; e < DB; ++e)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int ch = e * 32 + 8 * (i / 4) + 4 * half + i % 4;
            if (ch >= a.D) continue;
            if (SPLIT) tp[ch * a.tqp] = dq[e][i] * a.scale;
            else Elt<T>::st(to + ch * a.tq, dq[e][i] * a.scale);
        }
}

// Sums of the splits of a backward pass, in a fixed order: [nh][split][rows][tp] ->
// the tensor's channels (rows = D for dq, 2 D for dk and dv).
struct JoinArgs {
    const float* part;
    void *a, *b;               // channels 0 .. D-1 and D .. rows-1
    int64_t a_stride, b_stride, tokens, tp;
    const int *idx, *count;
    int heads, D, rows, splits, tiles;
};
template <typename T>
__global__ __launch_bounds__(256) void attn_sum_k(JoinArgs j) {
    const int lane = threadIdx.x & 63, sub = threadIdx.x >> 6;
    const int tile = blockIdx.x % j.tiles, nh = blockIdx.x / j.tiles;
    const int vol = nh / j.heads, h = nh - vol * j.heads;
    const int64_t t = (int64_t)tile * 64 + lane;
    if (t >= (j.count ? j.count[vol] : j.tokens)) return;
    const int64_t tok = j.idx ? j.idx[vol * j.tp + t] : t;
    const float* p = j.part + (int64_t)nh * j.splits * j.rows * j.tp + t;
    for (int c = sub; c < j.rows; c += 4) {
        float v = 0.f;
        for (int s = 0; s < j.splits; ++s) v += p[((int64_t)s * j.rows + c) * j.tp];
        T* to = c < j.D ? (T*)j.a + vol * j.a_stride + ((int64_t)h * j.D + c) * j.tokens
                        : (T*)j.b + vol * j.b_stride + ((int64_t)h * j.D + c - j.D) * j.tokens;
        Elt<T>::st(to + tok, v);
    }
}

// dK = dV = 0 at masked keys.
template <typename T>
__global__ __launch_bounds__(256) void attn_dead_k(const uint8_t* __restrict__ mask, int64_t tk,
                                                   int tiles, int rows, int64_t k_stride,
                                                   int64_t v_stride, T* dk, T* dv) {
    const int vol = blockIdx.x / tiles;
    const int64_t t = (int64_t)(blockIdx.x - vol * tiles) * 256 + threadIdx.x;
    if (t >= tk || mask[vol * tk + t]) return;
    for (int r = 0; r < rows; ++r) {
        Elt<T>::st(dk + vol * k_stride + r * tk + t, 0.f);
        Elt<T>::st(dv + vol * v_stride + r * tk + t, 0.f);
    }
}

// ------------------------------------------------------------------ host
struct AttnPlan {
    int64_t tqp, tkp;
    int DB, es;
    int fs, ks, qs;  // splits of the forward, of dK/dV, of dQ
    size_t idx, count, kr, kt, vr, vt, qr, qt, orr, ot, lse2, delta, part, fpart, stat, bytes[2];
};

// Ways to split a long walk: until there are two workgroups for each CU, but not
// into pieces of fewer than `least` turns.
static int splits_for(int64_t groups, int64_t turns, int least) {
    const int64_t want = 2 * (int64_t)device_cus();
    int64_t s = ceil_div(want, groups);
    if (s > turns / least) s = turns / least;
    if (s > 256) s = 256;
    return s < 2 ? 1 : (int)s;
}

static AttnPlan attn_plan(const rat3d_attention_desc& d) {
    AttnPlan p = {};
    p.es = d.dtype == RAT3D_BF16 ? 2 : 4;
    p.DB = (d.head_dim + 31) / 32;
    p.tqp = ceil_div(d.tq, 64) * 64;
    p.tkp = ceil_div(d.tk, 64) * 64;
    const int64_t nq = (int64_t)d.n * d.heads, nk = (int64_t)d.n * d.kv_heads;
    const int64_t qtiles = ceil_div(d.tq, 128), ktiles = ceil_div(d.tk, 128);
    p.fs = splits_for(nq * qtiles, p.tkp / 64, 2);
    p.qs = splits_for(nq * qtiles, p.tkp / 32, 4);
    p.ks = splits_for(nk * ktiles, p.tqp / 32 * (d.heads / d.kv_heads), 4);
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t r = at;
        at += (bytes + 255) / 256 * 256;
        return r;
    };
    const size_t qb = (size_t)nq * p.tqp * p.DB * 32 * p.es;
    const size_t kb = (size_t)nk * p.tkp * p.DB * 32 * p.es;
    p.idx = take((size_t)d.n * p.tkp * sizeof(int));
    p.count = take((size_t)d.n * sizeof(int));
    p.kr = take(kb);
    const size_t both = at;
    // forward
    p.vt = take(kb);
    if (p.fs > 1) {
        p.stat = take((size_t)nq * p.fs * 2 * p.tqp * sizeof(float));
        p.fpart = take((size_t)nq * p.fs * d.head_dim * p.tqp * sizeof(float));
    }
    p.bytes[0] = at;
    // backward
    at = both;
    p.kt = take(kb);
    p.vr = take(kb);
    p.qr = take(qb);
    p.qt = take(qb);
    p.orr = take(qb);
    p.ot = take(qb);
    p.lse2 = take((size_t)nq * p.tqp * sizeof(float));
    p.delta = take((size_t)nq * p.tqp * sizeof(float));
    const size_t kp = p.ks > 1 ? (size_t)nk * p.ks * 2 * d.head_dim * p.tkp * sizeof(float) : 0;
    const size_t qp = p.qs > 1 ? (size_t)nq * p.qs * d.head_dim * p.tqp * sizeof(float) : 0;
    p.part = take(kp > qp ? kp : qp);
    p.bytes[1] = at;
    return p;
}

size_t attention_ws_bytes(const rat3d_attention_desc& d, int pass) {
    return attn_plan(d).bytes[pass];
}

bool attention_fits(const rat3d_attention_desc& d) {
    const AttnPlan p = attn_plan(d);
    const int64_t nq = (int64_t)d.n * d.heads;
    // workgroups of the largest launches (each of 256 threads, 2^32 threads a launch)
    return 2 * nq * ceil_div(d.tq, 64) + 2 * (int64_t)d.n * d.kv_heads * ceil_div(d.tk, 64) <
               (1 << 24) &&
           nq * ceil_div(d.tq, 128) * p.fs < (1 << 24) && nq * ceil_div(d.tq, 128) * p.qs < (1 << 24) &&
           (int64_t)d.n * d.kv_heads * ceil_div(d.tk, 128) * p.ks < (1 << 24) &&
           p.tqp / 32 * (d.heads / d.kv_heads) < (1 << 30);
}

static AttnArgs attn_args(const rat3d_attention_desc& d, const AttnPlan& p, char* w) {
    AttnArgs a = {};
    a.tq = d.tq;
    a.tk = d.tk;
    a.tqp = p.tqp;
    a.tkp = p.tkp;
    a.heads = d.heads;
    a.kv = d.kv_heads;
    a.D = d.head_dim;
    a.scale = d.scale > 0.f ? d.scale : 1.f / sqrtf((float)d.head_dim);
    a.c = a.scale * kLog2e;
    a.q_stride = d.q_stride ? d.q_stride : (int64_t)d.heads * d.head_dim * d.tq;
    a.o_stride = d.o_stride ? d.o_stride : (int64_t)d.heads * d.head_dim * d.tq;
    a.k_stride = d.k_stride ? d.k_stride : (int64_t)d.kv_heads * d.head_dim * d.tk;
    a.v_stride = d.v_stride ? d.v_stride : (int64_t)d.kv_heads * d.head_dim * d.tk;
    a.kr = (const uint4*)(w + p.kr);
    return a;
}

static PackJob pack_job(const void* src, int64_t stride, int64_t tokens, int heads, void* r,
                        void* t, const AttnArgs& a, bool keys) {
    PackJob j = {};
    j.src = src;
    j.stride = stride;
    j.tokens = tokens;
    j.heads = heads;
    j.tiles = (int)ceil_div(tokens, kPackTok);
    j.r = r;
    j.t = t;
    if (keys) {
        j.idx = a.idx;
        j.count = a.count;
    }
    return j;
}

static rat3d_status pack_launch(PackArgs& pa, int n, rat3d_dtype dt, hipStream_t st) {
    int64_t blocks = 0;
    for (int i = 0; i < pa.jobs; ++i) {
        pa.job[i].first = (int)blocks;
        blocks += (int64_t)n * pa.job[i].heads * pa.job[i].tiles;
    }
    if (dt == RAT3D_BF16) attn_pack_k<bf16><<<(unsigned)blocks, 256, 0, st>>>(pa);
    else attn_pack_k<float><<<(unsigned)blocks, 256, 0, st>>>(pa);
    RAT3D_LAUNCH_CHECK();
    return RAT3D_OK;
}

static rat3d_status live_keys(const rat3d_attention_desc& d, const AttnPlan& p, char* w,
                              const uint8_t* mask, AttnArgs* a, hipStream_t st) {
    if (!mask) return RAT3D_OK;
    a->idx = (const int*)(w + p.idx);
    a->count = (const int*)(w + p.count);
    ProfScope ps("attn_live", st, 0.0, (double)d.n * d.tk);
    live_keys_k<<<d.n, 1024, 0, st>>>(mask, d.tk, p.tkp, (int*)(w + p.idx), (int*)(w + p.count));
    RAT3D_LAUNCH_CHECK();
    return RAT3D_OK;
}

#define RAT3D_TRY(x)                          \
    do {                                      \
        const rat3d_status s_ = (x);          \
        if (s_ != RAT3D_OK) return s_;        \
    } while (0)

template <typename T, int DB>
static void fwd_launch(const AttnArgs& a, int64_t grid, hipStream_t st) {
    constexpr int KB = sizeof(T) == 2 ? 2 : 1;
    if (a.splits > 1) attn_fwd_k<T, DB, KB, true><<<(unsigned)grid, 256, 0, st>>>(a);
    else attn_fwd_k<T, DB, KB, false><<<(unsigned)grid, 256, 0, st>>>(a);
}
template <typename T, int DB>
static void dkv_launch(const AttnArgs& a, int64_t grid, hipStream_t st) {
    if (a.splits > 1) attn_dkv_k<T, DB, true><<<(unsigned)grid, 256, 0, st>>>(a);
    else attn_dkv_k<T, DB, false><<<(unsigned)grid, 256, 0, st>>>(a);
}
template <typename T, int DB>
static void dq_launch(const AttnArgs& a, int64_t grid, hipStream_t st) {
    if (a.splits > 1) attn_dq_k<T, DB, true><<<(unsigned)grid, 256, 0, st>>>(a);
    else attn_dq_k<T, DB, false><<<(unsigned)grid, 256, 0, st>>>(a);
}
#define RAT3D_ATTN(F, dt, DB, ...)                                  \
    do {                                                            \
        if ((dt) == RAT3D_BF16) {                                   \
            if ((DB) == 1) F<bf16, 1>(__VA_ARGS__);                 \
            else if ((DB) == 2) F<bf16, 2>(__VA_ARGS__);            \
            else if ((DB) == 3) F<bf16, 3>(__VA_ARGS__);            \
            else F<bf16, 4>(__VA_ARGS__);                           \
        } else {                                                    \
            if ((DB) == 1) F<float, 1>(__VA_ARGS__);                \
            else if ((DB) == 2) F<float, 2>(__VA_ARGS__);           \
            else if ((DB) == 3) F<float, 3>(__VA_ARGS__);           \
            else F<float, 4>(__VA_ARGS__);                          \
        }                                                           \
        RAT3D_LAUNCH_CHECK();                                       \
    } while (0)

rat3d_status attention_fwd(const rat3d_attention_desc& d, const void* q, const void* k,
                           const void* v, const uint8_t* mask, void* o, float* lse, void* ws,
                           hipStream_t st) {
    const AttnPlan p = attn_plan(d);
    char* w = (char*)ws;
    AttnArgs a = attn_args(d, p, w);
    a.q = q;
    a.o = o;
    a.lse = lse;
    a.vt = (const uint4*)(w + p.vt);
    a.stat = (float*)(w + p.stat);
    a.part = (float*)(w + p.fpart);
    RAT3D_TRY(live_keys(d, p, w, mask, &a, st));
    const double nq = (double)d.n * d.heads, nk = (double)d.n * d.kv_heads;
    {
        ProfScope ps("attn_pack", st, 0.0, 4.0 * nk * d.tk * d.head_dim * p.es);
        PackArgs pa = {};
        pa.D = d.head_dim;
        pa.DB = p.DB;
        pa.jobs = 2;
        pa.job[0] = pack_job(k, a.k_stride, d.tk, d.kv_heads, w + p.kr, nullptr, a, true);
        pa.job[1] = pack_job(v, a.v_stride, d.tk, d.kv_heads, nullptr, w + p.vt, a, true);
        RAT3D_TRY(pack_launch(pa, d.n, d.dtype, st));
    }
    {
        ProfScope ps("attn_fwd", st, 4.0 * nq * d.tq * d.tk * d.head_dim, 0.0);
        a.splits = p.fs;
        a.tiles = (int)ceil_div(d.tq, 128);
        const int64_t grid = (int64_t)d.n * d.heads * a.tiles * a.splits;
        RAT3D_ATTN(fwd_launch, d.dtype, p.DB, a, grid, st);
    }
    if (p.fs > 1) {
        ProfScope ps("attn_join", st, 0.0, nq * d.tq * d.head_dim * (4.0 * p.fs + p.es));
        const unsigned grid = (unsigned)((int64_t)d.n * d.heads * ceil_div(d.tq, 64));
        if (d.dtype == RAT3D_BF16) attn_join_k<bf16><<<grid, 256, 0, st>>>(a);
        else attn_join_k<float><<<grid, 256, 0, st>>>(a);
        RAT3D_LAUNCH_CHECK();
    }
    return RAT3D_OK;
}

rat3d_status attention_bwd(const rat3d_attention_desc& d, const void* dout, const void* q,
                           const void* k, const void* v, const uint8_t* mask, const void* o,
                           const float* lse, void* dq, void* dk, void* dv, void* ws,
                           hipStream_t st) {
    const AttnPlan p = attn_plan(d);
    char* w = (char*)ws;
    AttnArgs a = attn_args(d, p, w);
    a.kt = (const uint4*)(w + p.kt);
    a.vr = (const uint4*)(w + p.vr);
    a.qr = (const uint4*)(w + p.qr);
    a.qt = (const uint4*)(w + p.qt);
    a.or_ = (const uint4*)(w + p.orr);
    a.ot = (const uint4*)(w + p.ot);
    a.lse2 = (const float*)(w + p.lse2);
    a.delta = (const float*)(w + p.delta);
    a.part = (float*)(w + p.part);
    a.dq = dq;
    a.dk = dk;
    a.dv = dv;
    RAT3D_TRY(live_keys(d, p, w, mask, &a, st));
    const double nq = (double)d.n * d.heads, nk = (double)d.n * d.kv_heads;
    const double one = 2.0 * nq * d.tq * d.tk * d.head_dim;
    {
        ProfScope ps("attn_pack", st, 0.0,
                     (5.0 * nk * d.tk + 7.0 * nq * d.tq) * d.head_dim * p.es);
        PackArgs pa = {};
        pa.D = d.head_dim;
        pa.DB = p.DB;
        pa.jobs = 4;
        pa.job[0] = pack_job(k, a.k_stride, d.tk, d.kv_heads, w + p.kr, w + p.kt, a, true);
        pa.job[1] = pack_job(v, a.v_stride, d.tk, d.kv_heads, w + p.vr, nullptr, a, true);
        pa.job[2] = pack_job(q, a.q_stride, d.tq, d.heads, w + p.qr, w + p.qt, a, false);
        pa.job[3] = pack_job(dout, a.o_stride, d.tq, d.heads, w + p.orr, w + p.ot, a, false);
        pa.job[3].other = o;
        pa.job[3].lse = lse;
        pa.job[3].lse2 = (float*)(w + p.lse2);
        pa.job[3].delta = (float*)(w + p.delta);
        RAT3D_TRY(pack_launch(pa, d.n, d.dtype, st));
    }
    const bool bf = d.dtype == RAT3D_BF16;
    if (mask) {
        ProfScope ps("attn_dead", st, 0.0, nk * d.tk * d.head_dim * p.es);
        const int tiles = (int)ceil_div(d.tk, 256);
        const int rows = d.kv_heads * d.head_dim;
        if (bf)
            attn_dead_k<bf16><<<(unsigned)(d.n * tiles), 256, 0, st>>>(
                mask, d.tk, tiles, rows, a.k_stride, a.v_stride, (bf16*)dk, (bf16*)dv);
        else
            attn_dead_k<float><<<(unsigned)(d.n * tiles), 256, 0, st>>>(
                mask, d.tk, tiles, rows, a.k_stride, a.v_stride, (float*)dk, (float*)dv);
        RAT3D_LAUNCH_CHECK();
    }
    {
        ProfScope ps("attn_dkv", st, 3.0 * one, 0.0);
        a.splits = p.ks;
        a.tiles = (int)ceil_div(d.tk, 128);
        const int64_t grid = (int64_t)d.n * d.kv_heads * a.tiles * a.splits;
        RAT3D_ATTN(dkv_launch, d.dtype, p.DB, a, grid, st);
        if (p.ks > 1) {
            JoinArgs j = {a.part, dk, dv, a.k_stride, a.v_stride, d.tk, p.tkp, a.idx, a.count,
                          d.kv_heads, d.head_dim, 2 * d.head_dim, p.ks, (int)ceil_div(d.tk, 64)};
            const unsigned g = (unsigned)((int64_t)d.n * d.kv_heads * j.tiles);
            if (bf) attn_sum_k<bf16><<<g, 256, 0, st>>>(j);
            else attn_sum_k<float><<<g, 256, 0, st>>>(j);
            RAT3D_LAUNCH_CHECK();
        }
    }
    {
        ProfScope ps("attn_dq", st, 2.0 * one, 0.0);
        a.splits = p.qs;
        a.tiles = (int)ceil_div(d.tq, 128);
        const int64_t grid = (int64_t)d.n * d.heads * a.tiles * a.splits;
        RAT3D_ATTN(dq_launch, d.dtype, p.DB, a, grid, st);
        if (p.qs > 1) {
            JoinArgs j = {a.part, dq, dq, a.q_stride, a.q_stride, d.tq, p.tqp, nullptr, nullptr,
                          d.heads, d.head_dim, d.head_dim, p.qs, (int)ceil_div(d.tq, 64)};
            const unsigned g = (unsigned)((int64_t)d.n * d.heads * j.tiles);
            if (bf) attn_sum_k<bf16><<<g, 256, 0, st>>>(j);
            else attn_sum_k<float><<<g, 256, 0, st>>>(j);
            RAT3D_LAUNCH_CHECK();
        }
    }
    return RAT3D_OK;
}

}  // namespace rat3d
