// Attention over the tokens of channel-first maps, forward and backward.
//
// Forward, for each query: one pass over the keys with the running maximum m and
// sum l of the softmax; o = sum_j exp(s_j - m) v_j / l.  Backward, with the
// logarithm of the sum (lse) and D_i = do_i . o_i:
//   P = exp(S - lse), dV = P^T dO, dS = P (dO V^T - D), dQ = scale dS K,
//   dK = scale dS^T Q,
// in two walks, one that keeps keys and goes over the queries (dK, dV), one that
// keeps queries and goes over the keys (dQ): S is formed three times in a training
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
// 64 (the backward's queries with the last query, see attn_pack_k).  Masked keys are left out: the live ones move up (an index list, made from
// the mask), so masked voxels cost nothing and what they hold is never read.
#include <math.h>

#include <type_traits>

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
    // The second operands that add, from a fragment of row constants, the first
    // (slots 0 to 2) or the second (slots 3 to 5) constant of each row to a product.
    __device__ __forceinline__ static frag pick(int second, int half) {
        frag f;
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = (__bf16)(half == 0 && j / 3 == second ? 1.f : 0.f);
        return f;
    }
    __device__ __forceinline__ static f32x16 add_row(frag a, frag b, f32x16 c) { return mul(a, b, c); }
    // a row's two constants as a lane of such a fragment: three bfloat16 terms each,
    // which hold a float32 value to its last bit or next to it
    __device__ __forceinline__ static u32x4 rows(float x, float y, int half) {
        if (half) return u32x4{0, 0, 0, 0};
        bf16 v[8] = {};
#pragma unroll
        for (int j = 0; j < 3; ++j) {
            v[j] = f2bf(x);
            x -= bf2f(v[j]);
            v[3 + j] = f2bf(y);
            y -= bf2f(v[3 + j]);
        }
        u32x4 u;
        __builtin_memcpy(&u, v, 16);
        return u;
    }
    __device__ __forceinline__ static f32x16 mul(frag a, frag b, f32x16 c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
    }
};
template <> struct Mm<float> {
    typedef f32x4 frag;
    static constexpr int kR = 8, kT = 8, kPer = 4;
    __device__ __forceinline__ static frag pick(int second, int half) {
        return frag{half == second ? 1.f : 0.f, 0.f, 0.f, 0.f};
    }
    __device__ __forceinline__ static f32x16 add_row(frag a, frag b, f32x16 c) {
        return __builtin_amdgcn_mfma_f32_32x32x2f32(a[0], b[0], c, 0, 0, 0);
    }
    __device__ __forceinline__ static u32x4 rows(float x, float y, int half) {
        return u32x4{__float_as_uint(half ? y : x), 0, 0, 0};
    }
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
// takes them; the sums over them stay in float32.  In bfloat16 this is a second rounding
// beside the result's own: sqrt(2) times its error (norm-wise 1.7e-3 -> 2.4e-3).  Unrounded
// they would need the float32 instructions, at a sixteenth of the rate, or a second
// product for what the rounding leaves.
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

// The same within a workgroup of 256 that needs only the live tokens t0 .. t0 + 63: their
// places go to `pick`, and the number of all live tokens is returned.  Each thread looks
// at kLook neighbouring tokens, so one scan over the threads finds every rank.
constexpr int kLook = 8;
struct __attribute__((packed, aligned(1))) MaskBytes {
    uint8_t b[kLook];
};
__device__ __forceinline__ int live_tokens(const uint8_t* __restrict__ m, int T, int t0,
                                           int* pick, int* wsum) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int at = (int)threadIdx.x * kLook;
    uint32_t on = 0;  // bit j: token at + j is live
    if (T >= kLook) {
        // the last tokens are read with those before them
        const int from = at < T - kLook ? at : T - kLook;
        const MaskBytes u = *reinterpret_cast<const MaskBytes*>(m + from);
#pragma unroll
        for (int j = 0; j < kLook; ++j) on |= (u.b[j] != 0 ? 1u : 0u) << j;
        on = at - from < kLook ? on >> (at - from) : 0;
    } else {
#pragma unroll
        for (int j = 0; j < kLook; ++j)
            on |= (at + j < T && m[at + j < T ? at + j : T - 1] != 0 ? 1u : 0u) << j;
    }
    const int mine = __builtin_popcount(on);
    int incl = mine;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int o = __shfl_up(incl, d);
        if (lane >= d) incl += o;
    }
    if (lane == 63) wsum[wave] = incl;
    __syncthreads();
    int rank = incl - mine, all = 0;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        if (w < wave) rank += wsum[w];
        all += wsum[w];
    }
    if (rank < t0 + 64 && rank + mine > t0)
        for (uint32_t b = on; b; b &= b - 1, ++rank)
            if (rank >= t0 && rank < t0 + 64) pick[rank - t0] = at + __builtin_ctz(b);
    __syncthreads();
    return all;
}

// ------------------------------------------------------------------ packing
struct PackJob {
    const void* src;     // [n][heads * D][tokens], volumes `stride` apart
    const void* other;   // o, where src is dout: D = sum over channels of src * other; o as
                         // stored, whose rounding is in dq and dk by sqrt(sum p^2) of what
                         // that of the score gradients gives (some ten live keys: 2.7e-3 in all)
    const float* lse;
    u32x4* rec;          // records of 32 tokens, `units` 16-byte units each:
    int units, r, t, x;  // where forms R and T and the row constants lie, or -1
    int again;           // behind the last token stands: 0, zeros; 1, that token again
    float* lse2;         // lse in units of log 2; +infinity behind the last query and for
                         // a query without keys: its probabilities are then 0
    float* delta;        // D, padded with 0
    int* idx;            // live tokens, or null: all are
    int* count;
    int scan;            // not 0: the job finds them from the mask; 2: and writes them down
    const uint8_t* mask; // what lies at masked tokens of `zero` (a gradient of src's layout,
    void* zero;          // or null) becomes 0
    int64_t stride, tokens;
    int heads, tiles;    // tiles of 64 tokens
    int first;           // first workgroup of the job
};
struct PackArgs {
    PackJob job[4];
    int jobs, D;
    float scale;
};

constexpr int kPackTok = 64;

// One workgroup: 64 tokens of one head of one volume, through LDS.
template <typename T, int DB>
__global__ __launch_bounds__(256) void attn_pack_k(PackArgs a) {
    typedef Mm<T> M;
    constexpr int Dp = 32 * DB;
    constexpr int ROW = kPackTok + (sizeof(T) == 2 ? 2 : 1);  // odd in banks: columns spread
    __shared__ T tile[Dp * ROW];
    __shared__ float part[4][kPackTok];
    __shared__ int pick[kPackTok], wsum[4];
    int ji = 0;
    while (ji + 1 < a.jobs && (int)blockIdx.x >= a.job[ji + 1].first) ++ji;
    const PackJob& J = a.job[ji];
    const int b = (int)blockIdx.x - J.first;
    const int tl = b % J.tiles, nh = b / J.tiles;
    const int vol = nh / J.heads, h = nh - vol * J.heads;
    const int64_t t0 = (int64_t)tl * kPackTok;
    const int col = threadIdx.x & 63, sub = threadIdx.x >> 6;
    const int64_t live = J.scan ? live_tokens(J.mask + vol * J.tokens, (int)J.tokens, (int)t0,
                                              pick, wsum)
                         : J.count ? J.count[vol]
                                   : J.tokens;
    if (J.scan == 2 && h == 0) {
        if (tl == 0 && threadIdx.x == 0) J.count[vol] = (int)live;
        if (sub == 0 && t0 + col < live)
            J.idx[vol * (int64_t)J.tiles * kPackTok + t0 + col] = pick[col];
    }
    if (J.zero && t0 + col < J.tokens && !J.mask[vol * J.tokens + t0 + col]) {
        T* z = (T*)J.zero + vol * J.stride + (int64_t)h * a.D * J.tokens + t0 + col;
        for (int c = sub; c < a.D; c += 4) Elt<T>::st(z + c * J.tokens, 0.f);
    }
    if (J.count && t0 >= live) return;  // never read: kernels stop at the live keys
    const bool in = t0 + col < live;
    const int64_t tok = !in      ? (J.again ? J.tokens - 1 : 0)
                        : J.scan ? pick[col]
                        : J.idx  ? J.idx[vol * (int64_t)J.tiles * kPackTok + t0 + col]
                                 : t0 + col;
    const int64_t base = vol * J.stride + (int64_t)h * a.D * J.tokens + tok;
    const T* src = (const T*)J.src + base;
    const T* oth = J.other ? (const T*)J.other + base : nullptr;
    float d = 0.f;
    // channels that do not count as 0; once for all, a condition an element costs 1 to 2 us
    const int channels = in || J.again ? a.D : 0;
    // all of a thread's loads are issued before the first is used; behind the last
    // channel it is read again, at a token that is there, and counts as 0
    T v[8 * DB], o[8 * DB];
#pragma unroll
    for (int i = 0; i < 8 * DB; ++i) {
        const int c = sub + 4 * i < a.D ? sub + 4 * i : a.D - 1;
        v[i] = src[c * J.tokens];
        if (oth) o[i] = oth[c * J.tokens];
    }
#pragma unroll
    for (int i = 0; i < 8 * DB; ++i) {
        const bool on = sub + 4 * i < channels;
        if (!on) v[i] = Elt<T>::to_bits(0.f);
        if (oth && on) d += Elt<T>::from_bits(v[i]) * Elt<T>::from_bits(o[i]);
        tile[(sub + 4 * i) * ROW + col] = v[i];
    }
    part[sub][col] = d;
    __syncthreads();
    const int64_t blk0 = ((int64_t)nh * J.tiles + tl) * 2;  // record of the first token
    if (J.delta && threadIdx.x < 2 * kPackTok) {
        const int tk = threadIdx.x & 63, half = threadIdx.x >> 6;
        const bool on = t0 + tk < live;
        const float d = (part[0][tk] + part[1][tk]) + (part[2][tk] + part[3][tk]);
        const float e = on ? J.lse[(int64_t)nh * J.tokens + t0 + tk] : -INFINITY;
        if (half == 0) {
            const int64_t at = (int64_t)nh * J.tiles * kPackTok + t0 + tk;
            J.delta[at] = d;
            J.lse2[at] = e == -INFINITY ? INFINITY : e * kLog2e;
        }
        // Row constants of the products with these rows: -lse in units of the scores,
        // and -D.  Behind the last query, and where a query has no key, a number so low
        // that its probabilities are 0 at any score, finite because it is multiplied by 0
        // elsewhere.  What stands behind the last query is that query again (`again`):
        // zeros would score 0 * infinity at a key that holds one, NaN, where every
        // query has -infinity and so the probability 0.
        J.rec[(blk0 + (tk >> 5)) * J.units + J.x + half * 32 + (tk & 31)] =
            M::rows(e == -INFINITY ? -3e38f : -e / a.scale, -d, half);
    }
    // fragments: 2 blocks of 32 tokens x Dp, 16 bytes a lane
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int per = Dp / M::kR;  // fragments of one block and form
    for (int f = wave; f < 2 * per; f += 4) {
        const int blk = f / per, g = f % per;
        u32x4* to = J.rec + (blk0 + blk) * J.units + g * 64 + lane;
        if (J.r >= 0) {
            const int ch = g * M::kR + (lane >> 5) * M::kPer;
            T v[M::kPer];
#pragma unroll
            for (int j = 0; j < M::kPer; ++j) v[j] = tile[(ch + j) * ROW + blk * 32 + (lane & 31)];
            u32x4 u;
            __builtin_memcpy(&u, v, 16);
            to[J.r] = u;
        }
        if (J.t >= 0) {
            const int w = g / DB, e = g % DB;
            const int ch = e * 32 + (lane & 31);
            T v[M::kPer];
#pragma unroll
            for (int j = 0; j < M::kPer; ++j)
                v[j] = tile[ch * ROW + blk * 32 + w * M::kT + 8 * (j / 4) + 4 * (lane >> 5) + j % 4];
            u32x4 u;
            __builtin_memcpy(&u, v, 16);
            to[J.t] = u;
        }
    }
}

// ------------------------------------------------------------------ shared pieces
struct AttnArgs {
    const void* q;  // forward only: queries as given
    void* o;
    float* lse;
    const u32x4 *kv_rec, *q_rec;  // records of 32 keys, of 32 queries
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
// multiplied.  What is left behind the last 256 is copied by several threads alike, so
// that no branch divides a turn.
template <int U> struct Stage {
    static constexpr int N = (U + 255) / 256, kRest = U % 256 ? U % 256 : 256;
    u32x4 v[N];
    __device__ __forceinline__ static int at(int i) {
        return i * 256 + (i + 1 < N ? (int)threadIdx.x : (int)threadIdx.x % kRest);
    }
    __device__ __forceinline__ void load(const u32x4* __restrict__ p) {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = p[at(i)];
    }
    __device__ __forceinline__ void store(u32x4* s) const {
#pragma unroll
        for (int i = 0; i < N; ++i) s[at(i)] = v[i];
    }
    __device__ __forceinline__ void store(u32x4* s, int i) const { s[at(i)] = v[i]; }
};

// The same in two halves, one after the other through the same registers.
template <int U> struct StageHalves {
    static constexpr int N = (U + 255) / 256, kFirst = (N + 1) / 2;
    u32x4 v[kFirst];
    template <int H> __device__ __forceinline__ void load(const u32x4* __restrict__ p) {
#pragma unroll
        for (int i = 0; i < (H ? N - kFirst : kFirst); ++i) v[i] = p[Stage<U>::at(H * kFirst + i)];
    }
    template <int H> __device__ __forceinline__ void store(u32x4* s) const {
#pragma unroll
        for (int i = 0; i < (H ? N - kFirst : kFirst); ++i) s[Stage<U>::at(H * kFirst + i)] = v[i];
    }
};

template <typename T>
__device__ __forceinline__ typename Mm<T>::frag frag_of(const u32x4* s, int f) {
    return __builtin_bit_cast(typename Mm<T>::frag, s[f * 64 + (threadIdx.x & 63)]);
}

// 32 tokens of a channel-first tensor as fragments of form R (second operand).  All
// loads are issued before one is used: what is behind the last channel is read from it
// again and counts as 0, and a token behind the last from the last (p: the tensor's
// first channel at this lane's token, or at the last one).
template <typename T, int NF>
__device__ __forceinline__ void load_cols(const T* __restrict__ p, int64_t row, int D, bool in,
                                          typename Mm<T>::frag (&f)[NF]) {
    typedef Mm<T> M;
    const int half = (threadIdx.x & 63) >> 5;
    T v[NF][M::kPer];
#pragma unroll
    for (int i = 0; i < NF; ++i)
#pragma unroll
        for (int j = 0; j < M::kPer; ++j) {
            const int ch = i * M::kR + half * M::kPer + j;
            v[i][j] = p[(ch < D ? ch : D - 1) * row];
        }
#pragma unroll
    for (int i = 0; i < NF; ++i) {
#pragma unroll
        for (int j = 0; j < M::kPer; ++j)
            if (!in || i * M::kR + half * M::kPer + j >= D) v[i][j] = Elt<T>::to_bits(0.f);
        __builtin_memcpy(&f[i], v[i], 16);
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
// The result of a lane's query qt leaves: o and lse, or a split's reference, sum and
// values.  l is the sum over the rows of this lane; the lane 32 away has the others.
template <typename T, int DB, bool SPLIT>
__device__ __forceinline__ void fwd_store(const AttnArgs& a, int nh, int sp, int64_t qt, float m,
                                          float l, const f32x16 (&acc)[DB]) {
    const int half = (threadIdx.x & 63) >> 5;
    float la, lb;
    halves(l, la, lb);
    l = la + lb;
    if (qt >= a.tq) return;
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
        const int vol = nh / a.heads, h = nh - vol * a.heads;
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

// A workgroup: 128 queries of one head, 32 a wave as columns; KB x 32 keys a turn.
template <typename T, int DB, int KB, bool SPLIT>
__global__ __launch_bounds__(256, (sizeof(T) * DB < 16 ? 2 : 1)) void attn_fwd_k(AttnArgs a) {
    typedef Mm<T> M;
    typedef typename M::frag frag;
    constexpr int NR = 32 * DB / M::kR;      // fragments of 32 tokens, form R
    constexpr int NT = 32 / M::kT;           // contraction steps of 32 tokens, form T
    constexpr int NF = 32 * DB / M::kPer * 32 / 64;  // fragments of 32 tokens (either form)
    constexpr int U = 2 * NF * 64;           // units of a record: K in form R, V in form T
    __shared__ u32x4 lds[2][KB * U];
    int bid = xcd_remap(blockIdx.x, gridDim.x);
    const int tile = bid % a.tiles;
    bid /= a.tiles;
    const int sp = SPLIT ? bid % a.splits : 0;
    const int nh = SPLIT ? bid / a.splits : bid;
    const int vol = nh / a.heads, h = nh - vol * a.heads;
    const int kvh = vol * a.kv + h / (a.heads / a.kv);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t live = a.count ? a.count[vol] : a.tk;
    const int64_t qt = ((int64_t)tile * 4 + wave) * 32 + (lane & 31);

    frag qf[NR];
    load_cols<T, NR>((const T*)a.q + vol * a.q_stride + (int64_t)h * a.D * a.tq +
                         (qt < a.tq ? qt : a.tq - 1),
                     a.tq, a.D, qt < a.tq, qf);
    f32x16 acc[DB];
#pragma unroll
    for (int e = 0; e < DB; ++e)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[e][i] = 0.f;
    float m = -INFINITY, l4[4] = {0.f, 0.f, 0.f, 0.f};  // the sum, of this lane's rows

    int b0, b1;
    split_range(live, 32 * KB, SPLIT ? a.splits : 1, sp, b0, b1);
    const u32x4* rec = a.kv_rec + ((int64_t)kvh * (a.tkp / 32) + (int64_t)b0 * KB) * U;
    Stage<KB * U> next;
    if (b0 < b1) {
        next.load(rec);
        next.store(lds[0]);
    }
    __syncthreads();
    for (int b = b0; b < b1; ++b) {
        const int buf = (b - b0) & 1;
        if (b + 1 < b1) {
            rec += KB * U;
            next.load(rec);
        }
        f32x16 s[KB];
#pragma unroll
        for (int k = 0; k < KB; ++k) {
#pragma unroll
            for (int i = 0; i < 16; ++i) s[k][i] = 0.f;
#pragma unroll
            for (int f = 0; f < NR; ++f) s[k] = M::mul(frag_of<T>(lds[buf] + k * U, f), qf[f], s[k]);
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
#pragma unroll
            for (int i = 0; i < 4; ++i) l4[i] *= f;
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
                l4[i % 4] += s[k][i];
            }
#pragma unroll
            for (int w = 0; w < NT; ++w) {
                const frag p = to_frag<T>(s[k], w);
#pragma unroll
                for (int e = 0; e < DB; ++e)
                    acc[e] = M::mul(frag_of<T>(lds[buf] + k * U, NF + w * DB + e), p, acc[e]);
            }
        }
        if (b + 1 < b1) next.store(lds[buf ^ 1]);
        __syncthreads();
    }
    fwd_store<T, DB, SPLIT>(a, nh, sp, qt, m, (l4[0] + l4[1]) + (l4[2] + l4[3]), acc);
}

// Joins the splits of the forward: a workgroup takes 64 queries and 8 channels.
template <typename T>
__global__ __launch_bounds__(256) void attn_join_k(AttnArgs a) {
    const int lane = threadIdx.x & 63, sub = threadIdx.x >> 6;
    const int tiles = (int)((a.tq + 63) / 64), groups = (a.D + 7) / 8;
    int b = blockIdx.x;
    const int tile = b % tiles;
    b /= tiles;
    const int c0 = b % groups * 8, nh = b / groups;
    const int64_t qt = (int64_t)tile * 64 + lane;
    if (qt >= a.tq) return;
    const float* st = a.stat + (int64_t)nh * a.splits * 2 * a.tqp + qt;
    const float* p = a.part + (int64_t)nh * a.splits * a.D * a.tqp + qt;
    const int c1 = c0 + sub, c2 = c1 + 4;
    const int64_t d1 = (int64_t)(c1 < a.D ? c1 : a.D - 1) * a.tqp;
    const int64_t d2 = (int64_t)(c2 < a.D ? c2 : a.D - 1) * a.tqp;
    float m = -INFINITY, l = 0.f, v1 = 0.f, v2 = 0.f;
    for (int s0 = 0; s0 < a.splits; s0 += 8) {  // eight splits' loads in flight
        float ms[8], ls[8], x1[8], x2[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int64_t s = s0 + i < a.splits ? s0 + i : a.splits - 1;
            ms[i] = st[s * 2 * a.tqp];
            ls[i] = st[(s * 2 + 1) * a.tqp];
            x1[i] = p[s * a.D * a.tqp + d1];
            x2[i] = p[s * a.D * a.tqp + d2];
        }
        float to = m;
#pragma unroll
        for (int i = 0; i < 8; ++i) to = fmaxf(to, ms[i]);
        const float ref = to == -INFINITY ? 0.f : to;
        const float f = __builtin_amdgcn_exp2f(m - ref);
        m = to;
        l *= f;
        v1 *= f;
        v2 *= f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (s0 + i >= a.splits) break;
            const float w = __builtin_amdgcn_exp2f(ms[i] - ref);
            l += ls[i] * w;
            v1 += x1[i] * w;
            v2 += x2[i] * w;
        }
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;
    const int vol = nh / a.heads, h = nh - vol * a.heads;
    T* to = (T*)a.o + vol * a.o_stride + (int64_t)h * a.D * a.tq + qt;
    if (c1 < a.D) Elt<T>::st(to + c1 * a.tq, v1 * inv);
    if (c2 < a.D) Elt<T>::st(to + c2 * a.tq, v2 * inv);
    if (a.lse && c0 + sub == 0)
        a.lse[(int64_t)nh * a.tq + qt] =
            l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * kLn2;
}

// ------------------------------------------------------------------ few rows
// A key head with few query rows (heads of its group times query tokens): read-out
// tokens.  The keys and values are read once, as they lie: the scores of
// neighbouring keys by neighbouring lanes (a channel's row is contiguous), then, with
// the probabilities in registers, the sums over a channel's row of values.  4 ROWS
// operations for each element read: bound by HBM.  A workgroup takes one piece of
// 256 VEC keys and up to four rows (neighbouring workgroups take a piece's other rows,
// and find it in their cache); its part of the softmax (maximum, sum, unnormalised
// values) is joined with the others' by attn_few_join_k.
struct FewArgs {
    const void *q, *k, *v;
    const uint8_t* mask;
    void* o;
    float* lse;
    float* part;  // [volume, key head][piece][group][row][2 + D]: maximum, sum, values
    int64_t tq, tk, q_stride, k_stride, v_stride, o_stride;
    int heads, kv, D, pieces, rows, groups;  // groups of rows
    float c;
};

template <typename T, int VEC> struct __attribute__((packed, aligned(sizeof(T)))) Keys {
    T v[VEC];
};
// VEC keys of a row from key t on; keys that are off (bit i of on is 0) count as 0,
// whatever lies there.  MODE 0: all are on; 1: all are inside the row; 2: some may lie
// behind its last key, which is read instead.  No branch: the loads of many channels
// are in flight together.
template <typename T, int VEC, int MODE>
__device__ __forceinline__ void ld_keys(const T* row, int64_t t, int64_t tk, uint32_t on,
                                        float (&o)[VEC]) {
    if (MODE < 2) {
        const Keys<T, VEC> u = *reinterpret_cast<const Keys<T, VEC>*>(row + t);
#pragma unroll
        for (int j = 0; j < VEC; ++j)
            o[j] = MODE == 0 || (on >> j & 1) ? Elt<T>::from_bits(u.v[j]) : 0.f;
    } else {
        T u[VEC];
#pragma unroll
        for (int j = 0; j < VEC; ++j) u[j] = row[t + j < tk ? t + j : tk - 1];
#pragma unroll
        for (int j = 0; j < VEC; ++j) o[j] = on >> j & 1 ? Elt<T>::from_bits(u[j]) : 0.f;
    }
}

template <typename T, int ROWS, int VEC>
__global__ __launch_bounds__(256, (ROWS == 4 && VEC == 8 ? 2 : 4)) void attn_few_k(FewArgs a) {
    __shared__ float qs[128][ROWS];
    __shared__ float ps[ROWS][256 * VEC];
    __shared__ uint32_t ons[256];
    __shared__ float red[2][4][ROWS];
    const int group = blockIdx.x % a.groups, pk = blockIdx.x / a.groups;
    const int piece = pk % a.pieces, kvh = pk / a.pieces;
    const int vol = kvh / a.kv, hk = kvh - vol * a.kv, grp = a.heads / a.kv;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t t0 = (int64_t)piece * 256 * VEC;
    for (int i = tid; i < a.D * ROWS; i += 256) {
        // row: head row / tq of the key head's group, token row % tq
        const int r = i % ROWS, ch = i / ROWS, row = group * ROWS + r;
        const int h = hk * grp + row / (int)a.tq, tok = row % (int)a.tq;
        qs[ch][r] = row < a.rows ? Elt<T>::ld((const T*)a.q + vol * a.q_stride +
                                            ((int64_t)h * a.D + ch) * a.tq + tok) * a.c
                               : 0.f;
    }
    const int64_t t = t0 + tid * VEC;
    uint32_t on = 0;
#pragma unroll
    for (int j = 0; j < VEC; ++j)
        on |= (t + j < a.tk && (!a.mask || a.mask[vol * a.tk + t + j]) ? 1u : 0u) << j;
    ons[tid] = on;
    const bool inside = t0 + 256 * VEC <= a.tk;  // the whole piece
    __syncthreads();

    float s[ROWS][VEC];
#pragma unroll
    for (int r = 0; r < ROWS; ++r)
#pragma unroll
        for (int j = 0; j < VEC; ++j) s[r][j] = 0.f;
    const T* kp = (const T*)a.k + vol * a.k_stride + (int64_t)hk * a.D * a.tk;
    auto scores = [&](auto mode) {
        // channels whose loads are in flight together
        constexpr int SC = VEC <= 2 ? 16 : decltype(mode)::value == 2 ? 2 : 8;
#pragma unroll 1
        for (int c0 = 0; c0 < a.D; c0 += SC) {
            // behind the last channel it is read again and not used
            float x[SC][VEC];
#pragma unroll
            for (int i = 0; i < SC; ++i) {
                const int ch = c0 + i < a.D ? c0 + i : a.D - 1;
                ld_keys<T, VEC, decltype(mode)::value>(kp + ch * a.tk, t, a.tk, on, x[i]);
            }
#pragma unroll
            for (int i = 0; i < SC; ++i) {
                if (c0 + i >= a.D) break;
#pragma unroll
                for (int r = 0; r < ROWS; ++r) {
                    const float q = qs[c0 + i][r];
#pragma unroll
                    for (int j = 0; j < VEC; ++j) s[r][j] = __builtin_fmaf(q, x[i][j], s[r][j]);
                }
            }
        }
    };
    if (__all(on == (1u << VEC) - 1)) scores(std::integral_constant<int, 0>{});
    else if (inside) scores(std::integral_constant<int, 1>{});
    else scores(std::integral_constant<int, 2>{});

    float m[ROWS], l[ROWS];
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        m[r] = -INFINITY;
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
            if (!(on >> j & 1)) s[r][j] = -INFINITY;
            m[r] = fmaxf(m[r], s[r][j]);
        }
#pragma unroll
        for (int d = 32; d >= 1; d >>= 1) m[r] = fmaxf(m[r], __shfl_xor(m[r], d));
        if (lane == 0) red[0][wave][r] = m[r];
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        m[r] = fmaxf(fmaxf(red[0][0][r], red[0][1][r]), fmaxf(red[0][2][r], red[0][3][r]));
        const float ref = m[r] == -INFINITY ? 0.f : m[r];
        l[r] = 0.f;
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
            const float p = __builtin_amdgcn_exp2f(s[r][j] - ref);
            l[r] += p;
            // [quarter of the piece][key of the vector][lane]: what a lane of any wave
            // reads in the second half are the keys that the same lane has here
            ps[r][(wave * VEC + j) * 64 + lane] = p;
        }
#pragma unroll
        for (int d = 32; d >= 1; d >>= 1) l[r] += __shfl_xor(l[r], d);
        if (lane == 0) red[1][wave][r] = l[r];
    }
    __syncthreads();
    float* part = a.part + (int64_t)blockIdx.x * ROWS * (a.D + 2);
    if (tid < ROWS) {
        part[tid * (a.D + 2)] =
            fmaxf(fmaxf(red[0][0][tid], red[0][1][tid]), fmaxf(red[0][2][tid], red[0][3][tid]));
        part[tid * (a.D + 2) + 1] =
            (red[1][0][tid] + red[1][1][tid]) + (red[1][2][tid] + red[1][3][tid]);
    }
    // values: a wave takes every fourth channel over all the piece's keys
    float p[ROWS][4][VEC];
    uint32_t live[4];
    bool every = true;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        live[k] = ons[k * 64 + lane];
        every = every && live[k] == (1u << VEC) - 1;
#pragma unroll
        for (int r = 0; r < ROWS; ++r)
#pragma unroll
            for (int j = 0; j < VEC; ++j) p[r][k][j] = ps[r][(k * VEC + j) * 64 + lane];
    }
    const T* vp = (const T*)a.v + vol * a.v_stride + (int64_t)hk * a.D * a.tk;
    constexpr int VC = VEC <= 2 ? 4 : VEC == 4 || ROWS == 4 ? 2 : 1;  // the same of the values, a wave's channels
    auto values = [&](auto mode) {
#pragma unroll 1
        for (int c0 = wave; c0 < a.D; c0 += 4 * VC) {
            float x[VC][4][VEC];
#pragma unroll
            for (int i = 0; i < VC; ++i) {
                const int ch = c0 + 4 * i < a.D ? c0 + 4 * i : a.D - 1;
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    ld_keys<T, VEC, decltype(mode)::value>(
                        vp + ch * a.tk, t0 + (k * 64 + lane) * VEC, a.tk, live[k], x[i][k]);
            }
            float o[VC][ROWS];
#pragma unroll
            for (int i = 0; i < VC; ++i)
#pragma unroll
                for (int r = 0; r < ROWS; ++r) {
                    o[i][r] = 0.f;
#pragma unroll
                    for (int k = 0; k < 4; ++k)
#pragma unroll
                        for (int j = 0; j < VEC; ++j)
                            o[i][r] = __builtin_fmaf(p[r][k][j], x[i][k][j], o[i][r]);
                }
#pragma unroll
            for (int d = 32; d >= 1; d >>= 1)
#pragma unroll
                for (int i = 0; i < VC; ++i)
#pragma unroll
                    for (int r = 0; r < ROWS; ++r) o[i][r] += __shfl_xor(o[i][r], d);
            if (lane == 0) {
#pragma unroll
                for (int i = 0; i < VC; ++i)
                    if (c0 + 4 * i < a.D) {
#pragma unroll
                        for (int r = 0; r < ROWS; ++r)
                            part[r * (a.D + 2) + 2 + c0 + 4 * i] = o[i][r];
                    }
            }
        }
    };
    if (__all(every)) values(std::integral_constant<int, 0>{});
    else if (inside) values(std::integral_constant<int, 1>{});
    else values(std::integral_constant<int, 2>{});
}

// One workgroup a query row: weighs the pieces by their maxima and adds them up, thread =
// channel and slice of the pieces, in a fixed order.
template <typename T>
__global__ __launch_bounds__(256) void attn_few_join_k(FewArgs a, int stride) {  // rows a piece
    __shared__ float red[256], rl[4];
    const int nhq = blockIdx.x;  // [volume][head][query token]
    const int nh = nhq / (int)a.tq, tok = nhq - nh * (int)a.tq;
    const int vol = nh / a.heads, h = nh - vol * a.heads, grp = a.heads / a.kv;
    const int kvh = vol * a.kv + h / grp, row = h % grp * (int)a.tq + tok;
    const int tid = threadIdx.x;
    const int64_t step = (int64_t)stride * (a.D + 2);  // from one piece to the next
    const float* p = a.part + ((int64_t)kvh * a.pieces * stride + row) * (a.D + 2);
    float m = -INFINITY;
    for (int i = tid; i < a.pieces; i += 256) m = fmaxf(m, p[i * step]);
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) m = fmaxf(m, __shfl_xor(m, d));
    if ((tid & 63) == 0) rl[tid >> 6] = m;
    __syncthreads();
    m = fmaxf(fmaxf(rl[0], rl[1]), fmaxf(rl[2], rl[3]));
    const float ref = m == -INFINITY ? 0.f : m;
    // channels 0 .. D - 1 and, as channel D, the sum itself
    const int per = a.D < 32 ? 32 : a.D < 64 ? 64 : a.D < 128 ? 128 : 256;  // > D: threads a slice
    const int ch = tid & (per - 1), slice = tid / per, slices = 256 / per;
    float v = 0.f;
    if (ch <= a.D) {
        const int at = ch == a.D ? 1 : 2 + ch;
#pragma unroll 4
        for (int i = slice; i < a.pieces; i += slices)
            v += p[i * step + at] * __builtin_amdgcn_exp2f(p[i * step] - ref);
    }
    __syncthreads();
    red[tid] = v;
    __syncthreads();
    if (tid <= a.D) {
        float l = 0.f;
        v = 0.f;
        for (int i = 0; i < slices; ++i) {
            v += red[i * per + tid];
            l += red[i * per + a.D];
        }
        if (tid < a.D)
            Elt<T>::st((T*)a.o + vol * a.o_stride + ((int64_t)h * a.D + tid) * a.tq + tok,
                       l == 0.f ? 0.f : v / l);
        else if (a.lse)
            a.lse[nhq] = l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * kLn2;
    }
}

// ------------------------------------------------------------------ backward
// Records of the backward, in fragments: 32 keys are K and V in form R and K in form
// T; 32 queries are Q and dO in form R, the row constants, and Q and dO in form T.
template <typename T, int DB> struct Rec {
    static constexpr int NF = 32 * DB / Mm<T>::kPer * 32 / 64;  // fragments of one form
    static constexpr int kK = 0, kV = NF, kKt = 2 * NF, kKeys = 3 * NF * 64;
    static constexpr int kQ = 0, kO = NF, kX = 2 * NF, kQt = 2 * NF + 1, kOt = 3 * NF + 1;
    static constexpr int kQueries = (4 * NF + 1) * 64;  // units
};

// Where a workgroup of the dK/dV kernels stands.
struct DkvPlace {
    int vol, hk, kvh, sp, tile;
    int64_t live;
    __device__ __forceinline__ DkvPlace(const AttnArgs& a, bool split, int bid) {
        tile = bid % a.tiles;
        bid /= a.tiles;
        sp = split ? bid % a.splits : 0;
        kvh = split ? bid / a.splits : bid;
        vol = kvh / a.kv;
        hk = kvh - vol * a.kv;
        live = a.count ? a.count[vol] : a.tk;
    }
};

// The sums of 32 keys (block kb) leave: partial sums of a split, or the gradients.
template <typename T, int DB, bool SPLIT>
__device__ __forceinline__ void dkv_store(const AttnArgs& a, const DkvPlace& p, int64_t kb,
                                          const f32x16 (&dk)[DB], const f32x16 (&dv)[DB]) {
    const int lane = threadIdx.x & 63, half = lane >> 5;
    const int64_t j = kb * 32 + (lane & 31);
    if (j >= p.live) return;
    if (SPLIT) {
        float* to = a.part + ((int64_t)p.kvh * a.splits + p.sp) * 2 * a.D * a.tkp + j;
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
        const int64_t tok = a.idx ? a.idx[p.vol * a.tkp + j] : j;
        T* tk = (T*)a.dk + p.vol * a.k_stride + (int64_t)p.hk * a.D * a.tk + tok;
        T* tv = (T*)a.dv + p.vol * a.v_stride + (int64_t)p.hk * a.D * a.tk + tok;
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

// dK, dV: a workgroup keeps 128 live keys of one key head, 32 a wave as columns, and
// walks the queries of every head of the group, 32 a turn as rows.  Scores leave their
// product as s - lse / scale and dO V^T as dO V^T - D: both constants of a row are added
// by the matrix instruction, from a fragment of the record.
template <typename T, int DB, bool SPLIT>
__device__ __forceinline__ void dkv_block(const AttnArgs& a, int bid, u32x4* room) {
    typedef Mm<T> M;
    typedef typename M::frag frag;
    typedef Rec<T, DB> R;
    constexpr int NF = R::NF, NT = 32 / M::kT, U = R::kQueries;
    const DkvPlace at(a, SPLIT, bid);
    if ((int64_t)at.tile * 128 >= at.live) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t kb = (int64_t)at.tile * 4 + wave;  // block of 32 keys

    frag kf[NF], vf[NF];
#pragma unroll
    for (int f = 0; f < NF; ++f) {
        kf[f] = frag{};
        vf[f] = frag{};
        if (kb * 32 < at.live) {  // else the record need not exist
            const u32x4* rec = a.kv_rec + ((int64_t)at.kvh * (a.tkp / 32) + kb) * R::kKeys;
            kf[f] = frag_of<T>(rec, R::kK + f);
            vf[f] = frag_of<T>(rec, R::kV + f);
        }
    }
    const frag one_s = M::pick(0, lane >> 5), one_d = M::pick(1, lane >> 5);
    f32x16 dk[DB], dv[DB];
#pragma unroll
    for (int e = 0; e < DB; ++e)
#pragma unroll
        for (int i = 0; i < 16; ++i) dk[e][i] = dv[e][i] = 0.f;

    // turns: the records of the group's heads, one behind the other
    const int grp = a.heads / a.kv;
    const int turns = (int)(a.tqp / 32) * grp;
    const int per = SPLIT ? (turns + a.splits - 1) / a.splits : turns;
    const int i0 = SPLIT ? (at.sp * per < turns ? at.sp * per : turns) : 0;
    const int i1 = i0 + per < turns ? i0 + per : turns;
    const u32x4* rec =
        a.q_rec + ((int64_t)(at.vol * a.heads + at.hk * grp) * (a.tqp / 32) + i0) * U;
    StageHalves<U> next;
    if (i0 < i1) {
        next.template load<0>(rec);
        next.template store<0>(room);
        next.template load<1>(rec);
        next.template store<1>(room);
    }
    __syncthreads();
    for (int i = i0; i < i1; ++i) {
        const u32x4* cur = room + ((i - i0) & 1) * U;
        u32x4* other = room + (((i - i0) & 1) ^ 1) * U;
        if (i + 1 < i1) {
            rec += U;
            next.template load<0>(rec);
        }
        f32x16 s, dp;
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] = dp[r] = 0.f;
#pragma unroll
        for (int f = 0; f < NF; ++f) {
            s = M::mul(frag_of<T>(cur, R::kQ + f), kf[f], s);
            dp = M::mul(frag_of<T>(cur, R::kO + f), vf[f], dp);
        }
        const frag x = frag_of<T>(cur, R::kX);
        s = M::add_row(x, one_s, s);
        dp = M::add_row(x, one_d, dp);
        if (i + 1 < i1) {
            next.template store<0>(other);
            next.template load<1>(rec);
        }
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            s[r] = __builtin_amdgcn_exp2f(s[r] * a.c);
            dp[r] *= s[r];
        }
#pragma unroll
        for (int w = 0; w < NT; ++w) {
            const frag p = to_frag<T>(s, w), d = to_frag<T>(dp, w);
#pragma unroll
            for (int e = 0; e < DB; ++e) {
                dv[e] = M::mul(frag_of<T>(cur, R::kOt + w * DB + e), p, dv[e]);
                dk[e] = M::mul(frag_of<T>(cur, R::kQt + w * DB + e), d, dk[e]);
            }
        }
        if (i + 1 < i1) next.template store<1>(other);
        __syncthreads();
    }
    dkv_store<T, DB, SPLIT>(a, at, kb, dk, dv);
}

// The same in bfloat16 with 64 keys a wave, in two column blocks A and B, and the
// phases of neighbouring turns laid over each other, so that the matrix cores work
// while the vector ALU forms the other block's probabilities.  Turn i is
//   X: dV, dK of B for turn i - 1, scores of B for turn i   beside   exp of A, turn i
//   Y: dV, dK of A for turn i, scores of A for turn i + 1   beside   exp of B, turn i
// A fragment read from LDS feeds both blocks (it stays in registers from Y to X, or
// from X to Y): 9 (D <= 64: 17) reads for 20 (36) products of 32 cycles, where one
// block a wave would ask LDS for as many cycles as the products take.  One wave a SIMD
// holds all this (two at D <= 32); the order of instructions is pinned step by step.
// Three LDS buffers: turn i reads T of record i and R of i + 1 and writes record i + 2.
template <int DB, bool SPLIT>
__global__ __launch_bounds__(256, (DB == 1 ? 2 : 1)) void attn_dkv2_k(AttnArgs a) {
    typedef Mm<bf16> M;
    typedef bf16x8 frag;
    typedef Rec<bf16, DB> R;
    constexpr int NF = R::NF, U = R::kQueries;
    __shared__ u32x4 lds[3][U];
    const DkvPlace at(a, SPLIT, xcd_remap(blockIdx.x, gridDim.x));
    if ((int64_t)at.tile * 256 >= at.live) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t kb = ((int64_t)at.tile * 4 + wave) * 2;  // first block of 32 keys

    frag kf[2][NF], vf[2][NF];
#pragma unroll
    for (int c = 0; c < 2; ++c)
#pragma unroll
        for (int f = 0; f < NF; ++f) {
            kf[c][f] = frag{};
            vf[c][f] = frag{};
            if ((kb + c) * 32 < at.live) {  // else the record need not exist
                const u32x4* rec = a.kv_rec + ((int64_t)at.kvh * (a.tkp / 32) + kb + c) * R::kKeys;
                kf[c][f] = frag_of<bf16>(rec, R::kK + f);
                vf[c][f] = frag_of<bf16>(rec, R::kV + f);
            }
        }
    const frag one_s = M::pick(0, lane >> 5), one_d = M::pick(1, lane >> 5);
    f32x16 dk[2][DB], dv[2][DB], s[2], dp[2];
#pragma unroll
    for (int c = 0; c < 2; ++c)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            s[c][i] = dp[c][i] = 0.f;
#pragma unroll
            for (int e = 0; e < DB; ++e) dk[c][e][i] = dv[c][e][i] = 0.f;
        }
    uint32_t pw[2][8], dw[2][8];  // probabilities and score gradients, two a word
    frag qa[NF], oa[NF], xa, qt[NF], ot[NF];
#pragma unroll
    for (int i = 0; i < 8; ++i) pw[1][i] = dw[1][i] = 0;
#pragma unroll
    for (int f = 0; f < NF; ++f) qt[f] = ot[f] = frag{};

    const int grp = a.heads / a.kv;
    const int turns = (int)(a.tqp / 32) * grp;
    const int per = SPLIT ? (turns + a.splits - 1) / a.splits : turns;
    const int i0 = SPLIT ? (at.sp * per < turns ? at.sp * per : turns) : 0;
    const int i1 = i0 + per < turns ? i0 + per : turns;
    const u32x4* rec =
        a.q_rec + ((int64_t)(at.vol * a.heads + at.hk * grp) * (a.tqp / 32) + i0) * U;
    Stage<U> next;

    // one of the 2 NF products of dV and dK of block c
    auto grad_step = [&](int c, int t) {
        const int f = t >> 1, w = f / DB, e = f % DB;
        const u32x4 p = t & 1 ? u32x4{dw[c][4 * w], dw[c][4 * w + 1], dw[c][4 * w + 2], dw[c][4 * w + 3]}
                              : u32x4{pw[c][4 * w], pw[c][4 * w + 1], pw[c][4 * w + 2], pw[c][4 * w + 3]};
        if (t & 1) dk[c][e] = M::mul(qt[f], __builtin_bit_cast(frag, p), dk[c][e]);
        else dv[c][e] = M::mul(ot[f], __builtin_bit_cast(frag, p), dv[c][e]);
    };
    // one of the 2 NF + 2 products of the scores and of dO V^T of block c
    auto score_step = [&](int c, int t) {
        const f32x16 zero = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f,
                             0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        if (t == 0) s[c] = M::mul(qa[0], kf[c][0], zero);
        else if (t == 1) dp[c] = M::mul(oa[0], vf[c][0], zero);
        else if (t == 2 * NF) s[c] = M::mul(xa, one_s, s[c]);
        else if (t == 2 * NF + 1) dp[c] = M::mul(xa, one_d, dp[c]);
        else if (t & 1) dp[c] = M::mul(oa[t >> 1], vf[c][t >> 1], dp[c]);
        else s[c] = M::mul(qa[t >> 1], kf[c][t >> 1], s[c]);
    };
    // probabilities and score gradients of block c: the exponential of register r, and
    // what follows it for register r - 1 (an exponential's result is not ready for the
    // next instruction)
    auto exp_step = [&](int c, int r) {
        if (r < 16) s[c][r] = __builtin_amdgcn_exp2f(s[c][r] * a.c);
        if (r == 0) return;
        dp[c][r - 1] *= s[c][r - 1];
        if (!(r & 1)) {
            pw[c][(r >> 1) - 1] = pack_bf16x2(s[c][r - 2], s[c][r - 1]);
            dw[c][(r >> 1) - 1] = pack_bf16x2(dp[c][r - 2], dp[c][r - 1]);
            // formed here, not where it is used
            asm volatile("" : "+v"(pw[c][(r >> 1) - 1]), "+v"(dw[c][(r >> 1) - 1]));
        }
    };
    // fragments in the order in which the products take them
    auto read_r = [&](const u32x4* b, int f) {
        if (f == 2 * NF) xa = frag_of<bf16>(b, R::kX);
        else if (f & 1) oa[f >> 1] = frag_of<bf16>(b, R::kO + (f >> 1));
        else qa[f >> 1] = frag_of<bf16>(b, R::kQ + (f >> 1));
    };
    auto read_t = [&](const u32x4* b, int f) {
        if (f & 1) qt[f >> 1] = frag_of<bf16>(b, R::kQt + (f >> 1));
        else ot[f >> 1] = frag_of<bf16>(b, R::kOt + (f >> 1));
    };
    constexpr int N1 = 2 * NF, N2 = 2 * NF + 2, N = N1 + N2;  // products of X, as of Y

    if (i0 < i1) {
        next.load(rec);
        next.store(lds[0]);
        next.load(i0 + 1 < i1 ? rec + U : rec);
        next.store(lds[1]);
    }
    const u32x4* last = rec + (int64_t)(i1 - i0 - 1) * U;
    __syncthreads();
    if (i0 < i1) {
#pragma unroll
        for (int f = 0; f < 2 * NF + 1; ++f) read_r(lds[0], f);
#pragma unroll
        for (int t = 0; t < N2; ++t) score_step(0, t);
    }
    int b0 = 0, b1 = 1, b2 = 2;  // buffers of records i, i + 1, i + 2
    for (int i = i0; i < i1; ++i) {
        // behind the last record it is taken again, so that no branch divides the turn:
        // what is formed from it is not used
        next.load(i + 2 < i1 ? rec + 2 * U : last);
        // Reads of LDS are spread over the turn, as far as a fragment's last use before
        // and its first use behind allow: four waves that read at every step would ask
        // for all that LDS gives, and stand still for it.
        constexpr int kEarly = NF;  // fragments of R that X reads, behind its scores' first
        // X
#pragma unroll
        for (int t = 0; t < N; ++t) {
            if (t < N1) grad_step(1, t);
            else score_step(1, t - N1);
#pragma unroll
            for (int r = 0; r < 17; ++r)
                if (r * (N - 2) / 17 + 2 == t) exp_step(0, r);
            if (t & 1 && t / 2 < N1) read_t(lds[b0], t / 2);
            if (!(t & 1) && t >= N1 + 2 && (t - N1 - 2) / 2 < kEarly) read_r(lds[b1], (t - N1 - 2) / 2);
            __builtin_amdgcn_sched_barrier(0);
        }
        // Y
#pragma unroll
        for (int t = 0; t < N; ++t) {
            if (!(t & 1) && kEarly + t / 2 < 2 * NF + 1) read_r(lds[b1], kEarly + t / 2);
            if (t < N1) grad_step(0, t);
            else score_step(0, t - N1);
#pragma unroll
            for (int r = 0; r < 17; ++r)
                if (r * (N - 2) / 17 + 2 == t) exp_step(1, r);
            if (t >= N - 6 && t - (N - 6) < Stage<U>::N) next.store(lds[b2], t - (N - 6));
            __builtin_amdgcn_sched_barrier(0);
        }
        __syncthreads();
        rec += U;
        const int b = b0;
        b0 = b1;
        b1 = b2;
        b2 = b;
    }
#pragma unroll
    for (int t = 0; t < N1; ++t) grad_step(1, t);  // B of the last turn
    dkv_store<bf16, DB, SPLIT>(a, at, kb, dk[0], dv[0]);
    dkv_store<bf16, DB, SPLIT>(a, at, kb + 1, dk[1], dv[1]);
}

// The sums of 32 queries (block qb) leave: partial sums of a split, or the gradient.
template <typename T, int DB, bool SPLIT>
__device__ __forceinline__ void dq_store(const AttnArgs& a, int nh, int sp, int64_t qb,
                                         const f32x16 (&dq)[DB]) {
    const int lane = threadIdx.x & 63, half = lane >> 5;
    const int64_t qt = qb * 32 + (lane & 31);
    if (qt >= a.tq) return;
    const int vol = nh / a.heads, h = nh - vol * a.heads;
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

// dQ: a workgroup keeps 128 queries of one head, 32 a wave as columns, and walks the
// live keys, 32 a turn as rows.
template <typename T, int DB, bool SPLIT>
__device__ __forceinline__ void dq_block(const AttnArgs& a, int bid, u32x4* room) {
    typedef Mm<T> M;
    typedef typename M::frag frag;
    typedef Rec<T, DB> R;
    constexpr int NF = R::NF, NT = 32 / M::kT, U = R::kKeys;
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
    frag qf[NF], of[NF];
#pragma unroll
    for (int f = 0; f < NF; ++f) {
        qf[f] = frag{};
        of[f] = frag{};
        if (have) {
            const u32x4* rec = a.q_rec + ((int64_t)nh * (a.tqp / 32) + qb) * R::kQueries;
            qf[f] = frag_of<T>(rec, R::kQ + f);
            of[f] = frag_of<T>(rec, R::kO + f);
        }
    }
    const int64_t at = (int64_t)nh * a.tqp + qb * 32 + (lane & 31);
    const float ls = have ? a.lse2[at] : INFINITY, de = have ? a.delta[at] : 0.f;
    f32x16 dq[DB];
#pragma unroll
    for (int e = 0; e < DB; ++e)
#pragma unroll
        for (int i = 0; i < 16; ++i) dq[e][i] = 0.f;
    int b0, b1;
    split_range(live, 32, SPLIT ? a.splits : 1, sp, b0, b1);
    const u32x4* rec = a.kv_rec + ((int64_t)kvh * (a.tkp / 32) + b0) * U;
    Stage<U> next;
    if (b0 < b1) {
        next.load(rec);
        next.store(room);
    }
    __syncthreads();
    for (int b = b0; b < b1; ++b) {
        const u32x4* cur = room + ((b - b0) & 1) * U;
        if (b + 1 < b1) {
            rec += U;
            next.load(rec);
        }
        f32x16 s, dp;
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] = dp[r] = 0.f;
#pragma unroll
        for (int f = 0; f < NF; ++f) {
            s = M::mul(frag_of<T>(cur, R::kK + f), qf[f], s);
            dp = M::mul(frag_of<T>(cur, R::kV + f), of[f], dp);
        }
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            s[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r], a.c, -ls));
            dp[r] = s[r] * (dp[r] - de);
        }
        // rows behind the last key have K = V = 0 and so give nothing to dq, as
        // long as their P stays finite, which exp(-lse) might not
        const int left = live - (int64_t)b * 32 < 32 ? (int)(live - (int64_t)b * 32) : 32;
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
                dq[e] = M::mul(frag_of<T>(cur, R::kKt + w * DB + e), d, dq[e]);
        }
        if (b + 1 < b1) next.store(room + (((b - b0) & 1) ^ 1) * U);
        __syncthreads();
    }
    dq_store<T, DB, SPLIT>(a, nh, sp, qb, dq);
}

// Both walks of the backward in one launch, one behind the other in the grid: neither
// reads what the other writes, and on small maps, where each alone leaves CUs idle, they
// overlap (2 x 4 x 64 over 6x7x6 in float32: 22 us as two launches, 16 as one).
struct BwdArgs {
    AttnArgs kv, q;  // dK/dV, dQ
    int kv_blocks, q_blocks;
};
// Two waves a SIMD in bfloat16 at any head size: at head_dim 128 that spills 36 registers
// and still takes 1255 us against 1730 (8 x 4 heads over 4032 tokens).
template <typename T, int DB, bool KS, bool QS>
__global__ __launch_bounds__(256, (DB <= 2 || sizeof(T) == 2 ? 2 : 1)) void attn_bwd_k(BwdArgs g) {
    __shared__ u32x4 room[2 * Rec<T, DB>::kQueries];  // the larger record
    static_assert(Rec<T, DB>::kQueries >= Rec<T, DB>::kKeys, "room");
    const int b = (int)blockIdx.x;
    if (b < g.kv_blocks) dkv_block<T, DB, KS>(g.kv, xcd_remap(b, g.kv_blocks), room);
    else dq_block<T, DB, QS>(g.q, xcd_remap(b - g.kv_blocks, g.q_blocks), room);
}

// The same in bfloat16 with 64 queries a wave, in two column blocks A and B, and the
// phases of neighbouring turns laid over each other as in attn_dkv2_k:
//   X: dQ of B for turn i - 1, scores of B for turn i   beside   exp of A, turn i
//   Y: dQ of A for turn i, scores of A for turn i + 1   beside   exp of B, turn i
// -D is added to dO V^T by one more product: ones for every key times the query's
// constant.  The last keys, where they fill no record, are taken behind the loop.
// Never split: it is taken only where the queries alone fill the GPU.
template <int DB>
__global__ __launch_bounds__(256, (DB == 1 ? 2 : 1)) void attn_dq2_k(AttnArgs a) {
    typedef Mm<bf16> M;
    typedef bf16x8 frag;
    typedef Rec<bf16, DB> R;
    constexpr int NF = R::NF, U = R::kKeys;
    __shared__ u32x4 lds[3][U];
    const int bid = xcd_remap(blockIdx.x, gridDim.x);
    const int tile = bid % a.tiles;
    const int nh = bid / a.tiles;
    const int vol = nh / a.heads, h = nh - vol * a.heads;
    const int kvh = vol * a.kv + h / (a.heads / a.kv);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t live = a.count ? a.count[vol] : a.tk;
    const int64_t qb = ((int64_t)tile * 4 + wave) * 2;

    frag qf[2][NF], of[2][NF], low[2];
    float ls[2];
    f32x16 dq[2][DB], s[2], dp[2];
    uint32_t dw[2][8];  // score gradients, two a word
    frag ka[NF], va[NF], kt[NF];
#pragma unroll
    for (int c = 0; c < 2; ++c) {
        const bool have = (qb + c) * 32 < a.tqp;
#pragma unroll
        for (int f = 0; f < NF; ++f) {
            qf[c][f] = frag{};
            of[c][f] = frag{};
            if (have) {
                const u32x4* rec = a.q_rec + ((int64_t)nh * (a.tqp / 32) + qb + c) * R::kQueries;
                qf[c][f] = frag_of<bf16>(rec, R::kQ + f);
                of[c][f] = frag_of<bf16>(rec, R::kO + f);
            }
        }
        const int64_t at = (int64_t)nh * a.tqp + (qb + c) * 32 + (lane & 31);
        ls[c] = have ? a.lse2[at] : INFINITY;
        low[c] = __builtin_bit_cast(frag, M::rows(have ? -a.delta[at] : 0.f, 0.f, lane >> 5));
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            s[c][i] = dp[c][i] = 0.f;
#pragma unroll
            for (int e = 0; e < DB; ++e) dq[c][e][i] = 0.f;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) dw[c][i] = 0;
    }
    const frag ones = M::pick(0, lane >> 5);
#pragma unroll
    for (int f = 0; f < NF; ++f) kt[f] = frag{};

    const int whole = (int)(live / 32);  // records that keys fill
    const int left = (int)(live - (int64_t)whole * 32);  // keys behind them
    const u32x4* const first = a.kv_rec + (int64_t)kvh * (a.tkp / 32) * U;
    const u32x4* rec = first;
    const u32x4* last = rec + (int64_t)(whole - 1) * U;
    Stage<U> next;

    auto grad_step = [&](int c, int t) {  // one of the NF products of dQ of block c
        const int w = t / DB, e = t % DB;
        const u32x4 p = {dw[c][4 * w], dw[c][4 * w + 1], dw[c][4 * w + 2], dw[c][4 * w + 3]};
        dq[c][e] = M::mul(kt[t], __builtin_bit_cast(frag, p), dq[c][e]);
    };
    // one of the 2 NF + 1 products of the scores and of dO V^T - D of block c
    auto score_step = [&](int c, int t) {
        const f32x16 zero = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f,
                             0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        if (t == 0) dp[c] = M::mul(ones, low[c], zero);
        else if (t == 1) s[c] = M::mul(ka[0], qf[c][0], zero);
        else if (t & 1) s[c] = M::mul(ka[t >> 1], qf[c][t >> 1], s[c]);
        else dp[c] = M::mul(va[(t >> 1) - 1], of[c][(t >> 1) - 1], dp[c]);
    };
    // the exponential of register r, and what follows it for register r - 1
    auto exp_step = [&](int c, int r) {
        if (r < 16) s[c][r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[c][r], a.c, -ls[c]));
        if (r == 0) return;
        dp[c][r - 1] *= s[c][r - 1];
        if (!(r & 1)) {
            dw[c][(r >> 1) - 1] = pack_bf16x2(dp[c][r - 2], dp[c][r - 1]);
            // formed here, not where it is used
            asm volatile("" : "+v"(dw[c][(r >> 1) - 1]));
        }
    };
    auto read_r = [&](const u32x4* b, int f) {
        if (f & 1) va[f >> 1] = frag_of<bf16>(b, R::kV + (f >> 1));
        else ka[f >> 1] = frag_of<bf16>(b, R::kK + (f >> 1));
    };
    constexpr int N1 = NF, N2 = 2 * NF + 1, N = N1 + N2;  // products of X, as of Y

    if (whole > 0) {
        next.load(rec);
        next.store(lds[0]);
        next.load(whole > 1 ? rec + U : rec);
        next.store(lds[1]);
    }
    __syncthreads();
    if (whole > 0) {
#pragma unroll
        for (int f = 0; f < 2 * NF; ++f) read_r(lds[0], f);
#pragma unroll
        for (int t = 0; t < N2; ++t) score_step(0, t);
    }
    int u0 = 0, u1 = 1, u2 = 2;  // buffers of records i, i + 1, i + 2
    for (int i = 0; i < whole; ++i) {
        // behind the last record it is taken again, so that no branch divides the turn:
        // what is formed from it is not used
        next.load(i + 2 < whole ? rec + 2 * U : last);
        // reads of LDS spread over the turn, as in attn_dkv2_k
        // X
#pragma unroll
        for (int t = 0; t < N; ++t) {
            if (t < N1) grad_step(1, t);
            else score_step(1, t - N1);
#pragma unroll
            for (int r = 0; r < 17; ++r)
                if (r * (N - 2) / 17 + 2 == t) exp_step(0, r);
            if (t & 1 && t / 2 < N1) kt[t / 2] = frag_of<bf16>(lds[u0], R::kKt + t / 2);
            if (!(t & 1) && t >= N1 + 2 && (t - N1 - 2) / 2 < NF) read_r(lds[u1], (t - N1 - 2) / 2);
            __builtin_amdgcn_sched_barrier(0);
        }
        // Y
#pragma unroll
        for (int t = 0; t < N; ++t) {
            if (!(t & 1) && t / 2 < NF) read_r(lds[u1], NF + t / 2);
            if (t < N1) grad_step(0, t);
            else score_step(0, t - N1);
#pragma unroll
            for (int r = 0; r < 17; ++r)
                if (r * (N - 2) / 17 + 2 == t) exp_step(1, r);
            if (t >= N - 4 && t - (N - 4) < Stage<U>::N) next.store(lds[u2], t - (N - 4));
            __builtin_amdgcn_sched_barrier(0);
        }
        __syncthreads();
        rec += U;
        const int u = u0;
        u0 = u1;
        u1 = u2;
        u2 = u;
    }
#pragma unroll
    for (int t = 0; t < N1; ++t) grad_step(1, t);  // B of the last turn
    if (left > 0) {  // keys that fill no record: what lies behind them is cleared
        next.load(first + (int64_t)whole * U);
        next.store(lds[u2]);
        __syncthreads();
#pragma unroll
        for (int f = 0; f < NF; ++f) {
            read_r(lds[u2], 2 * f);
            read_r(lds[u2], 2 * f + 1);
            kt[f] = frag_of<bf16>(lds[u2], R::kKt + f);
        }
#pragma unroll
        for (int c = 0; c < 2; ++c) {
#pragma unroll
            for (int t = 0; t < N2; ++t) score_step(c, t);
#pragma unroll
            for (int r = 0; r < 16; ++r)
                if (8 * (r / 4) + 4 * (lane >> 5) + r % 4 >= left) {
                    s[c][r] = -INFINITY;
                    dp[c][r] = 0.f;
                }
#pragma unroll
            for (int r = 0; r < 17; ++r) exp_step(c, r);
#pragma unroll
            for (int t = 0; t < N1; ++t) grad_step(c, t);
        }
    }
#pragma unroll
    for (int c = 0; c < 2; ++c) dq_store<bf16, DB, false>(a, nh, 0, qb + c, dq[c]);
}

// Sums of the splits of the backward passes, in a fixed order: [nh][split][rows][tp] ->
// the tensors' channels (rows = D for dq, 2 D for dk and dv).  A workgroup takes 64
// tokens and 8 channels.
struct SumJob {
    const float* part;
    void *a, *b;               // channels 0 .. D-1 and D .. rows-1
    int64_t a_stride, b_stride, tokens, tp;
    const int *idx, *count;
    int heads, D, rows, splits, tiles, first;
};
struct SumArgs {
    SumJob job[2];
    int jobs;
};
template <typename T>
__global__ __launch_bounds__(256) void attn_sum_k(SumArgs g) {
    const SumJob& j = g.job[g.jobs > 1 && (int)blockIdx.x >= g.job[1].first ? 1 : 0];
    const int lane = threadIdx.x & 63, sub = threadIdx.x >> 6;
    const int groups = (j.rows + 7) / 8;
    int b = (int)blockIdx.x - j.first;
    const int tile = b % j.tiles;
    b /= j.tiles;
    const int c0 = b % groups * 8, nh = b / groups;
    const int vol = nh / j.heads, h = nh - vol * j.heads;
    const int64_t t = (int64_t)tile * 64 + lane;
    if (t >= (j.count ? j.count[vol] : j.tokens)) return;
    const int64_t tok = j.idx ? j.idx[vol * j.tp + t] : t;
    const float* p = j.part + (int64_t)nh * j.splits * j.rows * j.tp + t;
    const int64_t d1 = (int64_t)(c0 + sub < j.rows ? c0 + sub : j.rows - 1) * j.tp;
    const int64_t d2 = (int64_t)(c0 + sub + 4 < j.rows ? c0 + sub + 4 : j.rows - 1) * j.tp;
    float sum[2] = {0.f, 0.f};
    for (int s0 = 0; s0 < j.splits; s0 += 8) {  // eight splits' loads in flight
        float x1[8], x2[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int64_t s = s0 + i < j.splits ? s0 + i : j.splits - 1;
            x1[i] = p[s * j.rows * j.tp + d1];
            x2[i] = p[s * j.rows * j.tp + d2];
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (s0 + i >= j.splits) break;
            sum[0] += x1[i];
            sum[1] += x2[i];
        }
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int c = c0 + sub + 4 * k;
        if (c >= j.rows) continue;
        const float v = sum[k];
        T* to = c < j.D ? (T*)j.a + vol * j.a_stride + ((int64_t)h * j.D + c) * j.tokens
                        : (T*)j.b + vol * j.b_stride + ((int64_t)h * j.D + c - j.D) * j.tokens;
        Elt<T>::st(to + tok, v);
    }
}

// ------------------------------------------------------------------ host
struct AttnPlan {
    int64_t tqp, tkp;
    int DB, es;
    int kc, qc;      // blocks of 32 kept tokens a wave: dK/dV, dQ
    int fs, ks, qs;  // splits of the forward, of dK/dV, of dQ
    size_t few, idx, count, kv_rec, q_rec, lse2, delta, part, qpart, fpart, stat, bytes[2];
};

// Ways to split a long walk: until there are about two workgroups for each CU, but
// not into pieces of fewer than `least` turns.
static int splits_for(int64_t groups, int64_t turns, int64_t least, int per_cu = 2) {
    const int64_t want = per_cu * (int64_t)device_cus();
    int64_t s = (want + groups / 2) / groups;
    if (s > turns / least) s = turns / least;
    if (s > 256) s = 256;
    return s < 2 ? 1 : (int)s;
}

// Backward in bfloat16: two blocks of 32 kept tokens a wave up to head_dim 64, where that
// leaves three workgroups for two CUs.  Above 64 it is not built: dQ would find registers
// up to 128, dK/dV would spill 10 at 96 and 308 at 128; neither was timed.  Both walks at 4 x 2
// heads over 24x28x24 voxels: 2120 us with one block, 1714 with two at head_dim 64, 1220
// and 1060 at 32; 8 x 4 heads x 32 over 2100 tokens (288 workgroups) 126 and 127.  The
// forward gains nothing by it: its bound is the exponentials, whose number stays
// (head_dim 32: 433 us with one block, 473 with two; 64: 604 and 581).
static int columns_for(const rat3d_attention_desc& d, int DB, int64_t groups) {
    return d.dtype == RAT3D_BF16 && DB <= 2 && 2 * groups >= 3 * (int64_t)device_cus() ? 2 : 1;
}

// Keys of a piece of the kernel for few rows: 16-byte accesses where that leaves two
// workgroups for each CU, else 4-byte ones.
static int few_keys(const rat3d_attention_desc& d) {
    const int es = d.dtype == RAT3D_BF16 ? 2 : 4;
    const int64_t wide = 256 * 16 / es;
    const bool many = (int64_t)d.n * d.kv_heads * ceil_div(d.tk, wide) >= 2 * (int64_t)device_cus();
    return (int)(many ? wide : wide / 4);
}
// The kernel for few rows is taken up to eight rows in bfloat16, sixteen in float32.
// Measured against packing and tiles: 8 x 2 key heads x 32 over 48x56x48, 8 rows 117
// against 241 us (bfloat16) and 165 against 757 (float32), 16 rows 213 against 231 and
// 301 against 758; 4 x 2 x 64 over 24x28x24, 8 rows 39 against 44 and 51 against 106, 16
// rows 50 against 43 and 83 against 106.
static bool few_rows(const rat3d_attention_desc& d) {
    return d.heads / d.kv_heads * d.tq <= (d.dtype == RAT3D_BF16 ? 8 : 16);
}
static int few_stride(const rat3d_attention_desc& d) {  // rows that a piece's workgroups hold
    const int64_t rows = d.heads / d.kv_heads * d.tq;
    return rows <= 2 ? (int)rows : (int)(rows + 3) / 4 * 4;
}

// masked: whether a mask is given.  Where one is, much of dK/dV's workgroups find no
// live key (a brain fills about 0.4 of its box), so that walk is cut into twice as
// many pieces: 4 x 2 x 40 over 12x14x11, 0.38 live, 50 us in 480 workgroups, 31 in 1080.
static AttnPlan attn_plan(const rat3d_attention_desc& d, bool masked) {
    AttnPlan p = {};
    p.es = d.dtype == RAT3D_BF16 ? 2 : 4;
    p.DB = (d.head_dim + 31) / 32;
    p.tqp = ceil_div(d.tq, 64) * 64;
    p.tkp = ceil_div(d.tk, 64) * 64;
    const int64_t nq = (int64_t)d.n * d.heads, nk = (int64_t)d.n * d.kv_heads;
    p.qc = columns_for(d, p.DB, nq * ceil_div(d.tq, 256));
    p.kc = columns_for(d, p.DB, nk * ceil_div(d.tk, 256));
    // a turn of float32 takes microseconds, one of bfloat16 a fraction
    const int least = d.dtype == RAT3D_BF16 ? 4 : 1;
    p.fs = splits_for(nq * ceil_div(d.tq, 128), p.tkp / 32, least);
    // two column blocks are taken from 1.5 workgroups a CU on, where there is nothing to split
    p.qs = p.qc == 2 ? 1 : splits_for(nq * ceil_div(d.tq, 128), p.tkp / 32, least);
    p.ks = splits_for(nk * ceil_div(d.tk, 128 * p.kc), p.tqp / 32 * (d.heads / d.kv_heads), least,
                      masked ? 4 : 2);
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t r = at;
        at += (bytes + 255) / 256 * 256;
        return r;
    };
    const size_t qb = (size_t)nq * p.tqp * p.DB * 32 * p.es;  // one form of the queries
    const size_t kb = (size_t)nk * p.tkp * p.DB * 32 * p.es;
    if (few_rows(d)) {  // reads the mask itself: its sums alone
        p.few = take((size_t)nk * ceil_div(d.tk, few_keys(d)) * few_stride(d) * (d.head_dim + 2) *
                     sizeof(float));
        p.bytes[0] = at;
        at = 0;
    }
    p.idx = take((size_t)d.n * p.tkp * sizeof(int));
    p.count = take((size_t)d.n * sizeof(int));
    const size_t both = at;
    p.kv_rec = at;
    if (!few_rows(d)) {  // forward: records of two forms
        take(2 * kb);
        if (p.fs > 1) {
            p.stat = take((size_t)nq * p.fs * 2 * p.tqp * sizeof(float));
            p.fpart = take((size_t)nq * p.fs * d.head_dim * p.tqp * sizeof(float));
        }
        p.bytes[0] = at;
    }
    // backward: records of three forms, and of four and the row constants
    at = both;
    take(3 * kb);
    p.q_rec = take(4 * qb + (size_t)nq * (p.tqp / 32) * 1024);
    p.lse2 = take((size_t)nq * p.tqp * sizeof(float));
    p.delta = take((size_t)nq * p.tqp * sizeof(float));
    const size_t kp = p.ks > 1 ? (size_t)nk * p.ks * 2 * d.head_dim * p.tkp * sizeof(float) : 0;
    const size_t qp = p.qs > 1 ? (size_t)nq * p.qs * d.head_dim * p.tqp * sizeof(float) : 0;
    p.part = take(kp);
    p.qpart = take(qp);
    p.bytes[1] = at;
    return p;
}

size_t attention_ws_bytes(const rat3d_attention_desc& d, int pass) {
    const size_t a = attn_plan(d, false).bytes[pass], b = attn_plan(d, true).bytes[pass];
    return a > b ? a : b;
}

bool attention_fits(const rat3d_attention_desc& d) {
    const AttnPlan p = attn_plan(d, true);
    const int64_t nq = (int64_t)d.n * d.heads;
    // workgroups of the largest launches (each of 256 threads, 2^32 threads a launch);
    // joins and sums follow splits alone, which few workgroups get
    return 2 * nq * ceil_div(d.tq, 64) + 2 * (int64_t)d.n * d.kv_heads * ceil_div(d.tk, 64) <
               (1 << 24) &&
           nq * ceil_div(d.tq, 128) * p.fs < (1 << 24) &&
           nq * ceil_div(d.tq, 128) * p.qs + (int64_t)d.n * d.kv_heads * ceil_div(d.tk, 128) * p.ks <
               (1 << 24) &&
           (!few_rows(d) || ((int64_t)d.n * d.kv_heads * ceil_div(d.tk, few_keys(d)) * 4 < (1 << 24) &&
                             nq * d.tq < (1 << 24))) &&
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
    a.kv_rec = (const u32x4*)(w + p.kv_rec);
    return a;
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

// r, t: fragments of the record where forms R and T begin, or -1.
static PackJob pack_job(const void* src, int64_t stride, int64_t tokens, int heads,
                        const u32x4* rec, int units, int r, int t, const AttnArgs& a, bool keys) {
    PackJob j = {};
    j.src = src;
    j.stride = stride;
    j.tokens = tokens;
    j.heads = heads;
    j.tiles = (int)ceil_div(tokens, kPackTok);
    j.rec = const_cast<u32x4*>(rec);
    j.units = units;
    j.r = r < 0 ? -1 : r * 64;
    j.t = t < 0 ? -1 : t * 64;
    j.x = -1;
    if (keys) {
        j.idx = const_cast<int*>(a.idx);
        j.count = const_cast<int*>(a.count);
    }
    return j;
}

template <typename T, int DB>
static void pack_kernel(const PackArgs& pa, int64_t blocks, hipStream_t st) {
    attn_pack_k<T, DB><<<(unsigned)blocks, 256, 0, st>>>(pa);
}
static rat3d_status pack_launch(PackArgs& pa, int n, int DB, rat3d_dtype dt, hipStream_t st) {
    int64_t blocks = 0;
    for (int i = 0; i < pa.jobs; ++i) {
        pa.job[i].first = (int)blocks;
        blocks += (int64_t)n * pa.job[i].heads * pa.job[i].tiles;
    }
    RAT3D_ATTN(pack_kernel, dt, DB, pa, blocks, st);
    return RAT3D_OK;
}

// Small maps: each workgroup of the packing finds its live keys itself (one 8-byte read a
// thread and one scan), and a launch less is waited for: forward, backward at 2 heads x 32
// over 252 tokens 14.6 -> 13.0, 18.2 -> 15.8 us, at 4 x 4 heads x 40 over 1848 32.4 -> 30.7,
// 57.5 -> 55.7.  With 32 tokens a thread, which reaches 8192, the scan took longer than the
// launch that it saves at 252 (16.0 us) and 1000 tokens and gained 1 to 4 % from 4032 on.
static bool pack_scans(const rat3d_attention_desc& d) { return d.tk <= 256 * kLook; }

static rat3d_status live_keys(const rat3d_attention_desc& d, const AttnPlan& p, char* w,
                              const uint8_t* mask, AttnArgs* a, hipStream_t st) {
    if (!mask) return RAT3D_OK;
    a->idx = (const int*)(w + p.idx);
    a->count = (const int*)(w + p.count);
    if (pack_scans(d)) return RAT3D_OK;
    ProfScope ps("attn_live", st, 0.0, (double)d.n * d.tk);
    live_keys_k<<<d.n, 1024, 0, st>>>(mask, d.tk, p.tkp, (int*)(w + p.idx), (int*)(w + p.count));
    RAT3D_LAUNCH_CHECK();
    return RAT3D_OK;
}

// Jobs 0 and 1 pack keys and values.
static void pack_mask(const rat3d_attention_desc& d, const uint8_t* mask, PackArgs& pa) {
    if (!mask) return;
    pa.job[0].mask = pa.job[1].mask = mask;
    if (pack_scans(d)) {
        pa.job[0].scan = 2;
        pa.job[1].scan = 1;
    }
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
// kc, qc: column blocks of the two walks; both walks of one block go in one launch.  `one`:
// operations of one product over all keys, of which dK and dV need four and dQ the fifth.
template <typename T, int DB>
static void bwd_launch(const BwdArgs& g, int kc, int qc, double one, hipStream_t st) {
    const bool ks = g.kv.splits > 1, qs = g.q.splits > 1;
    BwdArgs rest = g;  // what the general kernel takes
    if constexpr (sizeof(T) == 2 && DB <= 2) {
        if (kc == 2) {
            ProfScope ps("attn_dkv2", st, 4.0 * one, 0.0);
            if (ks) attn_dkv2_k<DB, true><<<(unsigned)g.kv_blocks, 256, 0, st>>>(g.kv);
            else attn_dkv2_k<DB, false><<<(unsigned)g.kv_blocks, 256, 0, st>>>(g.kv);
            rest.kv_blocks = 0;
        }
        if (qc == 2) {
            ProfScope ps("attn_dq2", st, one, 0.0);
            attn_dq2_k<DB><<<(unsigned)g.q_blocks, 256, 0, st>>>(g.q);
            rest.q_blocks = 0;
        }
    }
    const unsigned grid = (unsigned)(rest.kv_blocks + rest.q_blocks);
    if (grid == 0) return;
    ProfScope ps("attn_bwd", st, ((rest.kv_blocks ? 4 : 0) + (rest.q_blocks ? 1 : 0)) * one, 0.0);
    if (ks && qs) attn_bwd_k<T, DB, true, true><<<grid, 256, 0, st>>>(rest);
    else if (ks) attn_bwd_k<T, DB, true, false><<<grid, 256, 0, st>>>(rest);
    else if (qs) attn_bwd_k<T, DB, false, true><<<grid, 256, 0, st>>>(rest);
    else attn_bwd_k<T, DB, false, false><<<grid, 256, 0, st>>>(rest);
}
template <typename T, int VEC>
static void few_launch(const FewArgs& f, unsigned grid, hipStream_t st) {
    if (f.rows == 1) attn_few_k<T, 1, VEC><<<grid, 256, 0, st>>>(f);
    else if (f.rows == 2) attn_few_k<T, 2, VEC><<<grid, 256, 0, st>>>(f);
    else attn_few_k<T, 4, VEC><<<grid, 256, 0, st>>>(f);
}

rat3d_status attention_fwd(const rat3d_attention_desc& d, const void* q, const void* k,
                           const void* v, const uint8_t* mask, void* o, float* lse, void* ws,
                           hipStream_t st) {
    const AttnPlan p = attn_plan(d, mask != nullptr);
    char* w = (char*)ws;
    AttnArgs a = attn_args(d, p, w);
    a.q = q;
    a.o = o;
    a.lse = lse;
    a.stat = (float*)(w + p.stat);
    a.part = (float*)(w + p.fpart);
    const double nq = (double)d.n * d.heads, nk = (double)d.n * d.kv_heads;
    if (few_rows(d)) {
        FewArgs f = {};
        f.q = q;
        f.k = k;
        f.v = v;
        f.mask = mask;
        f.o = o;
        f.lse = lse;
        f.part = (float*)(w + p.few);
        f.tq = d.tq;
        f.tk = d.tk;
        f.q_stride = a.q_stride;
        f.k_stride = a.k_stride;
        f.v_stride = a.v_stride;
        f.o_stride = a.o_stride;
        f.heads = d.heads;
        f.kv = d.kv_heads;
        f.D = d.head_dim;
        f.rows = (int)(d.heads / d.kv_heads * d.tq);
        f.c = a.c;
        const int keys = few_keys(d);
        f.pieces = (int)ceil_div(d.tk, keys);
        ProfScope ps("attn_few", st, 4.0 * nq * d.tq * d.tk * d.head_dim,
                     2.0 * nk * d.tk * d.head_dim * p.es);
        f.groups = f.rows <= 4 ? 1 : (f.rows + 3) / 4;
        const unsigned grid = (unsigned)((int64_t)d.n * d.kv_heads * f.pieces * f.groups);
        if (d.dtype == RAT3D_BF16) {
            if (keys == 2048) few_launch<bf16, 8>(f, grid, st);
            else few_launch<bf16, 2>(f, grid, st);
            attn_few_join_k<bf16><<<(unsigned)(d.n * d.heads * d.tq), 256, 0, st>>>(f, few_stride(d));
        } else {
            if (keys == 1024) few_launch<float, 4>(f, grid, st);
            else few_launch<float, 1>(f, grid, st);
            attn_few_join_k<float><<<(unsigned)(d.n * d.heads * d.tq), 256, 0, st>>>(f, few_stride(d));
        }
        RAT3D_LAUNCH_CHECK();
        return RAT3D_OK;
    }
    RAT3D_TRY(live_keys(d, p, w, mask, &a, st));
    {
        ProfScope ps("attn_pack", st, 0.0, 4.0 * nk * d.tk * d.head_dim * p.es);
        PackArgs pa = {};
        pa.D = d.head_dim;
        pa.jobs = 2;
        const int nf = 2 * p.DB * p.es / 2;  // fragments of one form
        pa.job[0] = pack_job(k, a.k_stride, d.tk, d.kv_heads, a.kv_rec, 128 * nf, 0, -1, a, true);
        pa.job[1] = pack_job(v, a.v_stride, d.tk, d.kv_heads, a.kv_rec, 128 * nf, -1, nf, a, true);
        pack_mask(d, mask, pa);
        RAT3D_TRY(pack_launch(pa, d.n, p.DB, d.dtype, st));
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
        const unsigned grid =
            (unsigned)((int64_t)d.n * d.heads * ceil_div(d.tq, 64) * ceil_div(d.head_dim, 8));
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
    const AttnPlan p = attn_plan(d, mask != nullptr);
    char* w = (char*)ws;
    AttnArgs a = attn_args(d, p, w);
    a.q_rec = (const u32x4*)(w + p.q_rec);
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
        pa.jobs = 4;
        pa.scale = a.scale;
        const int nf = 2 * p.DB * p.es / 2;  // fragments of one form
        const int ku = 3 * nf * 64, qu = (4 * nf + 1) * 64;
        pa.job[0] = pack_job(k, a.k_stride, d.tk, d.kv_heads, a.kv_rec, ku, 0, 2 * nf, a, true);
        pa.job[1] = pack_job(v, a.v_stride, d.tk, d.kv_heads, a.kv_rec, ku, nf, -1, a, true);
        pack_mask(d, mask, pa);
        if (mask) {
            pa.job[0].zero = dk;
            pa.job[1].zero = dv;
        }
        pa.job[2] = pack_job(q, a.q_stride, d.tq, d.heads, a.q_rec, qu, 0, 2 * nf + 1, a, false);
        pa.job[2].again = 1;
        pa.job[3] = pack_job(dout, a.o_stride, d.tq, d.heads, a.q_rec, qu, nf, 3 * nf + 1, a, false);
        pa.job[3].x = 2 * nf * 64;
        pa.job[3].other = o;
        pa.job[3].lse = lse;
        pa.job[3].lse2 = (float*)(w + p.lse2);
        pa.job[3].delta = (float*)(w + p.delta);
        RAT3D_TRY(pack_launch(pa, d.n, p.DB, d.dtype, st));
    }
    const bool bf = d.dtype == RAT3D_BF16;
    {
        BwdArgs g;
        g.kv = g.q = a;
        g.kv.splits = p.ks;
        g.kv.tiles = (int)ceil_div(d.tk, 128 * p.kc);
        g.kv_blocks = d.n * d.kv_heads * g.kv.tiles * p.ks;
        g.q.part = (float*)(w + p.qpart);
        g.q.splits = p.qs;
        g.q.tiles = (int)ceil_div(d.tq, 128 * p.qc);
        g.q_blocks = d.n * d.heads * g.q.tiles * p.qs;
        RAT3D_ATTN(bwd_launch, d.dtype, p.DB, g, p.kc, p.qc, one, st);
    }
    if (p.ks > 1 || p.qs > 1) {
        SumArgs g = {};
        int64_t blocks = 0;
        auto add = [&](SumJob j) {
            j.tiles = (int)ceil_div(j.tokens, 64);
            j.first = (int)blocks;
            blocks += (int64_t)d.n * j.heads * j.tiles * ceil_div(j.rows, 8);
            g.job[g.jobs++] = j;
        };
        if (p.ks > 1)
            add({(const float*)(w + p.part), dk, dv, a.k_stride, a.v_stride, d.tk, p.tkp, a.idx,
                 a.count, d.kv_heads, d.head_dim, 2 * d.head_dim, p.ks, 0, 0});
        if (p.qs > 1)
            add({(const float*)(w + p.qpart), dq, dq, a.q_stride, a.q_stride, d.tq, p.tqp, nullptr,
                 nullptr, d.heads, d.head_dim, d.head_dim, p.qs, 0, 0});
        ProfScope ps("attn_sum", st, 0.0,
                     4.0 * d.head_dim * (2.0 * nk * d.tk * p.ks + nq * d.tq * p.qs));
        if (bf) attn_sum_k<bf16><<<(unsigned)blocks, 256, 0, st>>>(g);
        else attn_sum_k<float><<<(unsigned)blocks, 256, 0, st>>>(g);
        RAT3D_LAUNCH_CHECK();
    }
    return RAT3D_OK;
}

}  // namespace rat3d
