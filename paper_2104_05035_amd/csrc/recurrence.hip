// Gated linear recurrence along the voxels of a map, a state for each channel:
//   a_t = exp(-w sigmoid(r_t)),  w = rate softplus(lambda),
//   h_t = a_t h_{t-1} + b_t,  b_t = beta_t sigmoid(i_t) x_t,  beta_t = sqrt(1 - a_t^2)
// and y = h.  Masked voxels hand the state on (a = 1, b = 0) and have y = 0.
// Backward, E_t = a_t D_t being what a voxel hands on to the one before it:
//   D_t = dy_t + E_{t+1}  (behind the last voxel dh_last),  dh0 = E of the first,
//   dx = D beta sigmoid(i),  di = dx x (1 - sigmoid(i)),
//   K = D la (a h_{t-1} - sigmoid(i) x a^2 / beta),  la = -w sigmoid(r),
//   dr = K (1 - sigmoid(r)),  dlambda = sigmoid(lambda) / softplus(lambda) sum K
// Both directions are linear recurrences, whose steps (a, b) join associatively:
// (a, b) behind (a', b') is (a a', a b' + b).
//
// Layout: 16 bytes of neighbouring voxels a lane, in the order of memory, so a wave holds
// one block of a row; the walk goes up or down through the lanes.  A lane joins its own
// steps, the 16 lanes of a DPP row theirs, the four rows of a wave are joined by values
// read from single lanes, the waves of a workgroup through LDS: a workgroup takes as many
// blocks at once as it has waves, one barrier a turn, the next turn's loads in flight.
// h_{t-1} is formed again in the backward from the states that the forward left before
// every block, in float32.  Rows of up to 16 lanes share a wave.
// Few rows are cut into segments of one turn: a workgroup leaves its segment's joined
// steps in the workspace, takes those of the segments before it, and goes on with the
// voxels that it holds in registers, so every tensor passes once.  A workgroup waits only
// for ones that drew their segment before it from a counter, so each of them is running
// or done, and none of them waits before it has left its own: every wait ends.  What is
// joined is the same in any order of arrival.  Beyond kSegs segments a launch of its own
// joins each segment's steps first (a workgroup reads all segments before its own, so the
// reads would grow with their square).
//
// beta: 1 - a^2 is -expm1(-2 w sigmoid(r)), by its series where the argument is small.
// Bound: HBM.  Bfloat16, 16 x 64 rows of 48x56x48 voxels: forward 222 us (4.8 TB/s),
// gradient 374 us (4.9), with a mask 242 and 413; 32 such rows, cut, 14 and 27 us.  (Calls
// among others; single kernels under a profiler take 230 and 405.)
#include "kernels.hpp"
#include "prof.hpp"
#include "tokens.hpp"

namespace rat3d {

template <typename T> constexpr int tok() { return 16 / (int)sizeof(T); }  // voxels a lane
template <typename T> constexpr int block() { return 64 * tok<T>(); }      // voxels a wave
constexpr int kWaves = 16;  // of a workgroup, at most
constexpr int kCuts = 64;    // segments of a row that a launch of their own joins, at most
constexpr int kSegs = 2048;  // segments of a row that find one another, at most
constexpr int kPolls = 1 << 22;
constexpr int kLine = 32;    // words of a cache line

struct RecArgs {
    const void *r, *i, *x, *dy;
    const float* lam;
    const uint8_t* mask;
    const float* h0;   // the state (backward: its gradient) that the walk begins with
    void *y, *dr, *di, *dx;
    float *h_last;     // what it ends with
    float *carry, *part;
    // segments: (a, b) of each, [row][segment], and the walk's first state, [row]
    float2* joined;
    float* first;
    uint32_t* drawn;   // segments of each row that workgroups have taken on, a line each
    int64_t sr, si, sx, sy, len;
    int64_t rows;
    int c, blocks, segs, one, lanes, stream;  // of a row; lanes: of a short row
    float rate;
};

// rate softplus(lambda), finite: with an infinite one a shut gate would give 0 times it.
__device__ __forceinline__ float decay_of(float rate, float lam) {
    const float w = rate * (lam > 0.f ? lam + log1pf(expf(-lam)) : log1pf(expf(lam)));
    return w > 1e30f ? 1e30f : w;
}

// One voxel's step.
struct Step {
    float rest, la, a, p;  // rest = 1 - sigmoid(r), p = 1 - a^2
    __device__ __forceinline__ Step(float r, float w) {
        const Sig g(r);
        rest = g.rest;
        la = -w * g.s;
        a = __builtin_amdgcn_exp2f(la * 1.44269504f);
        // -expm1(-t): five terms are off by less than t^5 / 720 = 4e-8 at 1/8, from where
        // on 1 - a^2 is off by 1.5e-6 at most
        const float t = -2.f * la;
        float s = __builtin_fmaf(t, 1.f / 120.f, -1.f / 24.f);
        s = __builtin_fmaf(t, s, 1.f / 6.f);
        s = __builtin_fmaf(t, s, -0.5f);
        s = t * __builtin_fmaf(t, s, 1.f);
        asm volatile("" : "+v"(s));  // formed in every lane: a branch would keep voxels apart
        p = t < 0.125f ? s : __builtin_fmaf(-a, a, 1.f);
    }
};

template <int CTRL> __device__ __forceinline__ float dpp_or(float old, float v) {
    return __uint_as_float(__builtin_amdgcn_update_dpp(__float_as_uint(old), __float_as_uint(v),
                                                       CTRL, 0xf, 0xf, false));
}
__device__ __forceinline__ float lane_of(float v, int lane) {
    return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v), lane));
}

// The steps of a wave's lanes joined in the order of a walk up (or DOWN) the lanes.
template <bool DOWN> struct WaveWalk {
    float a, b;        // this lane's and all before it in its row of 16
    float ra[4], rb[4];  // the rows, in the walk's order
    __device__ __forceinline__ WaveWalk(float a_, float b_) : a(a_), b(b_) {
        constexpr int SH = DOWN ? 0x100 : 0x110;  // row_shl, row_shr
        join<SH + 1>();
        join<SH + 2>();
        join<SH + 4>();
        join<SH + 8>();
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int last = DOWN ? 16 * (3 - k) : 16 * k + 15;
            ra[k] = lane_of(a, last);
            rb[k] = lane_of(b, last);
        }
    }
    template <int CTRL> __device__ __forceinline__ void join() {
        const float pa = dpp_or<CTRL>(1.f, a), pb = dpp_or<CTRL>(0.f, b);
        b = __builtin_fmaf(a, pb, b);
        a *= pa;
    }
    // the whole wave
    __device__ __forceinline__ float2 all() const {
        float A = ra[0], B = rb[0];
#pragma unroll
        for (int k = 1; k < 4; ++k) {
            B = __builtin_fmaf(ra[k], B, rb[k]);
            A *= ra[k];
        }
        return make_float2(A, B);
    }
    // what this lane begins with, if the wave begins with s
    __device__ __forceinline__ float begin(float s) const {
        const int row = (threadIdx.x >> 4) & 3, k = DOWN ? 3 - row : row;
        float t = s;
#pragma unroll
        for (int j = 0; j < 3; ++j) {
            s = __builtin_fmaf(ra[j], s, rb[j]);
            t = k > j ? s : t;
        }
        constexpr int BY1 = DOWN ? 0x101 : 0x111;
        return __builtin_fmaf(dpp_or<BY1>(1.f, a), t, dpp_or<BY1>(0.f, b));
    }
};

// A lane's voxels of a row, `at` the first of them, `over` of them behind the row's end.
// They are read from `from` on, no further than the end (a row has at least as many), and
// shifted; stores leave them out.
template <typename T> struct Place {
    int64_t at, from;
    int over;
    uint32_t live;  // bit j: voxel at + j is there and not masked
    template <bool ALL> __device__ __forceinline__ void find(int64_t v, int64_t len) {
        constexpr int TOK = tok<T>();
        at = from = v;
        over = 0;
        live = (1u << TOK) - 1u;
        if (!ALL && v + TOK > len) {
            from = len - TOK;
            over = v >= len ? TOK : (int)(v - from);
            live >>= over;
        }
    }
    template <bool ALL>
    __device__ __forceinline__ Toks<T, tok<T>()> load(const T* row) const {
        Toks<T, tok<T>()> t;
        t.load(row + (ALL ? at : from), 0);
        if (!ALL) t.shift(over);
        return t;
    }
    __device__ __forceinline__ void apply(const uint8_t* mask) {
        constexpr int TOK = tok<T>();
        struct __attribute__((packed, aligned(1))) Bytes { uint32_t w[TOK / 4]; };
        const Bytes m = *reinterpret_cast<const Bytes*>(mask + from);
        uint32_t on = 0;
#pragma unroll
        for (int j = 0; j < TOK; ++j) on |= (m.w[j / 4] >> (8 * (j & 3)) & 0xffu ? 1u : 0u) << j;
        live &= on >> over;
    }
    // 0 where nothing is to be stored but a zero
    __device__ __forceinline__ void clear(float (&o)[tok<T>()]) const {
#pragma unroll
        for (int j = 0; j < tok<T>(); ++j) o[j] = live >> j & 1u ? o[j] : 0.f;
    }
};

// Raw inputs of a lane's voxels.  A row shorter than a lane's voxels is read by elements.
template <typename T, int N> struct Raw {
    Toks<T, tok<T>()> t[N];
    Place<T> at;
};
template <typename T, int N, bool ALL>
__device__ __forceinline__ void read(Raw<T, N>& d, const T* const (&row)[N], const uint8_t* mask,
                                     int64_t v, int64_t len) {
    d.at.template find<ALL>(v, len);
#pragma unroll
    for (int i = 0; i < N; ++i) d.t[i] = d.at.template load<ALL>(row[i]);
    if (!ALL && mask) d.at.apply(mask);
}

// What the forward needs of a lane's voxels: the steps.
template <typename T> struct Steps {
    static constexpr int TOK = tok<T>();
    float a[TOK], b[TOK];
    // r, i, x as they lie; ALL: every voxel counts
    template <bool ALL> __device__ __forceinline__ void form(const Raw<T, 3>& d, float w) {
#pragma unroll
        for (int j = 0; j < TOK; ++j) {
            const Step s(d.t[0][j], w);
            const bool is = ALL || d.at.live >> j & 1u;
            a[j] = is ? s.a : 1.f;
            b[j] = is ? __builtin_amdgcn_sqrtf(s.p) * Sig(d.t[1][j]).s * d.t[2][j] : 0.f;
        }
    }
    template <bool DOWN> __device__ __forceinline__ float2 all() const {
        float A = 1.f, B = 0.f;
#pragma unroll
        for (int k = 0; k < TOK; ++k) {
            const int j = DOWN ? TOK - 1 - k : k;
            B = __builtin_fmaf(a[j], B, b[j]);
            A *= a[j];
        }
        return make_float2(A, B);
    }
    // the states behind a lane's voxels, from that before them
    template <bool DOWN> __device__ __forceinline__ void states(float h, float (&o)[TOK]) const {
#pragma unroll
        for (int k = 0; k < TOK; ++k) {
            const int j = DOWN ? TOK - 1 - k : k;
            h = __builtin_fmaf(a[j], h, b[j]);
            o[j] = h;
        }
    }
};

// What the backward needs: the steps, and the factors of the gradients.  DOWN is the way
// of the gradient's walk, against the forward's.
template <typename T, bool DOWN> struct GradSteps {
    static constexpr int TOK = tok<T>();
    float a[TOK], la[TOK], m[TOK], g[TOK], rr[TOK], ri[TOK], x[TOK], d[TOK];
    // r, i, x, dy as they lie
    template <bool ALL> __device__ __forceinline__ void form(const Raw<T, 4>& q, float w) {
#pragma unroll
        for (int j = 0; j < TOK; ++j) {
            const Step s(q.t[0][j], w);
            const Sig gi(q.t[1][j]);
            // at p = 0 (a shut gate) la inv and p inv come out as 0, their limits; a root
            // of less than the smallest normal number would be infinite
            const float inv = __builtin_amdgcn_rsqf(s.p < 0x1p-126f ? 0x1p-126f : s.p);
            const bool is = ALL || q.at.live >> j & 1u;
            a[j] = is ? s.a : 1.f;
            la[j] = is ? s.la * s.a : 0.f;                        // by the past state
            m[j] = is ? gi.s * (s.a * s.a) * (s.la * inv) : 0.f;  // by x
            g[j] = is ? s.p * inv * gi.s : 0.f;                   // beta sigmoid(i)
            rr[j] = is ? s.rest : 0.f;
            ri[j] = is ? gi.rest : 0.f;
            x[j] = is ? q.t[2][j] : 0.f;
            d[j] = is ? q.t[3][j] : 0.f;
        }
    }
    // the lane's steps of the gradient's walk, and the inhomogeneous part of the forward's
    __device__ __forceinline__ void all(float& A, float& B, float& F) const {
        A = 1.f;
        B = F = 0.f;
#pragma unroll
        for (int k = 0; k < TOK; ++k) {
            const int j = DOWN ? TOK - 1 - k : k, i = DOWN ? k : TOK - 1 - k;
            A *= a[j];
            B = a[j] * (d[j] + B);
            F = __builtin_fmaf(a[i], F, g[i] * x[i]);
        }
    }
    // dr, di, dx from E behind the lane's voxels and h before them; returns the sum of K.
    // Where no voxel is live the caller drops it: the factors are 0, but a state or gradient
    // that is handed on need not be finite.
    __device__ __forceinline__ float grads(float E, float h, float (&dr)[TOK], float (&di)[TOK],
                                           float (&dx)[TOK]) const {
#pragma unroll
        for (int k = 0; k < TOK; ++k) {  // dr holds la a h_{t-1} first
            const int j = DOWN ? k : TOK - 1 - k;
            dr[j] = la[j] * h;
            h = __builtin_fmaf(a[j], h, g[j] * x[j]);
        }
        float sum = 0.f;
#pragma unroll
        for (int k = 0; k < TOK; ++k) {
            const int j = DOWN ? TOK - 1 - k : k;
            const float D = d[j] + E;
            E = a[j] * D;
            const float K = D * __builtin_fmaf(-m[j], x[j], dr[j]);
            sum += K;
            dr[j] = K * rr[j];
            dx[j] = D * g[j];
            di[j] = dx[j] * x[j] * ri[j];
        }
        return sum;
    }
};

// The walk's state at the beginning of a segment: the segments before it joined, one a
// lane, so that their loads are under way together.
__device__ __forceinline__ float segment_begin(const RecArgs& q, int64_t row, int seg) {
    static_assert(kCuts <= 64, "a segment a lane");
    if (q.segs == 1) return q.h0 ? q.h0[row] : 0.f;
    const int lane = threadIdx.x & 63;
    const float2 o = q.joined[row * q.segs + (lane < seg ? lane : 0)];
    const float s = q.first[row];
    const float2 all = WaveWalk<false>(lane < seg ? o.x : 1.f, lane < seg ? o.y : 0.f).all();
    return __builtin_fmaf(all.x, s, all.y);
}

// The blocks of a segment, first to last in the order of the walk.
struct Segment {
    int first, count;  // `first` counted in the walk's order
    __device__ __forceinline__ Segment(const RecArgs& q, int seg) {
        const int size = (q.blocks + q.segs - 1) / q.segs;
        first = seg * size;
        count = q.blocks - first < size ? q.blocks - first : size;
        if (count < 0) count = 0;
    }
};

// Rows beyond 16 lanes: a workgroup a segment of a row.  JOIN: only the segments' steps.
template <typename T, bool DOWN, bool JOIN>
__global__ __launch_bounds__(64 * kWaves, 8) void recurrence_fwd_k(RecArgs q) {
    constexpr int TOK = tok<T>(), BLOCK = block<T>();
    __shared__ float2 tot[2][kWaves];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int waves = blockDim.x >> 6;
    const uint32_t row_ = blockIdx.x / (uint32_t)q.segs, vol_ = row_ / (uint32_t)q.c;
    const int seg = (int)(blockIdx.x - row_ * q.segs), ch = (int)(row_ - vol_ * q.c);
    const int64_t row = row_, vol = vol_;
    const float lam = q.lam[ch];
    const T* const in[3] = {(const T*)q.r + vol * q.sr + (int64_t)ch * q.len,
                            (const T*)q.i + vol * q.si + (int64_t)ch * q.len,
                            (const T*)q.x + vol * q.sx + (int64_t)ch * q.len};
    T* y = (T*)q.y + vol * q.sy + (int64_t)ch * q.len;
    const uint8_t* mask = q.mask ? q.mask + vol * q.len : nullptr;
    const Segment sg(q, seg);
    auto place = [&](int k) {  // the block in memory of the walk's k-th
        return DOWN ? q.blocks - 1 - (sg.first + k) : sg.first + k;
    };
    auto whole = [&](int k) { return !mask && (int64_t)(place(k) + 1) * BLOCK <= q.len; };
    Raw<T, 3> cur, nxt;
    auto fetch = [&](Raw<T, 3>& d, int k) {
        if (k >= sg.count) return;
        const int64_t v = (int64_t)place(k) * BLOCK + lane * TOK;
        if (whole(k)) read<T, 3, true>(d, in, mask, v, q.len);
        else read<T, 3, false>(d, in, mask, v, q.len);
    };
    fetch(cur, wave);  // under way while the walk's beginning is found
    const float w = decay_of(q.rate, lam);
    float state = JOIN ? 0.f : segment_begin(q, row, seg), prod = 1.f;
    int par = 0;
    for (int k0 = 0; k0 < sg.count; k0 += waves, par ^= 1) {
        const int k = k0 + wave;
        fetch(nxt, k + waves);
        const bool all = k < sg.count && whole(k);
        Steps<T> s;
        if (k >= sg.count) cur.at.live = 0;  // steps that change nothing
        if (all) s.template form<true>(cur, w);
        else s.template form<false>(cur, w);
        const float2 mine = s.template all<DOWN>();
        const WaveWalk<DOWN> walk(mine.x, mine.y);
        if (lane == 0) tot[par][wave] = walk.all();
        __syncthreads();  // one a turn: the next turn writes the other half
        float begin = state;
        for (int j = 0; j < waves; ++j) {
            const float2 o = tot[par][j];
            if (j == wave) begin = state;
            state = __builtin_fmaf(o.x, state, o.y);
            if (JOIN) prod *= o.x;
        }
        if (!JOIN && k < sg.count) {
            if (q.carry && lane == 0) q.carry[row * q.blocks + place(k)] = begin;
            float o[TOK];
            s.template states<DOWN>(walk.begin(begin), o);
            if (all) {
                put_tokens<T, TOK, true>(y + cur.at.at, 0, TOK, o, q.stream);
            } else {
                cur.at.clear(o);
                put_tokens<T, TOK, false>(y + cur.at.at, 0, TOK - cur.at.over, o, q.stream);
            }
        }
        cur = nxt;
    }
    if (threadIdx.x == 0) {
        if (JOIN) {
            q.joined[row * q.segs + seg] = make_float2(prod, state);
            // kept, for the walk's last state may take the first one's place
            if (seg == 0) q.first[row] = q.h0 ? q.h0[row] : 0.f;
        } else if (q.h_last && seg == q.segs - 1) {
            q.h_last[row] = state;
        }
    }
}

// DOWN: the way of the gradient's walk, against that of the forward.
template <typename T, bool DOWN>
__global__ __launch_bounds__(64 * kWaves, 4) void recurrence_bwd_k(RecArgs q) {
    constexpr int TOK = tok<T>(), BLOCK = block<T>();
    __shared__ float2 tot[2][kWaves];
    __shared__ double sums[kWaves];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int waves = blockDim.x >> 6;
    const uint32_t row_ = blockIdx.x / (uint32_t)q.segs, vol_ = row_ / (uint32_t)q.c;
    const int seg = (int)(blockIdx.x - row_ * q.segs), ch = (int)(row_ - vol_ * q.c);
    const int64_t row = row_, vol = vol_;
    const float lam = q.lam[ch];
    const T* const in[4] = {(const T*)q.r + vol * q.sr + (int64_t)ch * q.len,
                            (const T*)q.i + vol * q.si + (int64_t)ch * q.len,
                            (const T*)q.x + vol * q.sx + (int64_t)ch * q.len,
                            (const T*)q.dy + vol * q.sy + (int64_t)ch * q.len};
    T* dr = (T*)q.dr + vol * q.sr + (int64_t)ch * q.len;
    T* di = (T*)q.di + vol * q.si + (int64_t)ch * q.len;
    T* dx = (T*)q.dx + vol * q.sx + (int64_t)ch * q.len;
    const uint8_t* mask = q.mask ? q.mask + vol * q.len : nullptr;
    const Segment sg(q, seg);
    auto place = [&](int k) { return DOWN ? q.blocks - 1 - (sg.first + k) : sg.first + k; };
    auto whole = [&](int k) { return !mask && (int64_t)(place(k) + 1) * BLOCK <= q.len; };
    Raw<T, 4> cur, nxt;
    float past0 = 0.f, past1 = 0.f;  // the states before the blocks
    auto fetch = [&](Raw<T, 4>& d, float& past, int k) {
        if (k >= sg.count) return;
        past = q.carry[row * q.blocks + place(k)];
        const int64_t v = (int64_t)place(k) * BLOCK + lane * TOK;
        if (whole(k)) read<T, 4, true>(d, in, mask, v, q.len);
        else read<T, 4, false>(d, in, mask, v, q.len);
    };
    fetch(cur, past0, wave);
    const float w = decay_of(q.rate, lam);
    float state = segment_begin(q, row, seg);  // E
    double sum = 0.0;
    int par = 0;
    for (int k0 = 0; k0 < sg.count; k0 += waves, par ^= 1) {
        const int k = k0 + wave;
        fetch(nxt, past1, k + waves);
        const bool all = k < sg.count && whole(k);
        GradSteps<T, DOWN> s;
        if (k >= sg.count) cur.at.live = 0;
        if (all) s.template form<true>(cur, w);
        else s.template form<false>(cur, w);
        float A, B, F;
        s.all(A, B, F);
        const WaveWalk<DOWN> walk(A, B);
        if (lane == 0) tot[par][wave] = walk.all();
        const float h = WaveWalk<!DOWN>(A, F).begin(past0);
        __syncthreads();
        float begin = state;
        for (int j = 0; j < waves; ++j) {
            const float2 o = tot[par][j];
            if (j == wave) begin = state;
            state = __builtin_fmaf(o.x, state, o.y);
        }
        if (k < sg.count) {
            float o[3][TOK];
            const float K = s.grads(walk.begin(begin), h, o[0], o[1], o[2]);
            sum += (double)(all || cur.at.live ? K : 0.f);
            auto put = [&](auto all) {
                constexpr bool ALL = decltype(all)::value;
                const int left = TOK - cur.at.over;
                if (!ALL)
                    for (auto& v : o) cur.at.clear(v);
                put_tokens<T, TOK, ALL>(dr + cur.at.at, 0, left, o[0], q.stream);
                put_tokens<T, TOK, ALL>(di + cur.at.at, 0, left, o[1], q.stream);
                put_tokens<T, TOK, ALL>(dx + cur.at.at, 0, left, o[2], q.stream);
            };
            if (all) put(std::true_type{});
            else put(std::false_type{});
        }
        cur = nxt;
        past0 = past1;
    }
#pragma unroll
    for (int m = 32; m >= 1; m >>= 1) sum += __shfl_xor(sum, m);
    if (lane == 0) sums[wave] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int j = 1; j < waves; ++j) sum += sums[j];
        q.part[(int64_t)ch * (q.rows / q.c) * q.segs + vol * q.segs + seg] = (float)sum;
        if (q.h_last && seg == q.segs - 1) q.h_last[row] = state;
    }
}

// The gradient's walk through each segment: decays, and what reaches its end from dy.
template <typename T, bool DOWN>
__global__ __launch_bounds__(64 * kWaves) void recurrence_bwd_join_k(RecArgs q) {
    constexpr int TOK = tok<T>(), BLOCK = block<T>();
    __shared__ float2 tot[2][kWaves];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int waves = blockDim.x >> 6;
    const uint32_t row_ = blockIdx.x / (uint32_t)q.segs, vol_ = row_ / (uint32_t)q.c;
    const int seg = (int)(blockIdx.x - row_ * q.segs), ch = (int)(row_ - vol_ * q.c);
    const int64_t row = row_, vol = vol_;
    const float lam = q.lam[ch];
    const T* const in[2] = {(const T*)q.r + vol * q.sr + (int64_t)ch * q.len,
                            (const T*)q.dy + vol * q.sy + (int64_t)ch * q.len};
    const uint8_t* mask = q.mask ? q.mask + vol * q.len : nullptr;
    const Segment sg(q, seg);
    const float w = decay_of(q.rate, lam);
    float state = 0.f, prod = 1.f;
    int par = 0;
    for (int k0 = 0; k0 < sg.count; k0 += waves, par ^= 1) {
        const int k = k0 + wave;
        float A = 1.f, B = 0.f;
        if (k < sg.count) {
            const int at = DOWN ? q.blocks - 1 - (sg.first + k) : sg.first + k;
            Raw<T, 2> d;
            read<T, 2, false>(d, in, mask, (int64_t)at * BLOCK + lane * TOK, q.len);
#pragma unroll
            for (int e = 0; e < TOK; ++e) {
                const int j = DOWN ? TOK - 1 - e : e;
                const float a = __builtin_amdgcn_exp2f(-w * Sig(d.t[0][j]).s * 1.44269504f);
                const bool is = d.at.live >> j & 1u;
                B = is ? a * (d.t[1][j] + B) : B;
                A = is ? A * a : A;
            }
        }
        const WaveWalk<DOWN> walk(A, B);
        if (lane == 0) tot[par][wave] = walk.all();
        __syncthreads();
        for (int j = 0; j < waves; ++j) {
            const float2 o = tot[par][j];
            state = __builtin_fmaf(o.x, state, o.y);
            prod *= o.x;
        }
    }
    if (threadIdx.x == 0) {
        q.joined[row * q.segs + seg] = make_float2(prod, state);
        if (seg == 0) q.first[row] = q.h0 ? q.h0[row] : 0.f;
    }
}

// Before the segments that find one another: nothing drawn, nothing joined, and the walks'
// first states, for their last ones may take their place.
__global__ __launch_bounds__(256) void recurrence_begin_k(RecArgs q) {
    const int64_t k = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (k < q.rows * q.segs) q.joined[k] = make_float2(0.f, 0.f);
    if (k < q.rows) {
        q.drawn[k * kLine] = 0;
        q.first[k] = q.h0 ? q.h0[k] : 0.f;
    }
}

// A workgroup's segment of one turn.  (a, b) lie in one word of 64 bits, so that they
// arrive together; a is never negative, and its sign bit says that they are there.
struct OneTurn {
    int64_t row;
    int seg, wave, waves;
    float pa, pb;  // the waves before this one, joined

    __device__ __forceinline__ OneTurn(const RecArgs& q, int* draw)
        : wave(__builtin_amdgcn_readfirstlane(threadIdx.x >> 6)), waves(blockDim.x >> 6) {
        // a counter a row: one for all took 15 us for 1000 workgroups
        row = blockIdx.x % (uint32_t)q.rows;
        if (threadIdx.x == 0)
            *draw = (int)__hip_atomic_fetch_add(q.drawn + row * kLine, 1u, __ATOMIC_RELAXED,
                                                __HIP_MEMORY_SCOPE_AGENT);
        __syncthreads();
        seg = __builtin_amdgcn_readfirstlane(*draw);
    }
    // the block in the walk's order
    __device__ __forceinline__ int block() const { return seg * waves + wave; }
    // Joins the waves' steps, leaves the segment's, and returns what the wave begins with;
    // `end` becomes what the segment ends with.
    __device__ __forceinline__ float begin(const RecArgs& q, float2 mine, float2* tot,
                                           float* from, float& end) {
        const int lane = threadIdx.x & 63;
        if (lane == 0) tot[wave] = mine;
        __syncthreads();
        float A = 1.f, B = 0.f;
        for (int j = 0; j < waves; ++j) {
            if (j == wave) {
                pa = A;
                pb = B;
            }
            const float2 o = tot[j];
            B = __builtin_fmaf(o.x, B, o.y);
            A *= o.x;
        }
        if (wave == 0) {
            uint64_t* to = (uint64_t*)q.joined + row * q.segs;
            const uint64_t there = (uint64_t)1 << 63;
            if (lane == 0)
                __hip_atomic_store(to + seg,
                                   there | (uint64_t)__float_as_uint(A) << 32 | __float_as_uint(B),
                                   __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            float s = q.first[row];
            for (int k0 = 0; k0 < seg; k0 += 64) {  // the segments before, one a lane
                uint64_t v = (uint64_t)0x3f800000u << 32;
                if (k0 + lane < seg) {
                    for (int i = 0; i < kPolls; ++i) {
                        v = __hip_atomic_load(to + k0 + lane, __ATOMIC_RELAXED,
                                              __HIP_MEMORY_SCOPE_AGENT);
                        if (v & there) break;
                        __builtin_amdgcn_s_sleep(1);
                    }
                    if (!(v & there)) v = (uint64_t)0x7fc00000u << 32;  // NaN: no wait is endless
                }
                const WaveWalk<false> all(__uint_as_float((uint32_t)(v >> 32) & 0x7fffffffu),
                                          __uint_as_float((uint32_t)v));
                const float2 o = all.all();
                s = __builtin_fmaf(o.x, s, o.y);
            }
            if (lane == 0) *from = s;
        }
        __syncthreads();
        const float s = *from;
        end = __builtin_fmaf(A, s, B);
        return __builtin_fmaf(pa, s, pb);
    }
};

template <typename T, bool DOWN>
__global__ __launch_bounds__(64 * kWaves, 8) void recurrence_fwd_one_k(RecArgs q) {
    constexpr int TOK = tok<T>(), BLOCK = block<T>();
    __shared__ float2 tot[kWaves];
    __shared__ float from;
    __shared__ int draw;
    OneTurn turn(q, &draw);
    const int lane = threadIdx.x & 63;
    const int64_t row = turn.row, vol = (uint32_t)row / (uint32_t)q.c;
    const int ch = (int)(row - vol * q.c);
    const float lam = q.lam[ch];
    const T* const in[3] = {(const T*)q.r + vol * q.sr + (int64_t)ch * q.len,
                            (const T*)q.i + vol * q.si + (int64_t)ch * q.len,
                            (const T*)q.x + vol * q.sx + (int64_t)ch * q.len};
    const uint8_t* mask = q.mask ? q.mask + vol * q.len : nullptr;
    const int k = turn.block(), at = DOWN ? q.blocks - 1 - k : k;
    const bool there = k < q.blocks, all = there && !mask && (int64_t)(at + 1) * BLOCK <= q.len;
    Raw<T, 3> d;
    d.at.live = 0;
    const int64_t v = (int64_t)at * BLOCK + lane * TOK;
    if (all) read<T, 3, true>(d, in, mask, v, q.len);
    else if (there) read<T, 3, false>(d, in, mask, v, q.len);
    const float w = decay_of(q.rate, lam);
    Steps<T> s;
    if (all) s.template form<true>(d, w);
    else s.template form<false>(d, w);
    const float2 mine = s.template all<DOWN>();
    const WaveWalk<DOWN> walk(mine.x, mine.y);
    float end;
    const float begin = turn.begin(q, walk.all(), tot, &from, end);
    if (there) {
        if (q.carry && lane == 0) q.carry[row * q.blocks + at] = begin;
        T* y = (T*)q.y + vol * q.sy + (int64_t)ch * q.len;
        float o[TOK];
        s.template states<DOWN>(walk.begin(begin), o);
        if (all) {
            put_tokens<T, TOK, true>(y + d.at.at, 0, TOK, o, q.stream);
        } else {
            d.at.clear(o);
            put_tokens<T, TOK, false>(y + d.at.at, 0, TOK - d.at.over, o, q.stream);
        }
    }
    if (q.h_last && turn.seg == q.segs - 1 && threadIdx.x == 0) q.h_last[row] = end;
}

template <typename T, bool DOWN>
__global__ __launch_bounds__(64 * kWaves, 4) void recurrence_bwd_one_k(RecArgs q) {
    constexpr int TOK = tok<T>(), BLOCK = block<T>();
    __shared__ float2 tot[kWaves];
    __shared__ double sums[kWaves];
    __shared__ float from;
    __shared__ int draw;
    OneTurn turn(q, &draw);
    const int lane = threadIdx.x & 63;
    const int64_t row = turn.row, vol = (uint32_t)row / (uint32_t)q.c;
    const int ch = (int)(row - vol * q.c);
    const float lam = q.lam[ch];
    const T* const in[4] = {(const T*)q.r + vol * q.sr + (int64_t)ch * q.len,
                            (const T*)q.i + vol * q.si + (int64_t)ch * q.len,
                            (const T*)q.x + vol * q.sx + (int64_t)ch * q.len,
                            (const T*)q.dy + vol * q.sy + (int64_t)ch * q.len};
    const uint8_t* mask = q.mask ? q.mask + vol * q.len : nullptr;
    const int k = turn.block(), at = DOWN ? q.blocks - 1 - k : k;
    const bool there = k < q.blocks, all = there && !mask && (int64_t)(at + 1) * BLOCK <= q.len;
    Raw<T, 4> d;
    d.at.live = 0;
    float past = 0.f;
    if (there) past = q.carry[row * q.blocks + at];
    const int64_t v = (int64_t)at * BLOCK + lane * TOK;
    if (all) read<T, 4, true>(d, in, mask, v, q.len);
    else if (there) read<T, 4, false>(d, in, mask, v, q.len);
    const float w = decay_of(q.rate, lam);
    GradSteps<T, DOWN> s;
    if (all) s.template form<true>(d, w);
    else s.template form<false>(d, w);
    float A, B, F, end;
    s.all(A, B, F);
    const WaveWalk<DOWN> walk(A, B);
    const float h = WaveWalk<!DOWN>(A, F).begin(past);
    const float begin = turn.begin(q, walk.all(), tot, &from, end);
    double sum = 0.0;
    if (there) {
        float o[3][TOK];
        const float K = s.grads(walk.begin(begin), h, o[0], o[1], o[2]);
        sum = (double)(all || d.at.live ? K : 0.f);
        T* const out[3] = {(T*)q.dr + vol * q.sr + (int64_t)ch * q.len,
                           (T*)q.di + vol * q.si + (int64_t)ch * q.len,
                           (T*)q.dx + vol * q.sx + (int64_t)ch * q.len};
        if (all) {
#pragma unroll
            for (int i = 0; i < 3; ++i)
                put_tokens<T, TOK, true>(out[i] + d.at.at, 0, TOK, o[i], q.stream);
        } else {
#pragma unroll
            for (int i = 0; i < 3; ++i) {
                d.at.clear(o[i]);
                put_tokens<T, TOK, false>(out[i] + d.at.at, 0, TOK - d.at.over, o[i], q.stream);
            }
        }
    }
#pragma unroll
    for (int m = 32; m >= 1; m >>= 1) sum += __shfl_xor(sum, m);
    if (lane == 0) sums[turn.wave] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int j = 1; j < turn.waves; ++j) sum += sums[j];
        q.part[((int64_t)ch * (q.rows / q.c) + vol) * q.segs + turn.seg] = (float)sum;
        if (q.h_last && turn.seg == q.segs - 1) q.h_last[row] = end;
    }
}

// Rows of up to 16 lanes: several a wave, each on `lanes` (a power of two) of them.
template <typename T, int N>
__device__ __forceinline__ void read_short(Raw<T, N>& d, const T* const (&row)[N],
                                           const uint8_t* mask, int64_t v, int64_t len) {
    constexpr int TOK = tok<T>();
    if (len >= TOK) {
        read<T, N, false>(d, row, mask, v, len);
        return;
    }
    // by elements, those behind the end as the last one
    d.at.template find<false>(v, len);
#pragma unroll
    for (int i = 0; i < N; ++i) {
        T e[TOK];
#pragma unroll
        for (int j = 0; j < TOK; ++j) e[j] = row[i][j < len ? j : len - 1];
#pragma unroll
        for (int j = 0; j < TOK; ++j) {
            if constexpr (sizeof(T) == 4) d.t[i].u.w[j] = __float_as_uint(e[j]);
            else if (j & 1) d.t[i].u.w[j / 2] |= (uint32_t)e[j] << 16;
            else d.t[i].u.w[j / 2] = e[j];
        }
    }
    if (mask)
#pragma unroll
        for (int j = 0; j < TOK; ++j)
            if (!mask[j < len ? j : len - 1]) d.at.live &= ~(1u << j);
}

// Joins the lanes of each row up (or DOWN) and returns what the lane begins with if its
// row begins with s; s becomes what the row ends with.
template <bool DOWN> __device__ __forceinline__ float short_walk(float a, float b, int lanes, float& s) {
    const int lane = threadIdx.x & (lanes - 1), k = DOWN ? lanes - 1 - lane : lane;
    for (int m = 1; m < lanes; m <<= 1) {
        const float pa = DOWN ? __shfl_down(a, m) : __shfl_up(a, m);
        const float pb = DOWN ? __shfl_down(b, m) : __shfl_up(b, m);
        if (k >= m) {
            b = __builtin_fmaf(a, pb, b);
            a *= pa;
        }
    }
    const float end = __builtin_fmaf(a, s, b);
    const float before = DOWN ? __shfl_down(end, 1) : __shfl_up(end, 1);
    const float begin = k == 0 ? s : before;
    s = __shfl(end, (threadIdx.x & 63) - lane + (DOWN ? 0 : lanes - 1));
    return begin;
}

template <typename T, bool DOWN>
__global__ __launch_bounds__(256) void recurrence_short_fwd_k(RecArgs q) {
    constexpr int TOK = tok<T>();
    const uint32_t id = blockIdx.x * 256 + threadIdx.x;
    const int64_t r_ = id >> (31 - __builtin_clz(q.lanes)), row = r_ < q.rows ? r_ : q.rows - 1;
    const int lane = (int)(id & (q.lanes - 1));
    const int64_t vol = (uint32_t)row / (uint32_t)q.c;
    const int ch = (int)(row - vol * q.c);
    const float lam = q.lam[ch];
    const T* const in[3] = {(const T*)q.r + vol * q.sr + (int64_t)ch * q.len,
                            (const T*)q.i + vol * q.si + (int64_t)ch * q.len,
                            (const T*)q.x + vol * q.sx + (int64_t)ch * q.len};
    Raw<T, 3> d;
    read_short<T, 3>(d, in, q.mask ? q.mask + vol * q.len : nullptr, lane * TOK, q.len);
    float state = q.h0 ? q.h0[row] : 0.f;
    const float first = state;
    Steps<T> s;
    s.template form<false>(d, decay_of(q.rate, lam));
    const float2 mine = s.template all<DOWN>();
    float o[TOK];
    s.template states<DOWN>(short_walk<DOWN>(mine.x, mine.y, q.lanes, state), o);
    d.at.clear(o);
    if (r_ >= q.rows) return;
    put_tokens<T, TOK, false>((T*)q.y + vol * q.sy + (int64_t)ch * q.len + d.at.at, 0,
                              TOK - d.at.over, o, false);
    if (lane == 0) {
        if (q.carry) q.carry[row] = first;
        if (q.h_last) q.h_last[row] = state;
    }
}

template <typename T, bool DOWN>
__global__ __launch_bounds__(256) void recurrence_short_bwd_k(RecArgs q) {
    constexpr int TOK = tok<T>();
    const uint32_t id = blockIdx.x * 256 + threadIdx.x;
    const int64_t r_ = id >> (31 - __builtin_clz(q.lanes)), row = r_ < q.rows ? r_ : q.rows - 1;
    const int lane = (int)(id & (q.lanes - 1));
    const int64_t vol = (uint32_t)row / (uint32_t)q.c;
    const int ch = (int)(row - vol * q.c);
    const float lam = q.lam[ch];
    const T* const in[4] = {(const T*)q.r + vol * q.sr + (int64_t)ch * q.len,
                            (const T*)q.i + vol * q.si + (int64_t)ch * q.len,
                            (const T*)q.x + vol * q.sx + (int64_t)ch * q.len,
                            (const T*)q.dy + vol * q.sy + (int64_t)ch * q.len};
    Raw<T, 4> d;
    read_short<T, 4>(d, in, q.mask ? q.mask + vol * q.len : nullptr, lane * TOK, q.len);
    GradSteps<T, DOWN> s;
    s.template form<false>(d, decay_of(q.rate, lam));
    float A, B, F;
    s.all(A, B, F);
    float state = q.h0 ? q.h0[row] : 0.f, fwd = q.carry[row];
    const float E = short_walk<DOWN>(A, B, q.lanes, state);
    const float h = short_walk<!DOWN>(A, F, q.lanes, fwd);
    float o[3][TOK];
    float part = s.grads(E, h, o[0], o[1], o[2]);
    if (!d.at.live) part = 0.f;
    for (auto& v : o) d.at.clear(v);
    for (int m = q.lanes / 2; m >= 1; m >>= 1) part += __shfl_xor(part, m);
    if (r_ >= q.rows) return;
    const int64_t at = (int64_t)ch * q.len + d.at.at;
    const int left = TOK - d.at.over;
    put_tokens<T, TOK, false>((T*)q.dr + vol * q.sr + at, 0, left, o[0], false);
    put_tokens<T, TOK, false>((T*)q.di + vol * q.si + at, 0, left, o[1], false);
    put_tokens<T, TOK, false>((T*)q.dx + vol * q.sx + at, 0, left, o[2], false);
    if (lane == 0) {
        q.part[(int64_t)ch * (q.rows / q.c) + vol] = part;
        if (q.h_last) q.h_last[row] = state;
    }
}

// dlambda (+)= sigmoid(lambda) / softplus(lambda) times the sum of K, its parts added in
// float64 in a fixed order.  Far below zero the ratio is 1.
__global__ __launch_bounds__(256) void recurrence_lambda_k(const float* __restrict__ part,
                                                           int parts, const float* lam,
                                                           float* dlam, int accumulate) {
    __shared__ double red[4];
    const int ch = blockIdx.x;
    double s = 0.0;
    for (int i = threadIdx.x; i < parts; i += 256) s += (double)part[(int64_t)ch * parts + i];
#pragma unroll
    for (int m = 32; m >= 1; m >>= 1) s += __shfl_xor(s, m);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
    __syncthreads();
    if (threadIdx.x == 0) {
        const double v = (double)lam[ch], e = exp(v < 0.0 ? v : -v);
        const double ratio = v < -40.0 ? 1.0 : (v < 0.0 ? e : 1.0) / (1.0 + e) / (log1p(e) + (v > 0.0 ? v : 0.0));
        s = ((red[0] + red[1]) + (red[2] + red[3])) * ratio;
        dlam[ch] = accumulate ? dlam[ch] + (float)s : (float)s;
    }
}

// ------------------------------------------------------------------ host
static void rec_plan(const rat3d_recurrence_desc& d, RecArgs* q, int* waves) {
    const int64_t packed = (int64_t)d.c * d.len;
    const int tok = d.dtype == RAT3D_BF16 ? 8 : 4;
    q->sr = d.r_stride ? d.r_stride : packed;
    q->si = d.i_stride ? d.i_stride : packed;
    q->sx = d.x_stride ? d.x_stride : packed;
    q->sy = d.y_stride ? d.y_stride : packed;
    q->len = d.len;
    q->c = d.c;
    q->rows = (int64_t)d.n * d.c;
    q->rate = d.rate;
    q->blocks = (int)ceil_div(d.len, 64 * tok);
    q->segs = 1;
    q->lanes = 0;
    // Past the memory-side cache, whether rows begin on cache lines or not: 16 x 64 rows of
    // 129024 voxels 224 -> 218 us, gradient 385 -> 373; of 129023 254 -> 250 and 444 -> 442,
    // 8 x 64 in float32 212 -> 210 and 385 -> 388.
    q->stream = (double)packed * d.n * 16 / tok > 256e6;
    if (d.len <= 16 * tok) {
        q->lanes = 1;
        while (q->lanes * tok < d.len) q->lanes *= 2;
        return;
    }
    // Eight waves a row (four take the same time from 1024 rows on), sixteen where that is
    // the whole row, and where a CU has one row or little more of 64 blocks or more: of 64 to
    // 252 blocks, in bfloat16, 256 rows take 12 to 17 % less time than with eight, their
    // gradient 6 to 9 %; 320 and 383 rows 1 to 7 % less, their gradient 5 to 8 % more.  Of 17
    // to 63 blocks sixteen waves are slower from 320 rows on (by up to 21 %; 256 rows of 32 to
    // 63 blocks would be 3 to 9 % faster).
    // Rows of less than one a CU are cut: a forward over 128 rows of 129024 voxels takes 70 us
    // uncut, 59 with a launch that joins segments, 39 as segments that find one another.  From
    // a row a CU on cutting loses: 256 such rows take 63 us uncut, 69 as segments that find one
    // another (gradient 108 and 132) and 108 with joins; 512 of 16128 voxels 20 and 25 (36
    // and 44).
    const int64_t cus = device_cus();
    int most = 8;
    if (q->rows >= cus ? 2 * q->rows < 3 * cus && q->blocks >= 64 : q->blocks <= kWaves) {
        most = kWaves;
    } else if (q->rows < cus) {
        const int64_t turns = ceil_div(q->blocks, most), want = ceil_div(2 * cus, q->rows);
        q->one = turns <= kSegs;
        q->segs = (int)(q->one ? turns : want < kCuts ? want : kCuts);
    }
    *waves = q->blocks < most ? q->blocks : most;
}

size_t recurrence_carry_bytes(const rat3d_recurrence_desc& d) {
    RecArgs q = {};
    int waves;
    rec_plan(d, &q, &waves);
    return (size_t)q.rows * q.blocks * sizeof(float);
}

// Workspace: the rows' counters, the joined segments, the first states, and for the backward
// the parts of dlambda.
static size_t rec_workspace(RecArgs* q, void* ws, int pass) {
    const size_t pairs = q->segs > 1 ? (size_t)q->rows * q->segs : 0;
    const size_t at = q->one ? 4 * kLine * (size_t)q->rows : 0, first = at + 8 * pairs;
    const size_t part = first + (q->segs > 1 ? 4 * (size_t)q->rows : 0);
    if (ws) {
        q->drawn = (uint32_t*)ws;
        q->joined = (float2*)((char*)ws + at);
        q->first = (float*)((char*)ws + first);
        q->part = (float*)((char*)ws + part);
    }
    return part + (pass ? 4 * (size_t)q->rows * q->segs : 0);
}
size_t recurrence_ws_bytes(const rat3d_recurrence_desc& d, int pass) {
    RecArgs q = {};
    int waves;
    rec_plan(d, &q, &waves);
    return rec_workspace(&q, nullptr, pass);
}

static rat3d_status rec_begin(const RecArgs& q, hipStream_t st) {
    ProfScope ps("recurrence_begin", st, 0.0, 8.0 * q.rows * q.segs);
    recurrence_begin_k<<<(unsigned)ceil_div(q.rows * q.segs, 256), 256, 0, st>>>(q);
    RAT3D_LAUNCH_CHECK();
    return RAT3D_OK;
}

static double rec_bytes(const rat3d_recurrence_desc& d, int tensors) {
    return (double)d.n * d.c * d.len * tensors * (d.dtype == RAT3D_BF16 ? 2 : 4);
}

rat3d_status recurrence_fwd(const rat3d_recurrence_desc& d, const void* r, const void* i,
                            const void* x, const float* lam, const uint8_t* mask, const float* h0,
                            void* y, float* h_last, float* carry, void* ws, hipStream_t st) {
    RecArgs q = {};
    int waves = 0;
    rec_plan(d, &q, &waves);
    q.r = r;
    q.i = i;
    q.x = x;
    q.lam = lam;
    q.mask = mask;
    q.h0 = h0;
    q.y = y;
    q.h_last = h_last;
    q.carry = carry;
    rec_workspace(&q, ws, 0);
    if (q.lanes) {
        const unsigned grid = (unsigned)ceil_div(q.rows * q.lanes, 256);
        ProfScope ps("recurrence_short_fwd", st, 0.0, rec_bytes(d, 4));
#define RAT3D_REC(T, DOWN) recurrence_short_fwd_k<T, DOWN><<<grid, 256, 0, st>>>(q)
        if (d.dtype == RAT3D_BF16) {
            if (d.reverse) RAT3D_REC(bf16, true);
            else RAT3D_REC(bf16, false);
        } else {
            if (d.reverse) RAT3D_REC(float, true);
            else RAT3D_REC(float, false);
        }
#undef RAT3D_REC
        RAT3D_LAUNCH_CHECK();
        return RAT3D_OK;
    }
    const unsigned grid = (unsigned)(q.rows * q.segs), threads = 64 * waves;
#define RAT3D_REC(KERNEL, ...)                                                           \
    do {                                                                                 \
        if (d.dtype == RAT3D_BF16) {                                                     \
            if (d.reverse) KERNEL<bf16, true __VA_ARGS__><<<grid, threads, 0, st>>>(q);  \
            else KERNEL<bf16, false __VA_ARGS__><<<grid, threads, 0, st>>>(q);           \
        } else {                                                                         \
            if (d.reverse) KERNEL<float, true __VA_ARGS__><<<grid, threads, 0, st>>>(q); \
            else KERNEL<float, false __VA_ARGS__><<<grid, threads, 0, st>>>(q);          \
        }                                                                                \
        RAT3D_LAUNCH_CHECK();                                                            \
    } while (0)
#define RAT3D_COMMA ,
    if (q.one) {
        const rat3d_status s = rec_begin(q, st);
        if (s != RAT3D_OK) return s;
        ProfScope ps("recurrence_fwd_one", st, 0.0, rec_bytes(d, 4));
        RAT3D_REC(recurrence_fwd_one_k);
        return RAT3D_OK;
    }
    if (q.segs > 1) {
        ProfScope ps("recurrence_fwd_join", st, 0.0, rec_bytes(d, 3));
        RAT3D_REC(recurrence_fwd_k, RAT3D_COMMA true);
    }
    ProfScope ps(q.segs > 1 ? "recurrence_fwd_cut" : "recurrence_fwd", st, 0.0, rec_bytes(d, 4));
    RAT3D_REC(recurrence_fwd_k, RAT3D_COMMA false);
#undef RAT3D_COMMA
#undef RAT3D_REC
    return RAT3D_OK;
}

rat3d_status recurrence_bwd(const rat3d_recurrence_desc& d, const void* dy, const float* dh_last,
                            const void* r, const void* i, const void* x, const float* lam,
                            const uint8_t* mask, const float* carry, void* dr, void* di, void* dx,
                            float* dlam, float* dh0, int accumulate, void* ws, hipStream_t st) {
    RecArgs q = {};
    int waves = 0;
    rec_plan(d, &q, &waves);
    q.dy = dy;
    q.h0 = dh_last;
    q.r = r;
    q.i = i;
    q.x = x;
    q.lam = lam;
    q.mask = mask;
    q.carry = const_cast<float*>(carry);
    q.dr = dr;
    q.di = di;
    q.dx = dx;
    q.h_last = dh0;
    rec_workspace(&q, ws, 1);
    // the gradient walks against the forward
#define RAT3D_REC(KERNEL, GRID, THREADS)                                           \
    do {                                                                           \
        if (d.dtype == RAT3D_BF16) {                                               \
            if (d.reverse) KERNEL<bf16, false><<<GRID, THREADS, 0, st>>>(q);       \
            else KERNEL<bf16, true><<<GRID, THREADS, 0, st>>>(q);                  \
        } else {                                                                   \
            if (d.reverse) KERNEL<float, false><<<GRID, THREADS, 0, st>>>(q);      \
            else KERNEL<float, true><<<GRID, THREADS, 0, st>>>(q);                 \
        }                                                                          \
        RAT3D_LAUNCH_CHECK();                                                      \
    } while (0)
    if (q.lanes) {
        const unsigned grid = (unsigned)ceil_div(q.rows * q.lanes, 256);
        ProfScope ps("recurrence_short_bwd", st, 0.0, rec_bytes(d, 7));
        RAT3D_REC(recurrence_short_bwd_k, grid, 256);
    } else {
        const unsigned grid = (unsigned)(q.rows * q.segs), threads = 64 * waves;
        if (q.one) {
            const rat3d_status s = rec_begin(q, st);
            if (s != RAT3D_OK) return s;
            ProfScope ps("recurrence_bwd_one", st, 0.0, rec_bytes(d, 7));
            RAT3D_REC(recurrence_bwd_one_k, grid, threads);
        } else {
            if (q.segs > 1) {
                ProfScope ps("recurrence_bwd_join", st, 0.0, rec_bytes(d, 2));
                RAT3D_REC(recurrence_bwd_join_k, grid, threads);
            }
            ProfScope ps(q.segs > 1 ? "recurrence_bwd_cut" : "recurrence_bwd", st, 0.0,
                         rec_bytes(d, 7));
            RAT3D_REC(recurrence_bwd_k, grid, threads);
        }
    }
#undef RAT3D_REC
    const int parts = d.n * q.segs;
    ProfScope ps("recurrence_lambda", st, 0.0, 4.0 * parts * d.c);
    recurrence_lambda_k<<<d.c, 256, 0, st>>>(q.part, parts, lam, dlam, accumulate);
    RAT3D_LAUNCH_CHECK();
    return RAT3D_OK;
}

}  // namespace rat3d
