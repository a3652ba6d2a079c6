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
// (a, b) behind (a', b') is (a a', a b' + b).  h_{t-1} is formed again from the states
// that the forward left every kBlock voxels, in float32.
//
// beta: 1 - a^2 is -expm1(-2 w sigmoid(r)), by its series where the argument is small.
// Bound: HBM.
#include "kernels.hpp"
#include "prof.hpp"
#include "vec.hpp"

namespace rat3d {

constexpr int kTok = 8;              // voxels a lane
constexpr int kBlock = 64 * kTok;    // voxels between two saved states

struct RecArgs {
    const void *r, *i, *x, *dy;
    const float* lam;
    const uint8_t* mask;
    const float* h0;
    const float* dh;
    void *y, *dr, *di, *dx;
    float *h_last, *carry, *dh0, *part;
    int64_t sr, si, sx, sy, len;
    int c, blocks, reverse;
    float rate;
};

__device__ __forceinline__ float softplusf(float v) {
    return v > 0.f ? v + log1pf(expf(-v)) : log1pf(expf(v));
}

// One voxel's step.
struct Step {
    float rest, la, a, p, inv;  // rest = 1 - sigmoid(r), p = 1 - a^2, inv = 1 / sqrt(p)
    __device__ __forceinline__ Step(float r, float w) {
        const Sig g(r);
        rest = g.rest;
        la = -w * g.s;
        a = expf(la);
        p = -expm1f(2.f * la);
        // at p = 0 (a shut gate) la inv and p inv come out as 0, their limits
        inv = __builtin_amdgcn_rsqf(p < 0x1p-100f ? 0x1p-100f : p);
    }
};

// (a, b) of this lane and of all lanes before it, joined; lanes behind in the walk's
// order have higher ids.
__device__ __forceinline__ void scan_wave(float& a, float& b) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) {
        const float pa = __shfl_up(a, m), pb = __shfl_up(b, m);
        if (lane >= m) {
            b = __builtin_fmaf(a, pb, b);
            a *= pa;
        }
    }
}

// One wave a row.  The walk's step k takes the voxels k * kBlock and up in its order;
// voxel v of the order lies at v, or from the end if REV.
template <typename T, bool REV>
__global__ __launch_bounds__(64) void recurrence_fwd_k(RecArgs q) {
    const int lane = threadIdx.x;
    const int64_t row = blockIdx.x;
    const int64_t vol = row / q.c;
    const int ch = (int)(row - vol * q.c);
    const float w = q.rate * softplusf(q.lam[ch]);
    const T* r = (const T*)q.r + vol * q.sr + (int64_t)ch * q.len;
    const T* g = (const T*)q.i + vol * q.si + (int64_t)ch * q.len;
    const T* x = (const T*)q.x + vol * q.sx + (int64_t)ch * q.len;
    T* y = (T*)q.y + vol * q.sy + (int64_t)ch * q.len;
    const uint8_t* mask = q.mask ? q.mask + vol * q.len : nullptr;
    float state = q.h0 ? q.h0[row] : 0.f;
    for (int k = 0; k < q.blocks; ++k) {
        if (q.carry && lane == 0) q.carry[row * q.blocks + k] = state;
        float a[kTok], b[kTok];
        float A = 1.f, B = 0.f;
        const int64_t v0 = (int64_t)k * kBlock + lane * kTok;
        uint32_t on = 0;
#pragma unroll
        for (int j = 0; j < kTok; ++j) {
            const int64_t v = v0 + j, at = REV ? q.len - 1 - v : v;
            a[j] = 1.f;
            b[j] = 0.f;
            if (v < q.len && (!mask || mask[at])) {
                on |= 1u << j;
                const Step s(Elt<T>::ld(r + at), w);
                a[j] = s.a;
                b[j] = s.p * s.inv * Sig(Elt<T>::ld(g + at)).s * Elt<T>::ld(x + at);
            }
            B = __builtin_fmaf(a[j], B, b[j]);
            A *= a[j];
        }
        scan_wave(A, B);
        float pa = __shfl_up(A, 1), pb = __shfl_up(B, 1);
        if (lane == 0) {
            pa = 1.f;
            pb = 0.f;
        }
        float h = __builtin_fmaf(pa, state, pb);
#pragma unroll
        for (int j = 0; j < kTok; ++j) {
            const int64_t v = v0 + j, at = REV ? q.len - 1 - v : v;
            h = __builtin_fmaf(a[j], h, b[j]);
            if (v < q.len) Elt<T>::st(y + at, on >> j & 1u ? h : 0.f);
        }
        state = __shfl(h, 63);
    }
    if (q.h_last && lane == 0) q.h_last[row] = state;
}

template <typename T, bool REV>
__global__ __launch_bounds__(64) void recurrence_bwd_k(RecArgs q) {
    const int lane = threadIdx.x;
    const int64_t row = blockIdx.x;
    const int64_t vol = row / q.c;
    const int ch = (int)(row - vol * q.c);
    const float w = q.rate * softplusf(q.lam[ch]);
    const T* r = (const T*)q.r + vol * q.sr + (int64_t)ch * q.len;
    const T* g = (const T*)q.i + vol * q.si + (int64_t)ch * q.len;
    const T* x = (const T*)q.x + vol * q.sx + (int64_t)ch * q.len;
    const T* dy = (const T*)q.dy + vol * q.sy + (int64_t)ch * q.len;
    T* dr = (T*)q.dr + vol * q.sr + (int64_t)ch * q.len;
    T* di = (T*)q.di + vol * q.si + (int64_t)ch * q.len;
    T* dx = (T*)q.dx + vol * q.sx + (int64_t)ch * q.len;
    const uint8_t* mask = q.mask ? q.mask + vol * q.len : nullptr;
    float end = q.dh ? q.dh[row] : 0.f;  // E behind the block
    double sum = 0.0;
    for (int k = q.blocks - 1; k >= 0; --k) {
        float a[kTok], b[kTok], la[kTok], rr[kTok], inv[kTok], p[kTok], si[kTok], ri[kTok], xv[kTok],
            d[kTok];
        const int64_t v0 = (int64_t)k * kBlock + lane * kTok;
        uint32_t on = 0;
        float A = 1.f, B = 0.f;
#pragma unroll
        for (int j = 0; j < kTok; ++j) {
            const int64_t v = v0 + j, at = REV ? q.len - 1 - v : v;
            a[j] = 1.f;
            b[j] = la[j] = rr[j] = inv[j] = p[j] = si[j] = ri[j] = xv[j] = d[j] = 0.f;
            if (v < q.len && (!mask || mask[at])) {
                on |= 1u << j;
                const Step s(Elt<T>::ld(r + at), w);
                a[j] = s.a;
                la[j] = s.la;
                rr[j] = s.rest;
                p[j] = s.p;
                inv[j] = s.inv;
                const Sig gi(Elt<T>::ld(g + at));
                si[j] = gi.s;
                ri[j] = gi.rest;
                xv[j] = Elt<T>::ld(x + at);
                d[j] = Elt<T>::ld(dy + at);
                b[j] = p[j] * inv[j] * si[j] * xv[j];
            }
            B = __builtin_fmaf(a[j], B, b[j]);
            A *= a[j];
        }
        scan_wave(A, B);
        float pa = __shfl_up(A, 1), pb = __shfl_up(B, 1);
        if (lane == 0) {
            pa = 1.f;
            pb = 0.f;
        }
        float h = __builtin_fmaf(pa, q.carry[row * q.blocks + k], pb);
        float past[kTok];
#pragma unroll
        for (int j = 0; j < kTok; ++j) {
            past[j] = h;
            h = __builtin_fmaf(a[j], h, b[j]);
        }
        // the walk back: the last lane comes first
        A = 1.f;
        B = 0.f;
#pragma unroll
        for (int j = kTok - 1; j >= 0; --j) {
            B = a[j] * (d[j] + B);
            A *= a[j];
        }
        A = __shfl(A, 63 - lane);
        B = __shfl(B, 63 - lane);
        scan_wave(A, B);
        const float total = __builtin_fmaf(__shfl(A, 63), end, __shfl(B, 63));
        pa = __shfl_up(A, 1);
        pb = __shfl_up(B, 1);
        if (lane == 0) {
            pa = 1.f;
            pb = 0.f;
        }
        pa = __shfl(pa, 63 - lane);
        pb = __shfl(pb, 63 - lane);
        float E = __builtin_fmaf(pa, end, pb);
        float part = 0.f;
#pragma unroll
        for (int j = kTok - 1; j >= 0; --j) {
            const int64_t v = v0 + j, at = REV ? q.len - 1 - v : v;
            const float D = d[j] + E;
            E = a[j] * D;
            const float u = si[j] * xv[j];
            const float K = D * (la[j] * a[j] * past[j] - u * (a[j] * a[j]) * (la[j] * inv[j]));
            const float gx = D * (p[j] * inv[j]) * si[j];
            const bool live = on >> j & 1u;
            part += live ? K : 0.f;
            if (v < q.len) {
                Elt<T>::st(dr + at, live ? K * rr[j] : 0.f);
                Elt<T>::st(di + at, live ? gx * xv[j] * ri[j] : 0.f);
                Elt<T>::st(dx + at, live ? gx : 0.f);
            }
        }
        sum += (double)part;
        end = total;
    }
#pragma unroll
    for (int m = 32; m >= 1; m >>= 1) sum += __shfl_xor(sum, m);
    if (lane == 0) {
        q.part[(int64_t)ch * (gridDim.x / q.c) + vol] = (float)sum;
        if (q.dh0) q.dh0[row] = end;
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
static void rec_plan(const rat3d_recurrence_desc& d, RecArgs* q) {
    const int64_t packed = (int64_t)d.c * d.len;
    q->sr = d.r_stride ? d.r_stride : packed;
    q->si = d.i_stride ? d.i_stride : packed;
    q->sx = d.x_stride ? d.x_stride : packed;
    q->sy = d.y_stride ? d.y_stride : packed;
    q->len = d.len;
    q->c = d.c;
    q->blocks = (int)ceil_div(d.len, kBlock);
    q->rate = d.rate;
}

size_t recurrence_carry_bytes(const rat3d_recurrence_desc& d) {
    return (size_t)d.n * d.c * ceil_div(d.len, kBlock) * sizeof(float);
}

size_t recurrence_ws_bytes(const rat3d_recurrence_desc& d, int pass) {
    return pass ? (size_t)d.n * d.c * sizeof(float) : 0;
}

static double rec_bytes(const rat3d_recurrence_desc& d, int tensors) {
    return (double)d.n * d.c * d.len * tensors * (d.dtype == RAT3D_BF16 ? 2 : 4);
}

rat3d_status recurrence_fwd(const rat3d_recurrence_desc& d, const void* r, const void* i,
                            const void* x, const float* lam, const uint8_t* mask, const float* h0,
                            void* y, float* h_last, float* carry, void* ws, hipStream_t st) {
    RecArgs q = {};
    rec_plan(d, &q);
    q.r = r;
    q.i = i;
    q.x = x;
    q.lam = lam;
    q.mask = mask;
    q.h0 = h0;
    q.y = y;
    q.h_last = h_last;
    q.carry = carry;
    const unsigned grid = (unsigned)(d.n * d.c);
    ProfScope ps("recurrence_fwd", st, 0.0, rec_bytes(d, 4));
    if (d.dtype == RAT3D_BF16) {
        if (d.reverse) recurrence_fwd_k<bf16, true><<<grid, 64, 0, st>>>(q);
        else recurrence_fwd_k<bf16, false><<<grid, 64, 0, st>>>(q);
    } else {
        if (d.reverse) recurrence_fwd_k<float, true><<<grid, 64, 0, st>>>(q);
        else recurrence_fwd_k<float, false><<<grid, 64, 0, st>>>(q);
    }
    RAT3D_LAUNCH_CHECK();
    return RAT3D_OK;
}

rat3d_status recurrence_bwd(const rat3d_recurrence_desc& d, const void* dy, const float* dh_last,
                            const void* r, const void* i, const void* x, const float* lam,
                            const uint8_t* mask, const float* carry, void* dr, void* di, void* dx,
                            float* dlam, float* dh0, int accumulate, void* ws, hipStream_t st) {
    RecArgs q = {};
    rec_plan(d, &q);
    q.dy = dy;
    q.dh = dh_last;
    q.r = r;
    q.i = i;
    q.x = x;
    q.lam = lam;
    q.mask = mask;
    q.carry = const_cast<float*>(carry);
    q.dr = dr;
    q.di = di;
    q.dx = dx;
    q.dh0 = dh0;
    q.part = (float*)ws;
    const unsigned grid = (unsigned)(d.n * d.c);
    {
        ProfScope ps("recurrence_bwd", st, 0.0, rec_bytes(d, 7));
        if (d.dtype == RAT3D_BF16) {
            if (d.reverse) recurrence_bwd_k<bf16, true><<<grid, 64, 0, st>>>(q);
            else recurrence_bwd_k<bf16, false><<<grid, 64, 0, st>>>(q);
        } else {
            if (d.reverse) recurrence_bwd_k<float, true><<<grid, 64, 0, st>>>(q);
            else recurrence_bwd_k<float, false><<<grid, 64, 0, st>>>(q);
        }
        RAT3D_LAUNCH_CHECK();
    }
    ProfScope ps("recurrence_lambda", st, 0.0, 4.0 * d.n * d.c);
    recurrence_lambda_k<<<d.c, 256, 0, st>>>(q.part, d.n, lam, dlam, accumulate);
    RAT3D_LAUNCH_CHECK();
    return RAT3D_OK;
}

}  // namespace rat3d
