// Norms of a voxel's channels before and behind a block, on channel-first maps.
//
// Before:  u = gamma x r,  r = 1/sqrt(mean x^2 + eps), the mean over a voxel's channels.
//   dx = [dres +] r (gamma du - x r^2 mean(gamma du x)),  dgamma = sum du x r
// Behind:  y = x + s phi(g) gamma z r_z,  phi = 1, sigmoid or silu, and, for the block
// that follows, u = gamma' y r_y (y before its rounding).
//   dY = dy + r_y (gamma' du - y r_y^2 mean(gamma' du y)) = dx,  dgamma' = sum du y r_y
//   t = sum dY phi z r_z over voxels:  dgamma = s t,  ds = gamma t
//   e = dY s gamma phi:  dz = r_z (e - z r_z^2 mean(e z)),  dg = dY s gamma z r_z phi'(g)
// Every r is formed again from the tensor it belongs to, which the backward reads
// anyway: nothing is saved.  A masked voxel has u = 0, y = x, dx = dy, dz = dg = 0 and
// no part in a gain; what its other inputs hold is not read into a result.
//
// Layout: 16 lanes along the voxels, 16 bytes each, by groups of threads along the
// channels, so a channel's row is read in pieces of 256 bytes; a group takes the
// channels grp, grp + groups, ... Sums over a voxel's channels are joined by lane swaps
// and through LDS.
// Bound: HBM.
#include <type_traits>

#include "kernels.hpp"
#include "prof.hpp"
#include "vec.hpp"

namespace rat3d {

constexpr int kLanes = 16;  // along the voxels

enum NormMode { PRE_FWD, PRE_BWD, POST_FWD, POST_BWD };

struct NormArgs {
    // forward: x, z, g -> y, u.  Backward: dy, du, y (before: x, dres for y, dy), z, g -> dx, dz, dg
    const void *x, *z, *g, *y, *dy, *du;
    void *oy, *ou, *dx, *dz, *dg;
    const float *gamma, *scale, *next;
    const uint8_t* mask;
    float* part;  // [workgroup][gain][channel]
    int64_t sx, sz, sg, sy, su;  // from one volume to the next
    int64_t V;
    int c, groups, tiles, gate;  // tiles of one volume
    int64_t all;                 // tiles of all volumes
    float eps;
};

// Sum over a voxel's channels of K values of each token: the four groups of a wave by
// lane swaps that leave every group a quarter of the tokens, the waves through LDS.
template <int TOK, int K>
__device__ __forceinline__ void channel_sums(float (&s)[K][TOK], float* lds, int waves) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, at = lane & 15;
#pragma unroll
    for (int k = 0; k < K; ++k) {
#pragma unroll
        for (int j = 0; j < TOK; ++j) {
            s[k][j] += __shfl_xor(s[k][j], 16);
            s[k][j] += __shfl_xor(s[k][j], 32);
        }
        if (lane < kLanes) {
#pragma unroll
            for (int j = 0; j < TOK; ++j) lds[((wave * K + k) * kLanes + at) * TOK + j] = s[k][j];
        }
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
        for (int j = 0; j < TOK; ++j) s[k][j] = 0.f;
    for (int w = 0; w < waves; ++w)
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int j = 0; j < TOK; ++j) s[k][j] += lds[((w * K + k) * kLanes + at) * TOK + j];
}

__device__ __forceinline__ float rsqrt_of(float sum, float inv_c, float eps) {
    return __builtin_amdgcn_rsqf(__builtin_fmaf(sum, inv_c, eps));
}

template <typename T, int TOK, NormMode MODE, bool GATED, bool NEXT>
__global__ __launch_bounds__(256) void block_norm_k(NormArgs a) {
    constexpr bool kBwd = MODE == PRE_BWD || MODE == POST_BWD;
    constexpr bool kPost = MODE == POST_FWD || MODE == POST_BWD;
    constexpr int TILE = kLanes * TOK;
    __shared__ float lds[2][4 * 3 * kLanes * TOK];
    const int at = threadIdx.x & 15, grp = threadIdx.x >> 4;
    const int waves = (a.groups * kLanes + 63) >> 6;
    const float inv_c = 1.f / (float)a.c;

    for (int64_t t = blockIdx.x; t < a.all; t += gridDim.x) {
        const int64_t vol = t / a.tiles;
        const int64_t t0 = (t - vol * a.tiles) * TILE + at * TOK;
        const int left = (int)(a.V - t0 < TOK ? (a.V - t0 > 0 ? a.V - t0 : 0) : TOK);
        uint32_t on = (1u << left) - 1u;
        if (a.mask)
#pragma unroll
            for (int j = 0; j < TOK; ++j)
                if (j < left && !a.mask[vol * a.V + t0 + j]) on &= ~(1u << j);
        auto rd = [&](const void* p, int64_t stride, int ch, float (&o)[TOK], bool live) {
            const T* q = (const T*)p + vol * stride + (int64_t)ch * a.V + t0;
#pragma unroll
            for (int j = 0; j < TOK; ++j)
                o[j] = (live ? on >> j & 1u : j < left) ? Elt<T>::ld(q + j) : 0.f;
        };
        auto wr = [&](void* p, int64_t stride, int ch, const float (&o)[TOK]) {
            T* q = (T*)p + vol * stride + (int64_t)ch * a.V + t0;
#pragma unroll
            for (int j = 0; j < TOK; ++j)
                if (j < left) Elt<T>::st(q + j, o[j]);
        };
        // the gate's value and slope
        auto gate = [&](float g, float& phi, float& slope) {
            const Sig sg(g);
            phi = a.gate == RAT3D_GATE_SILU ? g * sg.s : sg.s;
            slope = a.gate == RAT3D_GATE_SILU ? sg.s * (1.f + g * sg.rest) : sg.s * sg.rest;
        };
        auto gain = [&](int ch) { return a.gamma[ch] * (a.scale ? a.scale[ch] : 1.f); };
        float s[3][TOK], e[1][TOK];
#pragma unroll
        for (int j = 0; j < TOK; ++j) s[0][j] = s[1][j] = s[2][j] = e[0][j] = 0.f;

        if constexpr (MODE == PRE_FWD) {
            for (int ch = grp; ch < a.c; ch += a.groups) {
                float x[TOK];
                rd(a.x, a.sx, ch, x, true);
#pragma unroll
                for (int j = 0; j < TOK; ++j) e[0][j] += x[j] * x[j];
            }
            channel_sums(e, lds[0], waves);
            for (int ch = grp; ch < a.c; ch += a.groups) {
                float x[TOK];
                rd(a.x, a.sx, ch, x, true);
#pragma unroll
                for (int j = 0; j < TOK; ++j) x[j] *= rsqrt_of(e[0][j], inv_c, a.eps) * a.gamma[ch];
                wr(a.ou, a.su, ch, x);
            }
        }
        if constexpr (MODE == POST_FWD) {
            for (int ch = grp; ch < a.c; ch += a.groups) {
                float z[TOK];
                rd(a.z, a.sz, ch, z, true);
#pragma unroll
                for (int j = 0; j < TOK; ++j) e[0][j] += z[j] * z[j];
            }
            channel_sums(e, lds[0], waves);
            float rz[TOK];
#pragma unroll
            for (int j = 0; j < TOK; ++j) rz[j] = rsqrt_of(e[0][j], inv_c, a.eps);
            auto value = [&](int ch, float (&y)[TOK]) {
                float z[TOK], g[TOK];
                rd(a.z, a.sz, ch, z, true);
                if (GATED) rd(a.g, a.sg, ch, g, true);
                rd(a.x, a.sx, ch, y, false);
                const float k = gain(ch);
#pragma unroll
                for (int j = 0; j < TOK; ++j) {
                    float phi = 1.f, slope;
                    if (GATED) gate(g[j], phi, slope);
                    if (on >> j & 1u) y[j] += k * phi * (z[j] * rz[j]);
                }
            };
            if (NEXT) {
#pragma unroll
                for (int j = 0; j < TOK; ++j) e[0][j] = 0.f;
                for (int ch = grp; ch < a.c; ch += a.groups) {
                    float y[TOK];
                    value(ch, y);
#pragma unroll
                    for (int j = 0; j < TOK; ++j) e[0][j] += on >> j & 1u ? y[j] * y[j] : 0.f;
                }
                channel_sums(e, lds[1], waves);
            }
            for (int ch = grp; ch < a.c; ch += a.groups) {
                float y[TOK];
                value(ch, y);
                wr(a.oy, a.sy, ch, y);
                if (NEXT) {
#pragma unroll
                    for (int j = 0; j < TOK; ++j)
                        y[j] = on >> j & 1u ? y[j] * rsqrt_of(e[0][j], inv_c, a.eps) * a.next[ch] : 0.f;
                    wr(a.ou, a.su, ch, y);
                }
            }
        }
        if constexpr (kBwd) {
            constexpr bool kNext = MODE == PRE_BWD || NEXT;
            const float* gn = MODE == PRE_BWD ? a.gamma : a.next;
            for (int ch = grp; ch < a.c; ch += a.groups) {
                float y[TOK], du[TOK], z[TOK];
                if (kNext) {
                    rd(a.y, a.sy, ch, y, true);
                    rd(a.du, a.su, ch, du, true);
                }
                if (kPost) rd(a.z, a.sz, ch, z, true);
#pragma unroll
                for (int j = 0; j < TOK; ++j) {
                    if (kNext) {
                        s[0][j] += y[j] * y[j];
                        s[1][j] += gn[ch] * du[j] * y[j];
                    }
                    if (kPost) s[2][j] += z[j] * z[j];
                }
            }
            channel_sums(s, lds[0], waves);
            float ry[TOK], my[TOK], rz[TOK], mz[TOK];
#pragma unroll
            for (int j = 0; j < TOK; ++j) {
                ry[j] = rsqrt_of(s[0][j], inv_c, a.eps);
                my[j] = s[1][j] * inv_c * (ry[j] * ry[j]);
                rz[j] = rsqrt_of(s[2][j], inv_c, a.eps);
            }
            // dY, and what it leaves to the branch (0 where masked)
            auto residual = [&](int ch, float (&dY)[TOK], float (&du)[TOK], float (&y)[TOK]) {
                if (a.dy) rd(a.dy, MODE == PRE_BWD ? a.sx : a.sy, ch, dY, false);
                else
#pragma unroll
                    for (int j = 0; j < TOK; ++j) dY[j] = 0.f;
                if (kNext) {
                    rd(a.y, a.sy, ch, y, true);
                    rd(a.du, a.su, ch, du, true);
#pragma unroll
                    for (int j = 0; j < TOK; ++j)
                        if (on >> j & 1u) dY[j] += ry[j] * (gn[ch] * du[j] - y[j] * my[j]);
                }
            };
            if (kPost) {
                for (int ch = grp; ch < a.c; ch += a.groups) {
                    float dY[TOK], du[TOK], y[TOK], z[TOK], g[TOK];
                    residual(ch, dY, du, y);
                    rd(a.z, a.sz, ch, z, true);
                    if (GATED) rd(a.g, a.sg, ch, g, true);
                    const float k = gain(ch);
#pragma unroll
                    for (int j = 0; j < TOK; ++j) {
                        float phi = 1.f, slope;
                        if (GATED) gate(g[j], phi, slope);
                        if (on >> j & 1u) e[0][j] += dY[j] * k * phi * z[j];
                    }
                }
                channel_sums(e, lds[1], waves);
#pragma unroll
                for (int j = 0; j < TOK; ++j) mz[j] = e[0][j] * inv_c * (rz[j] * rz[j]);
            }
            for (int ch = grp; ch < a.c; ch += a.groups) {
                float dY[TOK], du[TOK], y[TOK];
                residual(ch, dY, du, y);
                float sum_n = 0.f, sum_t = 0.f;
                if (kNext) {
#pragma unroll
                    for (int j = 0; j < TOK; ++j) sum_n += du[j] * y[j] * ry[j];
                }
                if (kPost) {
                    float z[TOK], g[TOK], dz[TOK], dg[TOK];
                    rd(a.z, a.sz, ch, z, true);
                    if (GATED) rd(a.g, a.sg, ch, g, true);
                    const float k = gain(ch);
#pragma unroll
                    for (int j = 0; j < TOK; ++j) {
                        float phi = 1.f, slope = 0.f;
                        if (GATED) gate(g[j], phi, slope);
                        const float d = on >> j & 1u ? dY[j] : 0.f, zr = z[j] * rz[j];
                        sum_t += d * phi * zr;
                        dz[j] = rz[j] * (d * k * phi - z[j] * mz[j]);
                        dg[j] = d * k * zr * slope;
                    }
                    wr(a.dz, a.sz, ch, dz);
                    if (GATED) wr(a.dg, a.sg, ch, dg);
                }
                if (a.dx) wr(a.dx, a.sx, ch, dY);
                // gains: over the lanes, then this workgroup's tiles
#pragma unroll
                for (int m = 8; m >= 1; m >>= 1) {
                    sum_n += __shfl_xor(sum_n, m);
                    sum_t += __shfl_xor(sum_t, m);
                }
                if (at == 0) {
                    float* to = a.part + (int64_t)blockIdx.x * 2 * a.c;
                    const bool more = t != blockIdx.x;
                    if (kNext) to[ch] = more ? to[ch] + sum_n : sum_n;
                    if (kPost) to[a.c + ch] = more ? to[a.c + ch] + sum_t : sum_t;
                }
            }
        }
        __syncthreads();  // LDS is written again
    }
}

// The gains' gradients: the parts of the workgroups added in float64, in a fixed order.
__global__ __launch_bounds__(256) void norm_gain_k(const float* __restrict__ part, int parts, int c,
                                                   const float* gamma, const float* scale,
                                                   float* dnext, float* dgamma, float* dscale,
                                                   int accumulate) {
    __shared__ double red[4];
    const int ch = blockIdx.x, which = blockIdx.y;  // 0: the norm read by du, 1: the branch's
    double s = 0.0;
    for (int i = threadIdx.x; i < parts; i += 256)
        s += (double)part[((int64_t)i * 2 + which) * c + ch];
#pragma unroll
    for (int m = 32; m >= 1; m >>= 1) s += __shfl_xor(s, m);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
    __syncthreads();
    if (threadIdx.x == 0) {
        s = (red[0] + red[1]) + (red[2] + red[3]);
        auto put = [&](float* to, double v) {
            if (to) to[ch] = accumulate ? to[ch] + (float)v : (float)v;
        };
        if (which == 0) {
            put(dnext, s);
        } else {
            put(dgamma, scale ? s * (double)scale[ch] : s);
            put(dscale, s * (double)gamma[ch]);
        }
    }
}

// ------------------------------------------------------------------ host
static void norm_plan(const rat3d_norm_desc& d, NormArgs* a) {
    const int64_t packed = (int64_t)d.c * d.v;
    a->sx = d.x_stride ? d.x_stride : packed;
    a->sz = d.z_stride ? d.z_stride : packed;
    a->sg = d.g_stride ? d.g_stride : packed;
    a->sy = d.y_stride ? d.y_stride : packed;
    a->su = d.u_stride ? d.u_stride : packed;
    a->V = d.v;
    a->c = d.c;
    a->eps = d.eps;
    a->gate = d.gate;
    a->groups = 16;
    const int tile = kLanes * 16 / (d.dtype == RAT3D_BF16 ? 2 : 4);
    a->tiles = (int)ceil_div(d.v, tile);
    a->all = (int64_t)a->tiles * d.n;
}

static int norm_grid(const NormArgs& a) {
    const int64_t most = 8 * (int64_t)device_cus();
    return (int)(a.all < most ? a.all : most);
}

size_t norm_ws_bytes(const rat3d_norm_desc& d) {
    NormArgs a = {};
    norm_plan(d, &a);
    return (size_t)norm_grid(a) * 2 * d.c * sizeof(float);
}

template <NormMode MODE, bool GATED, bool NEXT>
static void norm_launch(const rat3d_norm_desc& d, const NormArgs& a, hipStream_t st) {
    const int grid = norm_grid(a);
    if (d.dtype == RAT3D_BF16) block_norm_k<bf16, 8, MODE, GATED, NEXT><<<grid, 256, 0, st>>>(a);
    else block_norm_k<float, 4, MODE, GATED, NEXT><<<grid, 256, 0, st>>>(a);
}

static double norm_bytes(const rat3d_norm_desc& d, int tensors) {
    return (double)d.n * d.c * d.v * tensors * (d.dtype == RAT3D_BF16 ? 2 : 4);
}

rat3d_status pre_norm_fwd(const rat3d_norm_desc& d, const void* x, const float* gamma,
                          const uint8_t* mask, void* u, hipStream_t st) {
    NormArgs a = {};
    norm_plan(d, &a);
    a.x = x;
    a.gamma = gamma;
    a.mask = mask;
    a.ou = u;
    ProfScope ps("pre_norm_fwd", st, 0.0, norm_bytes(d, 2));
    norm_launch<PRE_FWD, false, false>(d, a, st);
    RAT3D_LAUNCH_CHECK();
    return RAT3D_OK;
}

rat3d_status post_norm_fwd(const rat3d_norm_desc& d, const void* x, const void* z, const void* g,
                           const float* gamma, const float* scale, const float* next,
                           const uint8_t* mask, void* y, void* u, hipStream_t st) {
    NormArgs a = {};
    norm_plan(d, &a);
    a.x = x;
    a.z = z;
    a.g = g;
    a.gamma = gamma;
    a.scale = scale;
    a.next = next;
    a.mask = mask;
    a.oy = y;
    a.ou = u;
    ProfScope ps("post_norm_fwd", st, 0.0, norm_bytes(d, 3 + (d.gate != 0) + (next != nullptr)));
    if (d.gate && next) norm_launch<POST_FWD, true, true>(d, a, st);
    else if (d.gate) norm_launch<POST_FWD, true, false>(d, a, st);
    else if (next) norm_launch<POST_FWD, false, true>(d, a, st);
    else norm_launch<POST_FWD, false, false>(d, a, st);
    RAT3D_LAUNCH_CHECK();
    return RAT3D_OK;
}

static rat3d_status norm_gains(const NormArgs& a, float* dnext, float* dgamma, float* dscale,
                               int accumulate, hipStream_t st) {
    const int parts = norm_grid(a);
    ProfScope ps("norm_gain", st, 0.0, 8.0 * a.c * parts);
    norm_gain_k<<<dim3(a.c, 2), 256, 0, st>>>(a.part, parts, a.c, a.gamma, a.scale, dnext, dgamma,
                                              dscale, accumulate);
    RAT3D_LAUNCH_CHECK();
    return RAT3D_OK;
}

rat3d_status pre_norm_bwd(const rat3d_norm_desc& d, const void* du, const void* x,
                          const float* gamma, const uint8_t* mask, const void* dres, void* dx,
                          float* dgamma, int accumulate, void* ws, hipStream_t st) {
    NormArgs a = {};
    norm_plan(d, &a);
    a.du = du;
    a.y = x;
    a.sy = a.sx;
    a.dy = dres;
    a.gamma = gamma;
    a.mask = mask;
    a.dx = dx;
    a.part = (float*)ws;
    {
        ProfScope ps("pre_norm_bwd", st, 0.0, norm_bytes(d, 3 + (dres != nullptr)));
        norm_launch<PRE_BWD, false, true>(d, a, st);
        RAT3D_LAUNCH_CHECK();
    }
    return norm_gains(a, dgamma, nullptr, nullptr, accumulate, st);
}

rat3d_status post_norm_bwd(const rat3d_norm_desc& d, const void* dy, const void* du, const void* y,
                           const void* z, const void* g, const float* gamma, const float* scale,
                           const float* next, const uint8_t* mask, void* dx, void* dz, void* dg,
                           float* dgamma, float* dscale, float* dnext, int accumulate, void* ws,
                           hipStream_t st) {
    NormArgs a = {};
    norm_plan(d, &a);
    a.dy = dy;
    a.du = du;
    a.y = y;
    a.z = z;
    a.g = g;
    a.gamma = gamma;
    a.scale = scale;
    a.next = next;
    a.mask = mask;
    a.dx = dx;
    a.dz = dz;
    a.dg = dg;
    a.part = (float*)ws;
    {
        ProfScope ps("post_norm_bwd", st, 0.0,
                     norm_bytes(d, 3 + 2 * (d.gate != 0) + (next ? 3 : dx ? 1 : 0)));
        if (d.gate && next) norm_launch<POST_BWD, true, true>(d, a, st);
        else if (d.gate) norm_launch<POST_BWD, true, false>(d, a, st);
        else if (next) norm_launch<POST_BWD, false, true>(d, a, st);
        else norm_launch<POST_BWD, false, false>(d, a, st);
        RAT3D_LAUNCH_CHECK();
    }
    return norm_gains(a, dnext, dgamma, dscale, accumulate, st);
}

}  // namespace rat3d
