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
// channels grp, grp + groups, ... Up to 512 channels a thread keeps what it has read of
// its channels (4, or 8 of half as many voxels) in registers, so every tensor passes
// once; beyond, each sum reads its tensors again.  Sums over a voxel's channels are
// joined by lane swaps that leave each of a wave's four groups a quarter of the voxels,
// and through LDS.  Rows need no alignment.
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
    float* part;  // [gain][channel][workgroup]
    int64_t sx, sz, sg, sy, su;  // from one volume to the next
    int64_t V;
    int c, groups, tiles, gate;  // tiles of one volume
    int64_t all;                 // tiles of all volumes
    float eps;
};

// Half of a wave's rows of 16 lanes get x of their and the neighbouring row (or half of
// the wave) added, the others y.
__device__ __forceinline__ float join32(float x, float y) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(y), false,
                                                    false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ float join16(float x, float y) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(y), false,
                                                    false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// Sums over a voxel's channels of K values of each token, to all of the voxel's threads:
// in a wave, then through LDS [value][wave][lane][token].
template <int TOK, int K>
__device__ __forceinline__ void channel_sums(float (&s)[K][TOK], float* lds, int waves) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, at = lane & 15, row = lane >> 4;
#pragma unroll
    for (int k = 0; k < K; ++k) {
        float* to = lds + ((k * waves + wave) * kLanes + at) * TOK;
        if constexpr (TOK == 1) {
            const float h = join32(s[k][0], s[k][0]);
            const float v = join16(h, h);
            if (row == 0) *to = v;
        } else {
            constexpr int PART = TOK / 4;  // tokens that one group of a wave sums up
            float h[TOK / 2];
#pragma unroll
            for (int j = 0; j < TOK / 2; ++j) h[j] = join32(s[k][j], s[k][TOK / 2 + j]);
            // rows 0 and 1 keep the first half of the tokens, rows 0 and 2 its first half
            to += (row >> 1) * (TOK / 2) + (row & 1) * PART;
#pragma unroll
            for (int j = 0; j < PART; ++j) to[j] = join16(h[j], h[PART + j]);
        }
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const float* from = lds + (k * waves * kLanes + at) * TOK;
#pragma unroll
        for (int j = 0; j < TOK; ++j) s[k][j] = from[j];
        for (int w = 1; w < waves; ++w)
#pragma unroll
            for (int j = 0; j < TOK; ++j) s[k][j] += from[w * kLanes * TOK + j];
    }
}

__device__ __forceinline__ float rsqrt_of(float sum, float inv_c, float eps) {
    return __builtin_amdgcn_rsqf(__builtin_fmaf(sum, inv_c, eps));
}

// A thread's tokens of one channel, as they lie.
template <typename T, int TOK> struct __attribute__((packed, aligned(sizeof(T)))) Words {
    typename std::conditional<TOK * sizeof(T) < 4, uint16_t, uint32_t>::type
        w[TOK * sizeof(T) < 4 ? 1 : TOK * sizeof(T) / 4];
};
template <typename T, int TOK> struct Toks {
    Words<T, TOK> u;
    __device__ __forceinline__ float operator[](int j) const {
        if constexpr (sizeof(T) == 4) return __uint_as_float(u.w[j]);
        else if constexpr (TOK == 1) return Elt<T>::from_bits(u.w[0]);
        else return __uint_as_float(j & 1 ? u.w[j / 2] & 0xffff0000u : u.w[j / 2] << 16);
    }
    // The tokens at p, or without ALL, where p is `over` tokens (0 .. TOK) before its place
    // so that none lies behind the row's end, those from `over` on.
    template <bool ALL> __device__ __forceinline__ void load(const T* p, int over) {
        u = *reinterpret_cast<const Words<T, TOK>*>(p);
        if constexpr (!ALL && TOK > 1) {
            constexpr int N = TOK * sizeof(T) / 4;
            const int words = over * (int)sizeof(T) / 4;
#pragma unroll
            for (int m = N; m >= 1; m >>= 1)
#pragma unroll
                for (int i = 0; i < N; ++i) u.w[i] = words & m ? (i + m < N ? u.w[i + m] : 0u) : u.w[i];
            if constexpr (sizeof(T) == 2) {
                const uint32_t bits = over & 1 ? 16u : 0u;
#pragma unroll
                for (int i = 0; i < N; ++i)
                    u.w[i] = __builtin_amdgcn_alignbit(i + 1 < N ? u.w[i + 1] : 0u, u.w[i], bits);
            }
        }
    }
};
template <typename T, int TOK, bool ALL>
__device__ __forceinline__ void put_tokens(T* p, int left, const float (&o)[TOK]) {
    if (ALL || left == TOK) {
        Words<T, TOK> u;
#pragma unroll
        for (int j = 0; j < TOK; j += 4 / (int)sizeof(T)) {
            if constexpr (sizeof(T) == 4) u.w[j] = __float_as_uint(o[j]);
            else if constexpr (TOK == 1) u.w[0] = Elt<T>::to_bits(o[0]);
            else u.w[j / 2] = pack_bf16x2(o[j], o[j + 1]);
        }
        *reinterpret_cast<Words<T, TOK>*>(p) = u;
    } else {
#pragma unroll
        for (int j = 0; j < TOK; ++j)
            if (j < left) Elt<T>::st(p + j, o[j]);
    }
}

// PC: channels a thread, held in registers, c <= PC * groups; 0: any number, read again
// for every sum.
template <typename T, int TOK, int PC, NormMode MODE, bool GATED, bool NEXT, int THREADS>
__global__ __launch_bounds__(THREADS) void block_norm_k(NormArgs a) {
    constexpr bool kBwd = MODE == PRE_BWD || MODE == POST_BWD;
    constexpr bool kPost = MODE == POST_FWD || MODE == POST_BWD;
    constexpr bool kNext = kBwd ? MODE == PRE_BWD || NEXT : NEXT;  // a norm of y
    constexpr int TILE = kLanes * TOK, NP = PC ? PC : 1;
    constexpr int K = !kBwd ? 1 : kNext && kPost ? 3 : kNext ? 2 : 1;
    typedef Toks<T, TOK> V;
    __shared__ float lds[2][K * (THREADS / 64) * kLanes * TOK];
    const int at = threadIdx.x & 15, grp = threadIdx.x >> 4;
    const int waves = (a.groups * kLanes + 63) >> 6;
    const int rounds = PC ? 1 : (a.c + a.groups - 1) / a.groups;
    const float inv_c = 1.f / (float)a.c;
    const float* gn = MODE == PRE_BWD ? a.gamma : a.next;

    double sum_n[NP], sum_t[NP];  // PC: the gains' gradients over this workgroup's tiles
#pragma unroll
    for (int p = 0; p < NP; ++p) sum_n[p] = sum_t[p] = 0.0;
    auto put_gain = [&](int which, int ch, double v, bool more) {
#pragma unroll
        for (int m = 8; m >= 1; m >>= 1) v += __shfl_xor(v, m);
        if (at == 0 && ch < a.c) {
            float* to = a.part + ((int64_t)which * a.c + ch) * gridDim.x + blockIdx.x;
            *to = more ? *to + (float)v : (float)v;
        }
    };

    auto tile = [&](int64_t t, int64_t vol, int64_t first, auto all_) {
        constexpr bool kAll = decltype(all_)::value;  // every token and channel is there
        const int64_t t0 = first + at * TOK;
        int left = TOK, over = 0;
        uint32_t live = (1u << TOK) - 1u;
        if (!kAll) {
            left = (int)(a.V - t0 < TOK ? (a.V - t0 > 0 ? a.V - t0 : 0) : TOK);
            over = TOK - left;
            live = (1u << left) - 1u;
            if (a.mask)
#pragma unroll
                for (int j = 0; j < TOK; ++j)
                    if (j < left && !a.mask[vol * a.V + t0 + j]) live &= ~(1u << j);
        }
        // where the thread's tokens of its first channel lie, from its last row's end
        // counted back where they do not fill it
        const int64_t at0 = kAll || left == TOK ? t0 : a.V - TOK;
        const int64_t step = (int64_t)a.groups * a.V;
        V X[NP], Z[NP], G[NP], Y[NP], DU[NP];  // backward: X is dy (before a block dres)
        uint32_t on[NP];
        int ch[NP];
        auto load = [&](int k) {
#pragma unroll
            for (int p = 0; p < NP; ++p) {
                const int c = grp + (k + p) * a.groups;
                ch[p] = c;
                on[p] = c < a.c ? live : 0u;
            }
            auto get = [&](V(&to)[NP], const void* q, int64_t stride) {
                const T* from = (const T*)q + vol * stride + at0;
#pragma unroll
                for (int p = 0; p < NP; ++p)
                    to[p].template load<kAll>(
                        from + (kAll ? grp * a.V + (k + p) * step : (int64_t)(ch[p] < a.c ? ch[p] : a.c - 1) * a.V),
                        over);
            };
            if (kBwd && kNext) {
                get(Y, a.y, a.sy);
                get(DU, a.du, a.su);
            }
            if (kPost) get(Z, a.z, a.sz);
            if (GATED) get(G, a.g, a.sg);
            if (!kBwd) get(X, a.x, a.sx);
            else if (MODE == POST_BWD) get(X, a.dy, a.sy);
            else if (a.dy) get(X, a.dy, a.sx);
        };
        // a masked token's value is 0, whatever it holds
        auto val = [&](const V& v, int p, int j) { return kAll || on[p] >> j & 1u ? v[j] : 0.f; };
        auto put = [&](void* q, int64_t stride, int p, const float (&o)[TOK]) {
            if (kAll || ch[p] < a.c)
                put_tokens<T, TOK, kAll>((T*)q + vol * stride + (int64_t)ch[p] * a.V + t0, left, o);
        };
        // What is formed from a held value is formed again behind a barrier, not held too:
        // the registers are what limits the waves.
        auto forget = [&](V& v) {
#pragma unroll
            for (auto& w : v.u.w) asm volatile("" : "+v"(w));
        };
        auto again = [&]() {
            if (PC == 0) return;
#pragma unroll
            for (int p = 0; p < NP; ++p) {
                if (kBwd && kNext) {
                    forget(Y[p]);
                    forget(DU[p]);
                }
                if (kPost) forget(Z[p]);
                if (GATED) forget(G[p]);
                forget(X[p]);
            }
        };
        // all of the thread's channels
        auto each = [&](auto f) {
            for (int k = 0; k < rounds; ++k) {
                if (!PC) load(k);
#pragma unroll
                for (int p = 0; p < NP; ++p) {
                    f(p);
                    __builtin_amdgcn_sched_barrier(0);  // a channel's registers for the next
                }
            }
        };
        auto of = [&](const float* v, int p) { return v[kAll || ch[p] < a.c ? ch[p] : 0]; };
        auto gain = [&](int p) { return of(a.gamma, p) * (a.scale ? of(a.scale, p) : 1.f); };
        // the gate's value and slope
        auto gate = [&](int p, int j, float& phi, float& slope) {
            phi = 1.f;
            slope = 0.f;
            if (GATED) {
                const float g = val(G[p], p, j);
                const Sig sg(g);
                phi = a.gate == RAT3D_GATE_SILU ? g * sg.s : sg.s;
                slope = sg.s * (a.gate == RAT3D_GATE_SILU ? 1.f + g * sg.rest : sg.rest);
            }
        };
        if (PC) load(0);
        float s[K][TOK], e[1][TOK];
        auto clear = [&](auto& v) {
            for (auto& row : v)
                for (float& x : row) x = 0.f;
        };

        if constexpr (!kBwd) {
            clear(e);
            each([&](int p) {
#pragma unroll
                for (int j = 0; j < TOK; ++j) {
                    const float v = val(kPost ? Z[p] : X[p], p, j);
                    e[0][j] += v * v;
                }
            });
            channel_sums(e, lds[0], waves);
            again();
            float r[TOK];
#pragma unroll
            for (int j = 0; j < TOK; ++j) r[j] = rsqrt_of(e[0][j], inv_c, a.eps);
            if constexpr (MODE == PRE_FWD) {
                each([&](int p) {
                    const float k = of(a.gamma, p);
                    float u[TOK];
#pragma unroll
                    for (int j = 0; j < TOK; ++j) u[j] = k * (val(X[p], p, j) * r[j]);
                    put(a.ou, a.su, p, u);
                });
            } else {
                auto value = [&](int p, float (&y)[TOK]) {
                    const float k = gain(p);
#pragma unroll
                    for (int j = 0; j < TOK; ++j) {
                        float phi, slope;
                        gate(p, j, phi, slope);
                        const float b = k * phi * (val(Z[p], p, j) * r[j]);
                        y[j] = X[p][j] + (kAll || on[p] >> j & 1u ? b : 0.f);
                    }
                };
                if constexpr (!NEXT) {
                    each([&](int p) {
                        float y[TOK];
                        value(p, y);
                        put(a.oy, a.sy, p, y);
                    });
                } else {
                    clear(e);
                    each([&](int p) {
                        float y[TOK];
                        value(p, y);
#pragma unroll
                        for (int j = 0; j < TOK; ++j) {
                            const float v = kAll || on[p] >> j & 1u ? y[j] : 0.f;
                            e[0][j] += v * v;
                        }
                    });
                    channel_sums(e, lds[1], waves);
                    again();
                    float ry[TOK];
#pragma unroll
                    for (int j = 0; j < TOK; ++j) ry[j] = rsqrt_of(e[0][j], inv_c, a.eps);
                    each([&](int p) {
                        float y[TOK];
                        value(p, y);
                        put(a.oy, a.sy, p, y);
                        const float k = of(a.next, p);
#pragma unroll
                        for (int j = 0; j < TOK; ++j)
                            y[j] = kAll || on[p] >> j & 1u ? k * (y[j] * ry[j]) : 0.f;
                        put(a.ou, a.su, p, y);
                    });
                }
            }
        } else {
            clear(s);
            each([&](int p) {
                const float k = kNext ? of(gn, p) : 0.f;
#pragma unroll
                for (int j = 0; j < TOK; ++j) {
                    if constexpr (kPost) {
                        const float z = val(Z[p], p, j);
                        s[0][j] += z * z;
                    }
                    if constexpr (kNext) {
                        const float y = val(Y[p], p, j);
                        s[K - 2][j] += y * y;
                        s[K - 1][j] += k * val(DU[p], p, j) * y;
                    }
                }
            });
            channel_sums(s, lds[0], waves);
            again();
            float ry[TOK], my[TOK], rz[TOK], mz[TOK];
#pragma unroll
            for (int j = 0; j < TOK; ++j) {
                if constexpr (kNext) {
                    ry[j] = rsqrt_of(s[K - 2][j], inv_c, a.eps);
                    my[j] = s[K - 1][j] * inv_c * (ry[j] * ry[j]);
                }
                if constexpr (kPost) rz[j] = rsqrt_of(s[0][j], inv_c, a.eps);
            }
            // dY
            auto total = [&](int p, int j, float k) {
                float d = MODE == POST_BWD || a.dy ? X[p][j] : 0.f;
                if constexpr (kNext)
                    if (kAll || on[p] >> j & 1u)
                        d += ry[j] * (k * DU[p][j] - Y[p][j] * my[j]);
                return d;
            };
            if constexpr (kPost) {
                clear(e);
                each([&](int p) {
                    const float k = kNext ? of(gn, p) : 0.f, w = gain(p);
#pragma unroll
                    for (int j = 0; j < TOK; ++j) {
                        float phi, slope;
                        gate(p, j, phi, slope);
                        const float d = total(p, j, k);
                        e[0][j] += (kAll || on[p] >> j & 1u ? d : 0.f) * w * phi * val(Z[p], p, j);
                    }
                });
                channel_sums(e, lds[1], waves);
                again();
#pragma unroll
                for (int j = 0; j < TOK; ++j) mz[j] = e[0][j] * inv_c * (rz[j] * rz[j]);
            }
            each([&](int p) {
                const float k = kNext ? of(gn, p) : 0.f;
                float dY[TOK], n = 0.f, q = 0.f;
#pragma unroll
                for (int j = 0; j < TOK; ++j) {
                    dY[j] = total(p, j, k);
                    if constexpr (kNext) n += val(DU[p], p, j) * (val(Y[p], p, j) * ry[j]);
                }
                if constexpr (kPost) {
                    const float w = gain(p);
                    float dz[TOK], dg[TOK];
#pragma unroll
                    for (int j = 0; j < TOK; ++j) {
                        float phi, slope;
                        gate(p, j, phi, slope);
                        const float z = val(Z[p], p, j), zr = z * rz[j];
                        const float d = kAll || on[p] >> j & 1u ? dY[j] : 0.f;
                        q += d * phi * zr;
                        dz[j] = rz[j] * (d * w * phi - z * mz[j]);
                        dg[j] = d * w * zr * slope;
                    }
                    put(a.dz, a.sz, p, dz);
                    if (GATED) put(a.dg, a.sg, p, dg);
                }
                if (MODE == PRE_BWD || kNext || a.dx) put(a.dx, a.sx, p, dY);
                if constexpr (PC != 0) {
                    sum_n[p] += (double)n;
                    sum_t[p] += (double)q;
                } else {
                    const bool more = t != blockIdx.x;
                    if (kNext) put_gain(0, ch[p], (double)n, more);
                    if (kPost) put_gain(1, ch[p], (double)q, more);
                }
            });
        }
        // the first sums are written again only behind the barrier of the second, the
        // second only behind that of the next first
        if constexpr (!(kPost && (kBwd || NEXT))) __syncthreads();
    };

    for (int64_t t = blockIdx.x; t < a.all; t += gridDim.x) {
        const int64_t vol = t / a.tiles, first = (t - vol * a.tiles) * TILE;
        if (a.mask || first + TILE > a.V || a.c != NP * rounds * a.groups)
            tile(t, vol, first, std::false_type{});
        else tile(t, vol, first, std::true_type{});
    }
    if constexpr (kBwd && PC != 0) {
#pragma unroll
        for (int p = 0; p < NP; ++p) {
            if (kNext) put_gain(0, grp + p * a.groups, sum_n[p], false);
            if (kPost) put_gain(1, grp + p * a.groups, sum_t[p], false);
        }
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
        s += (double)part[((int64_t)which * c + ch) * parts + i];
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
// Tokens and channels a thread: 16 bytes of 4 channels up to 256 of them, 8 bytes of 8 up
// to 512, beyond that nothing is held.
struct NormShape {
    int tok, pc;
};
static NormShape norm_shape(const rat3d_norm_desc& d) {
    const int tok = d.dtype == RAT3D_BF16 ? 8 : 4;
    if (d.v < tok) return {1, d.c <= 256 ? 4 : 0};
    return {tok, d.c <= 256 ? 4 : 0};
}

static void norm_plan(const rat3d_norm_desc& d, NormArgs* a) {
    const int64_t packed = (int64_t)d.c * d.v;
    const NormShape shape = norm_shape(d);
    a->sx = d.x_stride ? d.x_stride : packed;
    a->sz = d.z_stride ? d.z_stride : packed;
    a->sg = d.g_stride ? d.g_stride : packed;
    a->sy = d.y_stride ? d.y_stride : packed;
    a->su = d.u_stride ? d.u_stride : packed;
    a->V = d.v;
    a->c = d.c;
    a->eps = d.eps;
    a->gate = d.gate;
    // whole waves
    a->groups = shape.pc ? (int)ceil_div(ceil_div(d.c, shape.pc), 4) * 4 : 16;
    a->tiles = (int)ceil_div(d.v, kLanes * shape.tok);
    a->all = (int64_t)a->tiles * d.n;
}

static int norm_grid(const NormArgs& a, bool bwd) {
    const int64_t most = bwd ? 8 * (int64_t)device_cus() : 1 << 24;
    return (int)(a.all < most ? a.all : most);
}

size_t norm_ws_bytes(const rat3d_norm_desc& d) {
    NormArgs a = {};
    norm_plan(d, &a);
    return (size_t)norm_grid(a, true) * 2 * d.c * sizeof(float);
}

template <NormMode MODE, bool GATED, bool NEXT>
static void norm_launch(const rat3d_norm_desc& d, const NormArgs& a, hipStream_t st) {
    const int grid = norm_grid(a, MODE == PRE_BWD || MODE == POST_BWD), threads = a.groups * kLanes;
    const NormShape shape = norm_shape(d);
#define RAT3D_NORM(T, TOK, PC, THREADS) \
    block_norm_k<T, TOK, PC, MODE, GATED, NEXT, THREADS><<<grid, threads, 0, st>>>(a)
#define RAT3D_NORM_T(T, TOK)                                     \
    do {                                                         \
        if (shape.tok == 1 && shape.pc) RAT3D_NORM(T, 1, 4, 1024); \
        else if (shape.tok == 1) RAT3D_NORM(T, 1, 0, 256);       \
        else if (shape.pc == 0) RAT3D_NORM(T, TOK, 0, 256);      \
        else if (threads <= 256) RAT3D_NORM(T, TOK, 4, 256);     \
        else RAT3D_NORM(T, TOK, 4, 1024);                        \
    } while (0)
    if (d.dtype == RAT3D_BF16) RAT3D_NORM_T(bf16, 8);
    else RAT3D_NORM_T(float, 4);
#undef RAT3D_NORM_T
#undef RAT3D_NORM
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
    const int parts = norm_grid(a, true);
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
