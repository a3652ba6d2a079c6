// Norm of each head's query and key vector and its rotation by the voxel's place,
// forward and backward, on channel-first maps.
//
// Forward, for one head and token: z = x g r, r = 1/sqrt(mean x^2 + eps); each pair
// of channels (a, b) of an axis is turned, (a cos - b sin, a sin + b cos).
// Backward: the turn is orthogonal, so dz is the incoming gradient turned back, and
//   dg = sum dz x r,   dx = r (g dz - x r^2 mean(g dz x)).
// r is formed again from x, which the backward reads anyway: nothing is saved.
//
// The angles depend on the grid alone: a table of (cos, sin) for each axis, pair and
// place (a few KB, formed in float64) is made once.
//
// Layout: a workgroup takes 128 or 256 neighbouring tokens of one head after another,
// queries' heads and then keys': 32 lanes along the tokens, four or eight tokens each
// (one 8- or 16-byte access a channel), by 8 to 24 groups of threads along the head's
// channel pairs, so that both halves of a pair are in one thread and a channel's row
// is read in whole cache lines.  The cosines and sines are loaded once for all heads.  The sum
// over the head's channels goes through LDS.  Rows need no alignment.
// Bound: HBM, every tensor once.
#include <type_traits>

#include "kernels.hpp"
#include "prof.hpp"

namespace rat3d {

// A head's channels as pairs: the three axes' turned pairs, then what is left in
// twos (turned by nothing).
struct QkPairs {
    int head_dim, half[3];  // pairs of each axis
    int size[3];            // places on each axis
    int64_t tab[3];         // first (cos, sin) of each axis in the table
};

struct QkSide {  // queries or keys
    const void* x;   // the norm's input
    const void* dy;  // backward: gradient of the result
    void* out;       // the result, or the input's gradient
    const float* gamma;
    int64_t x_stride, y_stride;  // from one volume to the next, of x (and dx), of y (and dy)
};

struct QkArgs {
    QkSide side[2];
    QkPairs pr;
    const float2* table;
    float* part;   // backward: partial gradients of the gains, [side][channel][part]
    int parts;     // workgroups
    int heads, kv; // the heads of both sides in one list, queries first
    int chunk, chunks;  // heads that a workgroup takes one after another; ceil(all / chunk)
    int n, H, W;
    int64_t V;
    float eps;
    int tiles;
};

// TOK tokens of one channel, in words: a row may begin at any element.  Without ALL only
// `left` of them are in the row, whose last token lies at p[end] (end may be negative):
// it is read in the others' place, without a branch, and they count as 0.  (The
// backward branches instead: its registers are full.)
template <typename T, int TOK> struct __attribute__((packed, aligned(sizeof(T)))) Toks {
    uint32_t w[TOK * sizeof(T) / 4];
};
template <typename T, int TOK, bool ALL, bool BRANCH>
__device__ __forceinline__ void ld_tok(const T* p, int left, int end, float (&o)[TOK]) {
    if (ALL) {
        const Toks<T, TOK> u = *reinterpret_cast<const Toks<T, TOK>*>(p);
#pragma unroll
        for (int j = 0; j < TOK; ++j) {
            if (sizeof(T) == 4) o[j] = __uint_as_float(u.w[j]);
            else o[j] = __uint_as_float(j & 1 ? u.w[j / 2] & 0xffff0000u : u.w[j / 2] << 16);
        }
    } else if (BRANCH) {
#pragma unroll
        for (int j = 0; j < TOK; ++j) o[j] = j < left ? Elt<T>::ld(p + j) : 0.f;
    } else {
        T u[TOK];
#pragma unroll
        for (int j = 0; j < TOK; ++j) u[j] = p[j < end ? j : end];
#pragma unroll
        for (int j = 0; j < TOK; ++j) o[j] = j < left ? Elt<T>::from_bits(u[j]) : 0.f;
    }
}
template <typename T, int TOK, bool ALL>
__device__ __forceinline__ void st_tok(T* p, int left, const float (&o)[TOK]) {
    if (ALL || left == TOK) {
        Toks<T, TOK> u;
#pragma unroll
        for (int j = 0; j < TOK; j += sizeof(T) == 4 ? 1 : 2) {
            if (sizeof(T) == 4) u.w[j] = __float_as_uint(o[j]);
            else u.w[j / 2] = pack_bf16x2(o[j], o[(j + 1) % TOK]);
        }
        *reinterpret_cast<Toks<T, TOK>*>(p) = u;
    } else {
#pragma unroll
        for (int j = 0; j < TOK; ++j)
            if (j < left) Elt<T>::st(p + j, o[j]);
    }
}

// The lower half of a wave gets x of both halves added, the upper half y.
__device__ __forceinline__ float join_groups(float x, float y) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(y), false,
                                                    false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// G: thread groups along the channel pairs, PP: pairs per thread, TOK: tokens per thread.
// The backward's waves a SIMD are held to what measured best at 8 x (4 + 2) heads over
// 24x28x24 voxels: head_dim 64 (16 groups of 2 pairs) 93 -> 73 us in bfloat16 at four;
// 40 (8 of 3) 50 -> 46 at three, but 81 -> 85 in float32, which is left alone.
template <typename T, int G, int PP, int TOK, bool NORM, bool BWD>
__global__ __launch_bounds__(32 * G, (BWD && PP * TOK == 8                        ? 4
                                      : BWD && G == 8 && PP == 3 && sizeof(T) == 2 ? 3
                                                                                   : 2))
void qk_rope_k(QkArgs a) {
    constexpr int TILE = 32 * TOK;
    // sums over a wave's channels: [parity][sum][wave][token of the lane][lane]
    __shared__ float sums[2][BWD ? 2 : 1][G / 2][TOK][32];
    const float inv_d = 1.f / (float)a.pr.head_dim;
    const int lane = threadIdx.x & 31, grp = threadIdx.x >> 5;
    int bid = blockIdx.x;
    const int tile = bid % a.tiles;
    bid /= a.tiles;
    const int c = bid % a.chunks;
    const int vol = bid / a.chunks;
    const int64_t t0 = (int64_t)tile * TILE + lane * TOK;
    const int left = (int)(a.V - t0 < TOK ? (a.V - t0 > 0 ? a.V - t0 : 0) : TOK);
    const int end = (int)(a.V - 1 - t0 < TOK ? a.V - 1 - t0 : TOK);
    const int D = a.pr.head_dim;

    // this thread's channels and their cosines and sines, the same for every head
    int ca[PP], cb[PP];
    float cs[PP][TOK], sn[PP][TOK];
    {
        // one division for the first token (32 bits: a launch holds fewer than 2^31
        // tokens), steps for its neighbours
        int at[TOK][3];
        const uint32_t first = left > 0 ? (uint32_t)t0 : 0u;
        const uint32_t r0 = first / (uint32_t)a.W;
        at[0][2] = (int)(first - r0 * (uint32_t)a.W);
        at[0][0] = (int)(r0 / (uint32_t)a.H);
        at[0][1] = (int)(r0 - (uint32_t)at[0][0] * (uint32_t)a.H);
#pragma unroll
        for (int j = 1; j < TOK; ++j) {
            const bool step = j < left;
            const bool row_end = step && at[j - 1][2] + 1 == a.W;
            const bool plane_end = row_end && at[j - 1][1] + 1 == a.H;
            at[j][2] = row_end ? 0 : at[j - 1][2] + (step ? 1 : 0);
            at[j][1] = plane_end ? 0 : at[j - 1][1] + (row_end ? 1 : 0);
            at[j][0] = at[j - 1][0] + (plane_end ? 1 : 0);
        }
        const bool row = left == TOK && at[0][2] + TOK - 1 == at[TOK - 1][2];  // all in one row
        const int e0 = a.pr.half[0], e1 = e0 + a.pr.half[1], e2 = e1 + a.pr.half[2];
#pragma unroll
        for (int p = 0; p < PP; ++p) {
            const int i = grp + p * G;  // pair of the head
            const float2* tab = nullptr;
            int axis = 0;
            if (i < e0) {
                ca[p] = i;
                cb[p] = i + a.pr.half[0];
                tab = a.table + a.pr.tab[0] + (int64_t)i * a.pr.size[0];
            } else if (i < e1) {
                axis = 1;
                ca[p] = 2 * e0 + i - e0;
                cb[p] = ca[p] + a.pr.half[1];
                tab = a.table + a.pr.tab[1] + (int64_t)(i - e0) * a.pr.size[1];
            } else if (i < e2) {
                axis = 2;
                ca[p] = 2 * e1 + i - e1;
                cb[p] = ca[p] + a.pr.half[2];
                tab = a.table + a.pr.tab[2] + (int64_t)(i - e1) * a.pr.size[2];
            } else {
                ca[p] = 2 * i;
                cb[p] = 2 * i + 1;
            }
            if (ca[p] >= D) ca[p] = -1;
            if (cb[p] >= D) cb[p] = -1;
#pragma unroll
            for (int j = 0; j < TOK; ++j) {
                cs[p][j] = 1.f;
                sn[p][j] = 0.f;
            }
            if (TOK == 4) {
                // without a branch, so that every load is in flight at once: small maps
                // wait for little else
                if (a.table) {
                    const float2* t = tab ? tab : a.table;
                    float2 v[TOK];
#pragma unroll
                    for (int j = 0; j < TOK; ++j)
                        v[j] = t[!tab ? 0 : axis == 0 ? at[j][0] : axis == 1 ? at[j][1] : at[j][2]];
#pragma unroll
                    for (int j = 0; j < TOK; ++j) {
                        cs[p][j] = tab ? v[j].x : 1.f;
                        sn[p][j] = tab ? v[j].y : 0.f;
                    }
                }
            } else if (tab && row) {
                // one row: one place on the first two axes, neighbours on the third
                if (axis < 2) {
                    const float2 v = tab[axis == 0 ? at[0][0] : at[0][1]];
#pragma unroll
                    for (int j = 0; j < TOK; ++j) {
                        cs[p][j] = v.x;
                        sn[p][j] = v.y;
                    }
                } else {
#pragma unroll
                    for (int j = 0; j < TOK; j += 2) {
                        float v[4];
                        ld_tok<float, 4, true, false>(
                            reinterpret_cast<const float*>(tab + at[0][2] + j), 4, 3, v);
                        cs[p][j] = v[0];
                        sn[p][j] = v[1];
                        cs[p][j + 1] = v[2];
                        sn[p][j + 1] = v[3];
                    }
                }
            } else if (tab) {
#pragma unroll
                for (int j = 0; j < TOK; ++j) {
                    const float2 v =
                        tab[axis == 0 ? at[j][0] : axis == 1 ? at[j][1] : at[j][2]];
                    cs[p][j] = v.x;
                    sn[p][j] = v.y;
                }
            }
        }
    }

    float ga[PP], gb[PP], dga[PP], dgb[PP];
    const int all = a.heads + a.kv;
    const int h0 = c * a.chunk, h1 = h0 + a.chunk < all ? h0 + a.chunk : all;
    // partial gradients of one side's gains, added up over this workgroup's tokens
    auto put_gains = [&](int si) {
#pragma unroll
        for (int p = 0; p < PP; ++p) {
            float u = dga[p], v = dgb[p];
#pragma unroll
            for (int m = 16; m >= 1; m >>= 1) {
                u += __shfl_xor(u, m);
                v += __shfl_xor(v, m);
            }
            if (lane == 0) {
                float* to = a.part + (int64_t)si * D * a.parts + blockIdx.x;
                if (ca[p] >= 0) to[(int64_t)ca[p] * a.parts] = u;
                if (cb[p] >= 0) to[(int64_t)cb[p] * a.parts] = v;
            }
            dga[p] = dgb[p] = 0.f;
        }
    };
#pragma unroll
    for (int p = 0; p < PP; ++p) dga[p] = dgb[p] = 0.f;
    if (BWD && NORM) {
        if (h0 >= a.heads) put_gains(0);  // no head of that side here: zeros
        if (h1 <= a.heads) put_gains(1);
    }

    int par = 0;
    auto head = [&](int h, auto all) {
        constexpr bool kAll = decltype(all)::value;
        const int si = h >= a.heads ? 1 : 0;
        const QkSide& s = a.side[si];
        if (h == h0 || h == a.heads) {
            if (BWD && NORM && h != h0) put_gains(0);
#pragma unroll
            for (int p = 0; p < PP; ++p) {
                ga[p] = NORM && ca[p] >= 0 ? s.gamma[ca[p]] : 1.f;
                gb[p] = NORM && cb[p] >= 0 ? s.gamma[cb[p]] : 1.f;
            }
        }
        const int64_t first = (int64_t)(si ? h - a.heads : h) * D * a.V + t0;
        const T* x = (const T*)s.x + vol * s.x_stride + first;
        const T* dy = BWD ? (const T*)s.dy + vol * s.y_stride + first : nullptr;
        T* out = (T*)s.out + vol * (BWD ? s.x_stride : s.y_stride) + first;
        float xa[PP][TOK], xb[PP][TOK];
        float da[PP][TOK], db[PP][TOK];
        const bool reads = NORM || !BWD;  // without a norm the backward needs dy alone
        // a channel that is none is read from the head's first and counts as 0
#pragma unroll
        for (int p = 0; p < PP; ++p) {
            const int64_t fa = (ca[p] >= 0 ? ca[p] : 0) * a.V, fb = (cb[p] >= 0 ? cb[p] : 0) * a.V;
            if (reads) {
                ld_tok<T, TOK, kAll, BWD>(x + fa, left, end, xa[p]);
                ld_tok<T, TOK, kAll, BWD>(x + fb, left, end, xb[p]);
            }
            if (BWD) {
                ld_tok<T, TOK, kAll, BWD>(dy + fa, left, end, da[p]);
                ld_tok<T, TOK, kAll, BWD>(dy + fb, left, end, db[p]);
            }
        }
#pragma unroll
        for (int p = 0; p < PP; ++p)
#pragma unroll
            for (int j = 0; j < TOK; ++j) {
                if (ca[p] < 0) xa[p][j] = da[p][j] = 0.f;
                if (cb[p] < 0) xb[p][j] = db[p][j] = 0.f;
            }
        float rs[TOK], mean[TOK];
        if (BWD) {
#pragma unroll
            for (int p = 0; p < PP; ++p)
#pragma unroll
                for (int j = 0; j < TOK; ++j) {
                    const float u = da[p][j], v = db[p][j];
                    da[p][j] = u * cs[p][j] + v * sn[p][j];
                    db[p][j] = v * cs[p][j] - u * sn[p][j];
                }
        }
        if (NORM) {
            float ss[TOK], sd[TOK];
#pragma unroll
            for (int j = 0; j < TOK; ++j) {
                ss[j] = sd[j] = 0.f;
#pragma unroll
                for (int p = 0; p < PP; ++p) {
                    ss[j] += xa[p][j] * xa[p][j] + xb[p][j] * xb[p][j];
                    if (BWD) sd[j] += ga[p] * da[p][j] * xa[p][j] + gb[p] * db[p][j] * xb[p][j];
                }
            }
            // both groups of a wave, then the waves through LDS: each half of a wave
            // writes half of the tokens
            const int half = grp & 1, wave = grp >> 1;
#pragma unroll
            for (int j = 0; j < TOK / 2; ++j) {
                const int k = half * (TOK / 2) + j;
                sums[par][0][wave][k][lane] = join_groups(ss[j], ss[TOK / 2 + j]);
                if (BWD) sums[par][BWD][wave][k][lane] = join_groups(sd[j], sd[TOK / 2 + j]);
            }
            // one barrier a head: the next head writes the other half, and this half
            // is written again only behind that head's barrier
            __syncthreads();
#pragma unroll
            for (int j = 0; j < TOK; ++j) {
                float t = 0.f, d = 0.f;
#pragma unroll
                for (int w = 0; w < G / 2; ++w) {
                    t += sums[par][0][w][j][lane];
                    if (BWD) d += sums[par][BWD][w][j][lane];
                }
                rs[j] = __builtin_amdgcn_rsqf(__builtin_fmaf(t, inv_d, a.eps));
                if (BWD) mean[j] = d * inv_d * (rs[j] * rs[j]);
            }
        }
#pragma unroll
        for (int p = 0; p < PP; ++p) {
            float oa[TOK], ob[TOK];
#pragma unroll
            for (int j = 0; j < TOK; ++j) {
                if (BWD) {
                    if (NORM) {
                        // x r once, and mean[j] already times r^2
                        const float r = rs[j], ya = xa[p][j] * r, yb = xb[p][j] * r;
                        dga[p] = __builtin_fmaf(da[p][j], ya, dga[p]);
                        dgb[p] = __builtin_fmaf(db[p][j], yb, dgb[p]);
                        oa[j] = __builtin_fmaf(-ya, mean[j], r * ga[p] * da[p][j]);
                        ob[j] = __builtin_fmaf(-yb, mean[j], r * gb[p] * db[p][j]);
                    } else {
                        oa[j] = da[p][j];
                        ob[j] = db[p][j];
                    }
                } else {
                    const float za = NORM ? xa[p][j] * rs[j] * ga[p] : xa[p][j];
                    const float zb = NORM ? xb[p][j] * rs[j] * gb[p] : xb[p][j];
                    oa[j] = za * cs[p][j] - zb * sn[p][j];
                    ob[j] = za * sn[p][j] + zb * cs[p][j];
                }
            }
            if (ca[p] >= 0) st_tok<T, TOK, kAll>(out + ca[p] * a.V, left, oa);
            if (cb[p] >= 0) st_tok<T, TOK, kAll>(out + cb[p] * a.V, left, ob);
        }
    };
    const bool inside = (int64_t)(tile + 1) * TILE <= a.V;
    for (int h = h0; h < h1; ++h, par ^= 1) {
        if (inside) head(h, std::true_type{});
        else head(h, std::false_type{});
    }
    if (BWD && NORM) put_gains(h1 > a.heads ? 1 : 0);
}

// dgamma[channel] (+)= the sum of its partial sums, in a fixed order.  In float64: a
// thread adds up to 2 * 10^4 parts one after another, and over 2^27 voxels of equal terms
// float32 drifted by 4.6e-5.  The backward of 16 x (2 + 2) heads x 32 over 48x56x48 takes
// 322 us with either.
__global__ __launch_bounds__(256) void qk_gain_k(const float* __restrict__ part, int parts, int D,
                                                 float* dgq, float* dgk, int accumulate) {
    __shared__ double red[4];
    const int si = blockIdx.x / D, ch = blockIdx.x - si * D;
    float* to = si ? dgk : dgq;
    if (!to) return;
    const float* p = part + ((int64_t)si * D + ch) * parts;
    double s = 0.0;
    for (int i = threadIdx.x; i < parts; i += 256) s += (double)p[i];
#pragma unroll
    for (int m = 32; m >= 1; m >>= 1) s += __shfl_xor(s, m);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
    __syncthreads();
    if (threadIdx.x == 0) {
        const float sum = (float)((red[0] + red[1]) + (red[2] + red[3]));
        to[ch] = accumulate ? to[ch] + sum : sum;
    }
}

// (cos, sin) of every axis, pair and place: the angle in float64 (a place of 2^24
// times a frequency keeps 29 bits behind the point), each result rounded once.
__global__ __launch_bounds__(256) void rope_table_k(QkPairs pr, int o0, int o1, int o2,
                                                    double base, int64_t total, float2* tab) {
    const int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (e >= total) return;
    const int axis = e >= pr.tab[2] ? 2 : e >= pr.tab[1] ? 1 : 0;
    const int64_t i = (e - pr.tab[axis]) / pr.size[axis];
    const int64_t at = (e - pr.tab[axis]) - i * pr.size[axis] + (axis == 0 ? o0 : axis == 1 ? o1 : o2);
    const double ang = (double)at * pow(base, -(double)i / (double)pr.half[axis]);
    double sv, cv;
    sincos(ang, &sv, &cv);
    tab[e] = make_float2((float)cv, (float)sv);
}

// ------------------------------------------------------------------ host
static QkPairs make_pairs(const rat3d_qk_desc& d, int64_t* total) {
    QkPairs p;
    p.head_dim = d.head_dim;
    const int rot[3] = {d.rot_d, d.rot_h, d.rot_w}, size[3] = {d.d, d.h, d.w};
    int64_t at = 0;
    for (int a = 0; a < 3; ++a) {
        p.half[a] = rot[a] / 2;
        p.size[a] = size[a];
        p.tab[a] = at;
        at += (int64_t)p.half[a] * size[a];
    }
    *total = at;
    return p;
}

size_t rope_table_bytes(const rat3d_qk_desc& d) {
    int64_t total;
    make_pairs(d, &total);
    return (size_t)total * sizeof(float2);
}

rat3d_status rope_table(const rat3d_qk_desc& d, void* table, hipStream_t st) {
    int64_t total;
    const QkPairs p = make_pairs(d, &total);
    if (total == 0) return RAT3D_OK;
    rope_table_k<<<(unsigned)ceil_div(total, 256), 256, 0, st>>>(
        p, d.origin_d, d.origin_h, d.origin_w, (double)d.base, total, (float2*)table);
    RAT3D_LAUNCH_CHECK();
    return RAT3D_OK;
}

// Tokens per thread: eight of bfloat16 (one 16-byte access a channel) where that is
// faster and there are tiles enough to fill the GPU, else four.  24 x (4 + 2) heads over
// 24x28x24 voxels, four and eight tokens: forward at head_dim 96 222 and 181 us, at 80
// 321 and 156, but at 48 89 and 101, at 64 119 and 127, at 128 260 and 428 (registers);
// backward at 48 214 and 165, at 64 218 and 204, but at 96 325 and 429.
static int qk_tokens(const rat3d_qk_desc& d, bool bwd) {
    const int64_t V = (int64_t)d.d * d.h * d.w;
    const bool fits = d.dtype == RAT3D_BF16 &&
                      (d.head_dim <= 32 || (bwd ? d.head_dim <= 64
                                                : d.head_dim > 64 && d.head_dim <= 96));
    return fits && ceil_div(V, 256) * d.n >= 4 * (int64_t)device_cus() ? 8 : 4;
}

// Heads per workgroup: as many as leave four workgroups for each CU (the table's
// values are then loaded once for several heads), at least one.
static void qk_plan(const rat3d_qk_desc& d, bool bwd, QkArgs* a) {
    a->V = (int64_t)d.d * d.h * d.w;
    a->n = d.n;
    a->H = d.h;
    a->W = d.w;
    a->eps = d.eps;
    a->heads = d.heads;
    a->kv = d.kv_heads;
    a->tiles = (int)ceil_div(a->V, 32 * qk_tokens(d, bwd));
    const int64_t whole = (int64_t)a->tiles * d.n;
    const int64_t want = ceil_div(4 * (int64_t)device_cus(), whole);  // chunks a volume and tile
    const int both = d.heads + d.kv_heads;
    a->chunk = (int)(both / (want < both ? want : both));
    a->chunks = (int)ceil_div(both, a->chunk);
    a->parts = d.n * a->chunks * a->tiles;
}

size_t qk_ws_bytes(const rat3d_qk_desc& d) {
    if (!d.norm) return 0;
    QkArgs a;
    qk_plan(d, true, &a);
    return (size_t)2 * d.head_dim * a.parts * sizeof(float);
}

template <typename T, bool BWD>
static void qk_launch(const rat3d_qk_desc& d, const QkArgs& a, hipStream_t st) {
    const unsigned grid = (unsigned)a.parts;
    const bool wide = sizeof(T) == 2 && qk_tokens(d, BWD) == 8;
#define RAT3D_QK(G, PP, TOK)                                                          \
    do {                                                                              \
        if (d.norm) qk_rope_k<T, G, PP, TOK, true, BWD><<<grid, 32 * (G), 0, st>>>(a);  \
        else qk_rope_k<T, G, PP, TOK, false, BWD><<<grid, 32 * (G), 0, st>>>(a);        \
    } while (0)
    constexpr bool kFew = sizeof(T) == 2 && !BWD;
    // groups and pairs so that few slots stay empty and four waves a SIMD find registers
    // (8 x 6 heads over 24x28x24 voxels in bfloat16, forward: at head_dim 96 16 groups of
    // 3 pairs 124 us, 24 of 2 85, backward 128 and 129; at 64 16 of 2 42, 8 of 4 36, in
    // float32 76 and 78)
    if constexpr (sizeof(T) == 2) {
        if (wide) {
            if (d.head_dim <= 16) RAT3D_QK(8, 1, 8);
            else if (d.head_dim <= 32) RAT3D_QK(8, 2, 8);
            else if constexpr (!BWD) RAT3D_QK(24, 2, 8);
            else if (d.head_dim <= 48) RAT3D_QK(12, 2, 8);
            else RAT3D_QK(16, 2, 8);
            return;
        }
    }
    if (d.head_dim <= 16) RAT3D_QK(8, 1, 4);
    else if (d.head_dim <= 32) RAT3D_QK(8, 2, 4);
    else if (d.head_dim <= 48) RAT3D_QK(8, 3, 4);
    else if (d.head_dim <= 64) RAT3D_QK(kFew ? 8 : 16, kFew ? 4 : 2, 4);
    else if (d.head_dim <= 96) RAT3D_QK(BWD ? 16 : 24, BWD ? 3 : 2, 4);
    else RAT3D_QK(16, 4, 4);
#undef RAT3D_QK
}

static double qk_bytes(const rat3d_qk_desc& d, int passes) {
    return (double)d.n * (d.heads + d.kv_heads) * d.head_dim * d.d * d.h * d.w * passes *
           (d.dtype == RAT3D_BF16 ? 2 : 4);
}

rat3d_status qk_rope_fwd(const rat3d_qk_desc& d, const void* q, const void* k, const float* gq,
                         const float* gk, const void* table, void* oq, void* ok, hipStream_t st) {
    QkArgs a = {};
    int64_t total;
    a.pr = make_pairs(d, &total);
    qk_plan(d, false, &a);
    a.table = total ? (const float2*)table : nullptr;
    a.side[0].x = q;
    a.side[0].out = oq;
    a.side[0].gamma = gq;
    a.side[0].x_stride = d.q_stride ? d.q_stride : (int64_t)d.heads * d.head_dim * a.V;
    a.side[0].y_stride = d.oq_stride ? d.oq_stride : (int64_t)d.heads * d.head_dim * a.V;
    a.side[1].x = k;
    a.side[1].out = ok;
    a.side[1].gamma = gk;
    a.side[1].x_stride = d.k_stride ? d.k_stride : (int64_t)d.kv_heads * d.head_dim * a.V;
    a.side[1].y_stride = d.ok_stride ? d.ok_stride : (int64_t)d.kv_heads * d.head_dim * a.V;
    ProfScope ps(qk_tokens(d, false) == 8 ? "qk_rope_fwd_8" : "qk_rope_fwd", st, 0.0, qk_bytes(d, 2));
    if (d.dtype == RAT3D_BF16) qk_launch<bf16, false>(d, a, st);
    else qk_launch<float, false>(d, a, st);
    RAT3D_LAUNCH_CHECK();
    return RAT3D_OK;
}

rat3d_status qk_rope_bwd(const rat3d_qk_desc& d, const void* doq, const void* dok, const void* q,
                         const void* k, const float* gq, const float* gk, const void* table,
                         void* dq, void* dk, float* dgq, float* dgk, int accumulate, void* ws,
                         hipStream_t st) {
    QkArgs a = {};
    int64_t total;
    a.pr = make_pairs(d, &total);
    qk_plan(d, true, &a);
    a.table = total ? (const float2*)table : nullptr;
    a.part = (float*)ws;
    a.side[0].x = q;
    a.side[0].dy = doq;
    a.side[0].out = dq;
    a.side[0].gamma = gq;
    a.side[0].x_stride = d.q_stride ? d.q_stride : (int64_t)d.heads * d.head_dim * a.V;
    a.side[0].y_stride = d.oq_stride ? d.oq_stride : (int64_t)d.heads * d.head_dim * a.V;
    a.side[1].x = k;
    a.side[1].dy = dok;
    a.side[1].out = dk;
    a.side[1].gamma = gk;
    a.side[1].x_stride = d.k_stride ? d.k_stride : (int64_t)d.kv_heads * d.head_dim * a.V;
    a.side[1].y_stride = d.ok_stride ? d.ok_stride : (int64_t)d.kv_heads * d.head_dim * a.V;
    {
        ProfScope ps(qk_tokens(d, true) == 8 ? "qk_rope_bwd_8" : "qk_rope_bwd", st, 0.0,
                     qk_bytes(d, 3));
        if (d.dtype == RAT3D_BF16) qk_launch<bf16, true>(d, a, st);
        else qk_launch<float, true>(d, a, st);
        RAT3D_LAUNCH_CHECK();
    }
    if (d.norm) {
        ProfScope ps("qk_gain", st, 0.0, 8.0 * d.head_dim * a.parts);
        qk_gain_k<<<2 * d.head_dim, 256, 0, st>>>(a.part, a.parts, d.head_dim,
                                                  d.heads ? dgq : nullptr,
                                                  d.kv_heads ? dgk : nullptr, accumulate);
        RAT3D_LAUNCH_CHECK();
    }
    return RAT3D_OK;
}

}  // namespace rat3d
