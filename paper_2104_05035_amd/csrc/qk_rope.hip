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
// Layout: a workgroup takes 128 neighbouring tokens of one head after another: 32
// lanes along the tokens, four tokens each (one 8- or 16-byte access a channel), by
// eight groups of threads along the head's channel pairs, so that both halves of a
// pair are in one thread and a channel's row is read in whole cache lines.  The sum
// over the head's channels goes through LDS.  Rows need no alignment.
// Bound: HBM, every tensor once.
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
    int heads;
    int64_t x_stride, y_stride;  // from one volume to the next, of x (and dx), of y (and dy)
    int chunk;                   // heads that a workgroup takes one after another
    int chunks;                  // ceil(heads / chunk)
};

struct QkArgs {
    QkSide side[2];
    QkPairs pr;
    const float2* table;
    float* part;  // backward: partial gradients of the gains, [side][channel][part]
    int parts;    // of one side
    int n, H, W;
    int64_t V;
    float eps;
    int tiles;
};

constexpr int kQkTok = 4;                    // tokens per thread
constexpr int kQkTile = 32 * kQkTok;         // tokens per workgroup
constexpr int kQkGroups = 8;                 // thread groups along the channel pairs

template <typename T> struct __attribute__((packed, aligned(sizeof(T)))) Tok4 { T v[kQkTok]; };

template <typename T>
__device__ __forceinline__ void ld_tok(const T* p, int left, float (&o)[kQkTok]) {
    if (left >= kQkTok) {
        const Tok4<T> u = *reinterpret_cast<const Tok4<T>*>(p);
#pragma unroll
        for (int j = 0; j < kQkTok; ++j) o[j] = Elt<T>::from_bits(u.v[j]);
    } else {
#pragma unroll
        for (int j = 0; j < kQkTok; ++j) o[j] = j < left ? Elt<T>::ld(p + j) : 0.f;
    }
}
template <typename T>
__device__ __forceinline__ void st_tok(T* p, int left, const float (&o)[kQkTok]) {
    if (left >= kQkTok) {
        Tok4<T> u;
#pragma unroll
        for (int j = 0; j < kQkTok; ++j) u.v[j] = Elt<T>::to_bits(o[j]);
        *reinterpret_cast<Tok4<T>*>(p) = u;
    } else {
#pragma unroll
        for (int j = 0; j < kQkTok; ++j)
            if (j < left) Elt<T>::st(p + j, o[j]);
    }
}

// PP: pairs per thread.
template <typename T, int PP, bool NORM, bool BWD>
__global__ __launch_bounds__(256) void qk_rope_k(QkArgs a) {
    __shared__ float sums[2][BWD ? 2 : 1][kQkGroups][kQkTile];  // [parity][sum][group][token]
    const int lane = threadIdx.x & 31, grp = threadIdx.x >> 5;
    int bid = blockIdx.x;
    const int tile = bid % a.tiles;
    bid /= a.tiles;
    const int per = a.side[0].chunks + a.side[1].chunks;
    int c = bid % per;
    const int vol = bid / per;
    const int si = c >= a.side[0].chunks ? 1 : 0;
    if (si) c -= a.side[0].chunks;
    const QkSide& s = a.side[si];
    const int64_t t0 = (int64_t)tile * kQkTile + lane * kQkTok;
    const int left = (int)(a.V - t0 < kQkTok ? (a.V - t0 > 0 ? a.V - t0 : 0) : kQkTok);
    const int D = a.pr.head_dim;

    // this thread's channels and their cosines and sines, the same for every head
    int ca[PP], cb[PP];
    float cs[PP][kQkTok], sn[PP][kQkTok], ga[PP], gb[PP];
    {
        int at[kQkTok][3];
#pragma unroll
        for (int j = 0; j < kQkTok; ++j) {
            const int64_t t = j < left ? t0 + j : 0;
            const int64_t row = t / a.W;
            at[j][2] = (int)(t - row * a.W);
            at[j][0] = (int)(row / a.H);
            at[j][1] = (int)(row - (int64_t)at[j][0] * a.H);
        }
        const int e0 = a.pr.half[0], e1 = e0 + a.pr.half[1], e2 = e1 + a.pr.half[2];
#pragma unroll
        for (int p = 0; p < PP; ++p) {
            const int i = grp + p * kQkGroups;  // pair of the head
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
            for (int j = 0; j < kQkTok; ++j) {
                const float2 v = tab ? tab[axis == 0 ? at[j][0] : axis == 1 ? at[j][1] : at[j][2]]
                                     : make_float2(1.f, 0.f);
                cs[p][j] = v.x;
                sn[p][j] = v.y;
            }
            ga[p] = NORM && ca[p] >= 0 ? s.gamma[ca[p]] : 1.f;
            gb[p] = NORM && cb[p] >= 0 ? s.gamma[cb[p]] : 1.f;
        }
    }

    float dga[PP], dgb[PP];
#pragma unroll
    for (int p = 0; p < PP; ++p) dga[p] = dgb[p] = 0.f;

    const int h1 = (c + 1) * s.chunk < s.heads ? (c + 1) * s.chunk : s.heads;
    int par = 0;
    for (int h = c * s.chunk; h < h1; ++h, par ^= 1) {
        const int64_t row = (int64_t)h * D;
        const T* x = (const T*)s.x + vol * s.x_stride + row * a.V + t0;
        const T* dy = BWD ? (const T*)s.dy + vol * s.y_stride + row * a.V + t0 : nullptr;
        T* out = (T*)s.out + vol * (BWD ? s.x_stride : s.y_stride) + row * a.V + t0;
        float xa[PP][kQkTok], xb[PP][kQkTok];
        float da[PP][kQkTok], db[PP][kQkTok];
        const bool reads = NORM || !BWD;  // without a norm the backward needs dy alone
#pragma unroll
        for (int p = 0; p < PP; ++p) {
            if (reads) ld_tok(x + ca[p] * a.V, ca[p] >= 0 ? left : 0, xa[p]);
            if (reads) ld_tok(x + cb[p] * a.V, cb[p] >= 0 ? left : 0, xb[p]);
            if (BWD) {
                ld_tok(dy + ca[p] * a.V, ca[p] >= 0 ? left : 0, da[p]);
                ld_tok(dy + cb[p] * a.V, cb[p] >= 0 ? left : 0, db[p]);
            }
        }
        float rs[kQkTok], mean[kQkTok];
        if (BWD) {
#pragma unroll
            for (int p = 0; p < PP; ++p)
#pragma unroll
                for (int j = 0; j < kQkTok; ++j) {
                    const float u = da[p][j], v = db[p][j];
                    da[p][j] = u * cs[p][j] + v * sn[p][j];
                    db[p][j] = v * cs[p][j] - u * sn[p][j];
                }
        }
        if (NORM) {
            float ss[kQkTok], sd[kQkTok];
#pragma unroll
            for (int j = 0; j < kQkTok; ++j) {
                ss[j] = sd[j] = 0.f;
#pragma unroll
                for (int p = 0; p < PP; ++p) {
                    ss[j] += xa[p][j] * xa[p][j] + xb[p][j] * xb[p][j];
                    if (BWD) sd[j] += ga[p] * da[p][j] * xa[p][j] + gb[p] * db[p][j] * xb[p][j];
                }
            }
#pragma unroll
            for (int j = 0; j < kQkTok; ++j) {
                sums[par][0][grp][lane * kQkTok + j] = ss[j];
                if (BWD) sums[par][BWD][grp][lane * kQkTok + j] = sd[j];
            }
            // one barrier a head: the next head writes the other half, and this half
            // is written again only behind that head's barrier
            __syncthreads();
#pragma unroll
            for (int j = 0; j < kQkTok; ++j) {
                float t = 0.f, d = 0.f;
#pragma unroll
                for (int g = 0; g < kQkGroups; ++g) {
                    t += sums[par][0][g][lane * kQkTok + j];
                    if (BWD) d += sums[par][BWD][g][lane * kQkTok + j];
                }
                rs[j] = 1.f / sqrtf(t / (float)D + a.eps);
                if (BWD) mean[j] = d / (float)D;
            }
        }
#pragma unroll
        for (int p = 0; p < PP; ++p) {
            float oa[kQkTok], ob[kQkTok];
#pragma unroll
            for (int j = 0; j < kQkTok; ++j) {
                if (BWD) {
                    if (NORM) {
                        const float r = rs[j], f = r * r * mean[j];
                        dga[p] += da[p][j] * xa[p][j] * r;
                        dgb[p] += db[p][j] * xb[p][j] * r;
                        oa[j] = r * (ga[p] * da[p][j] - xa[p][j] * f);
                        ob[j] = r * (gb[p] * db[p][j] - xb[p][j] * f);
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
            st_tok(out + ca[p] * a.V, ca[p] >= 0 ? left : 0, oa);
            st_tok(out + cb[p] * a.V, cb[p] >= 0 ? left : 0, ob);
        }
    }
    if (BWD && NORM) {
        const int part = (vol * s.chunks + c) * a.tiles + tile;
#pragma unroll
        for (int p = 0; p < PP; ++p) {
            float u = dga[p], v = dgb[p];
#pragma unroll
            for (int m = 16; m >= 1; m >>= 1) {
                u += __shfl_xor(u, m);
                v += __shfl_xor(v, m);
            }
            if (lane == 0) {
                float* to = a.part + (int64_t)si * D * a.parts;
                if (ca[p] >= 0) to[(int64_t)ca[p] * a.parts + part] = u;
                if (cb[p] >= 0) to[(int64_t)cb[p] * a.parts + part] = v;
            }
        }
    }
}

// dgamma[channel] (+)= the sum of its partial sums, in a fixed order.
__global__ __launch_bounds__(256) void qk_gain_k(const float* __restrict__ part, int parts,
                                                 int used0, int used1, int D, float* dgq,
                                                 float* dgk, int accumulate) {
    __shared__ float red[4];
    const int si = blockIdx.x / D, ch = blockIdx.x - si * D;
    const int used = si ? used1 : used0;
    float* to = si ? dgk : dgq;
    if (!to) return;
    const float* p = part + ((int64_t)si * D + ch) * parts;
    float s = 0.f;
    for (int i = threadIdx.x; i < used; i += 256) s += p[i];
#pragma unroll
    for (int m = 32; m >= 1; m >>= 1) s += __shfl_xor(s, m);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
    __syncthreads();
    if (threadIdx.x == 0) {
        s = (red[0] + red[1]) + (red[2] + red[3]);
        to[ch] = accumulate ? to[ch] + s : s;
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

// Heads per workgroup: as many as leave four workgroups for each CU (the table's
// values are then loaded once for several heads), at least one.
static void qk_plan(const rat3d_qk_desc& d, QkArgs* a) {
    a->V = (int64_t)d.d * d.h * d.w;
    a->n = d.n;
    a->H = d.h;
    a->W = d.w;
    a->eps = d.eps;
    a->tiles = (int)ceil_div(a->V, kQkTile);
    const int64_t whole = (int64_t)a->tiles * d.n;
    const int64_t want = ceil_div(4 * (int64_t)device_cus(), whole);  // chunks a volume and tile
    const int both = d.heads + d.kv_heads;
    int chunk = (int)(both / (want < both ? want : both));
    if (chunk < 1) chunk = 1;
    const int heads[2] = {d.heads, d.kv_heads};
    for (int i = 0; i < 2; ++i) {
        a->side[i].heads = heads[i];
        a->side[i].chunk = chunk;
        a->side[i].chunks = (int)ceil_div(heads[i], chunk);
    }
    const int most = a->side[0].chunks > a->side[1].chunks ? a->side[0].chunks : a->side[1].chunks;
    a->parts = d.n * most * a->tiles;
}

size_t qk_ws_bytes(const rat3d_qk_desc& d) {
    if (!d.norm) return 0;
    QkArgs a;
    qk_plan(d, &a);
    return (size_t)2 * d.head_dim * a.parts * sizeof(float);
}

template <typename T, bool BWD>
static void qk_launch(const rat3d_qk_desc& d, const QkArgs& a, hipStream_t st) {
    const unsigned grid =
        (unsigned)((int64_t)a.tiles * a.n * (a.side[0].chunks + a.side[1].chunks));
#define RAT3D_QK(PP)                                                        \
    do {                                                                    \
        if (d.norm) qk_rope_k<T, PP, true, BWD><<<grid, 256, 0, st>>>(a);   \
        else qk_rope_k<T, PP, false, BWD><<<grid, 256, 0, st>>>(a);         \
    } while (0)
    if (d.head_dim <= 16) RAT3D_QK(1);
    else if (d.head_dim <= 32) RAT3D_QK(2);
    else if (d.head_dim <= 64) RAT3D_QK(4);
    else RAT3D_QK(8);
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
    qk_plan(d, &a);
    a.table = (const float2*)table;
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
    ProfScope ps("qk_rope_fwd", st, 0.0, qk_bytes(d, 2));
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
    qk_plan(d, &a);
    a.table = (const float2*)table;
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
        ProfScope ps("qk_rope_bwd", st, 0.0, qk_bytes(d, 3));
        if (d.dtype == RAT3D_BF16) qk_launch<bf16, true>(d, a, st);
        else qk_launch<float, true>(d, a, st);
        RAT3D_LAUNCH_CHECK();
    }
    if (d.norm) {
        const int u0 = d.n * a.side[0].chunks * a.tiles, u1 = d.n * a.side[1].chunks * a.tiles;
        ProfScope ps("qk_gain", st, 0.0, 4.0 * d.head_dim * ((double)u0 + u1));
        qk_gain_k<<<2 * d.head_dim, 256, 0, st>>>(a.part, a.parts, u0, u1, d.head_dim,
                                                  d.heads ? dgq : nullptr,
                                                  d.kv_heads ? dgk : nullptr, accumulate);
        RAT3D_LAUNCH_CHECK();
    }
    return RAT3D_OK;
}

}  // namespace rat3d
