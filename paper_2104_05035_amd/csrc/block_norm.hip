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
// its 4 or 8 channels in registers (of half or a quarter as many voxels where they would
// not fit), so every tensor passes once; beyond, and in the backward of large maps beyond
// 256, each sum reads its tensors again.  Sums over a voxel's channels are
// joined by lane swaps that leave each of a wave's four groups a quarter of the voxels,
// and through LDS.  Rows need no alignment.
// Bound: HBM.  Bfloat16, 16 x 64 channels of 48x56x48 voxels: before a block 76 us (its
// input partly in the memory-side cache), its gradient 200 us (5.3 TB/s); behind one with
// gate and next norm 252 us (5.2), its gradient with all eight tensors 437 us (4.8); with a
// mask 93, 209, 254 and 445; float32, 8 x 64 channels: 77, 207, 261 and 430.
#include "kernels.hpp"
#include "prof.hpp"
#include "tokens.hpp"

namespace rat3d {

constexpr int kLanes = 16;  // along the voxels

enum NormMode { PRE_FWD, PRE_BWD, POST_FWD, POST_BWD };

struct NormArgs {
    // forward: x, z, g -> y, u.  Backward: dy, du, y (before a block dres, du, x), z, g ->
    // dx, dz, dg
    const void *x, *z, *g, *y, *dy, *du;
    void *oy, *ou, *dx, *dz, *dg;
    const float *gamma, *scale, *next;
    const uint8_t* mask;
    void* part;  // [gain][channel][workgroup], NormPart
    int64_t sx, sz, sg, sy, su;  // from one volume to the next
    int64_t V;
    int c, groups, gate;
    int stream, near;  // stores past the cache; neighbouring tiles on one XCD
    uint32_t tiles, all;  // of one volume, of all (below 2^31)
    uint32_t base;        // this launch's first tile
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
        } else if constexpr (TOK == 2) {
            const float h = join32(s[k][0], s[k][1]);
            const float v = join16(h, h);
            if (!(row & 1)) to[row >> 1] = v;
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
#pragma unroll 2
        for (int w = 1; w < waves; ++w)
#pragma unroll
            for (int j = 0; j < TOK; ++j) s[k][j] += from[w * kLanes * TOK + j];
    }
}

// Parts of the gains' gradients.  Where channels are read again (PC = 0) a workgroup adds
// every tile's to its part: a float32 one drifts by 190 units of 2^-24 over 862 equal tiles.
template <int PC> using NormPart = typename std::conditional<PC == 0, double, float>::type;

// PC: channels a thread, held in registers, c <= PC * groups; 0: any number, read again
// for every sum.  ALL: no mask, whole tiles, c = PC * groups (in kernels of their own, for
// what the other case needs is formed before the loop and takes registers).
template <typename T, int TOK, int PC, NormMode MODE, bool GATED, bool NEXT, bool ALL, int THREADS>
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
            typedef NormPart<PC> Part;
            Part* to = (Part*)a.part + ((int64_t)which * a.c + ch) * gridDim.x + blockIdx.x;
            *to = (Part)(more ? *to + v : v);
        }
    };

    // the gains of the held channels: gamma scale, and that of the norm of y
    float wgt[NP], nxt[NP];
    auto gains = [&](int round) {
#pragma unroll
        for (int p = 0; p < NP; ++p) {
            const int c = grp + (round + p) * a.groups, at_c = ALL || c < a.c ? c : 0;
            if (MODE != PRE_BWD) wgt[p] = a.gamma[at_c] * (kPost && a.scale ? a.scale[at_c] : 1.f);
            if (kNext) nxt[p] = gn[at_c];
        }
    };
    if (PC) gains(0);

    // more: not this workgroup's first tile
    auto tile = [&](bool more, int64_t vol, int64_t first) {
        constexpr bool kAll = ALL;
        const bool ragged = !ALL && first + TILE > a.V;
        const int64_t t0 = first + at * TOK;
        int left = TOK, over = 0;
        uint32_t live = (1u << TOK) - 1u;
        Words<T, TOK> keep;  // all bits of live tokens
        if (!kAll) {
            if (ragged) {
                left = (int)(a.V - t0 < TOK ? (a.V - t0 > 0 ? a.V - t0 : 0) : TOK);
                over = TOK - left;
                live = (1u << left) - 1u;
            }
            if (a.mask) {
                uint8_t m[TOK];
#pragma unroll
                for (int j = 0; j < TOK; ++j)  // read without a branch
                    m[j] = a.mask[vol * a.V + (t0 + j < a.V ? t0 + j : a.V - 1)];
#pragma unroll
                for (int j = 0; j < TOK; ++j)
                    if (!m[j]) live &= ~(1u << j);
            }
            keep = V::bits(live);
        }
        // Bytes from a volume's channel ch[p] - grp, which is the same for a workgroup, to
        // the thread's tokens; counted back from the row's end where they do not fill it.
        const uint32_t es = sizeof(T);
        const uint32_t off = (uint32_t)((int64_t)grp * a.V + t0) * es;
        V X[NP], Z[NP], G[NP], Y[NP], DU[NP];  // backward: X is dy (before a block dres)
        int ch[NP];
        // Masked tokens, and channels that are none, come as 0 but for X.
        auto load = [&](int k) {
#pragma unroll
            for (int p = 0; p < NP; ++p) ch[p] = grp + (k + p) * a.groups;
            auto get = [&](V(&to)[NP], const void* q, int64_t stride, bool masked) {
                const T* from = (const T*)q + vol * stride;
#pragma unroll
                for (int p = 0; p < NP; ++p) {
                    const int64_t first_ch = (int64_t)(k + p) * a.groups;
                    if (kAll) {
                        to[p].load(from + first_ch * a.V, off);
                    } else {
                        const int64_t base = first_ch < a.c ? first_ch : a.c - 1;
                        const int64_t row = grp < a.c - base ? grp : a.c - base - 1;
                        const int64_t at0 = left == TOK ? t0 : a.V - TOK;
                        to[p].load(from + base * a.V, (uint32_t)(row * a.V + at0) * es);
                        if (ragged) to[p].shift(over);
                        if (masked)
#pragma unroll
                            for (int i = 0; i < V::N; ++i)
                                to[p].u.w[i] &= ch[p] < a.c ? keep.w[i] : 0;
                    }
                }
            };
            if (kBwd && kNext) {
                get(Y, a.y, a.sy, true);
                get(DU, a.du, a.su, true);
            }
            if (kPost) get(Z, a.z, a.sz, true);
            if (GATED) get(G, a.g, a.sg, true);
            if (!kBwd) get(X, a.x, a.sx, !kPost);
            else if (MODE == POST_BWD) get(X, a.dy, a.sy, false);
            else if (a.dy) get(X, a.dy, a.sx, false);
            else
#pragma unroll
                for (int p = 0; p < NP; ++p) X[p].u = {};
        };
        int round = 0;
        // Results, at masked voxels 0 or (put_past) X as it lies: chosen by bits, for a gain
        // that is not finite leaves no 0 of what is formed there.
        auto put_bits = [&](void* q, int64_t stride, int p, const float (&o)[TOK], auto edit) {
            if (kAll || ch[p] < a.c)
                put_edited<T, TOK, kAll>(
                    (T*)q + vol * stride + (int64_t)(round + p) * a.groups * a.V, off, left, o,
                    a.stream, edit);
        };
        // keep, in kernels without a gate formed again: two registers more are one workgroup a
        // CU fewer for some of them (16 x 128 channels of 2016 voxels 22.1 -> 25.4 us)
        auto stay = [&] {
            constexpr bool AGAIN = PC && TOK > 1 && !GATED;
            uint32_t on = live;
            if (AGAIN) asm volatile("" : "+v"(on));
            return AGAIN ? V::bits(on) : keep;
        };
        auto put = [&](void* q, int64_t stride, int p, const float (&o)[TOK]) {
            put_bits(q, stride, p, o, [&](Words<T, TOK>& u) {
                if (kAll) return;
                const Words<T, TOK> m = stay();
#pragma unroll
                for (int i = 0; i < V::N; ++i) u.w[i] &= m.w[i];
            });
        };
        auto put_past = [&](void* q, int64_t stride, int p, const float (&o)[TOK]) {
            put_bits(q, stride, p, o, [&](Words<T, TOK>& u) {
                if (kAll) return;
                const Words<T, TOK> m = stay();
#pragma unroll
                for (int i = 0; i < V::N; ++i)
                    u.w[i] = (u.w[i] & m.w[i]) | (X[p].u.w[i] & ~m.w[i]);
            });
        };
        // What is formed from a held value is formed again behind a barrier, not held too.
        auto forget = [&](V(&v)[NP]) {
            if (PC)
#pragma unroll
                for (int p = 0; p < NP; ++p)
#pragma unroll
                    for (auto& w : v[p].u.w) asm volatile("" : "+v"(w));
        };
        // formed here, not where it is used
        auto pin = [&](float(&v)[TOK]) {
            if (PC)
#pragma unroll
                for (float& x : v) asm volatile("" : "+v"(x));
        };
        // All of the thread's channels, one after another: the order keeps a channel's
        // registers free for the next.
        auto each = [&](auto f) {
            for (round = 0; round < rounds; ++round) {
                if (!PC) {
                    load(round);
                    gains(round);
                }
#pragma unroll
                for (int p = 0; p < NP; ++p) {
                    f(p);
                    __builtin_amdgcn_sched_barrier(0);
                }
                if (PC) break;
            }
            round = 0;
        };
        auto is_live = [&](int p, int j) { return kAll || (ch[p] < a.c && (live >> j & 1u)); };
        // the gate's value and slope
        auto gate = [&](int p, int j, float& phi, float& slope) {
            phi = 1.f;
            slope = 0.f;
            if (GATED) {
                const float g = G[p][j];
                const Sig sg(g);
                phi = a.gate == RAT3D_GATE_SILU ? g * sg.s : sg.s;
                slope = sg.s * (a.gate == RAT3D_GATE_SILU ? 1.f + g * sg.rest : sg.rest);
            }
        };
        auto root = [&](float (&r)[TOK], const float (&sum)[TOK]) {
#pragma unroll
            for (int j = 0; j < TOK; ++j)
                r[j] = __builtin_amdgcn_rsqf(__builtin_fmaf(sum[j], inv_c, a.eps));
        };
        // mean(e x) r^2 of the sum e x; at a root of 0 the sum may be no number any more
        auto mean = [&](float sum, float r) { return (r == 0.f ? 0.f : sum) * inv_c * (r * r); };
        auto clear = [&](auto& v) {
            for (auto& row : v)
                for (float& x : row) x = 0.f;
        };
        if (PC) load(0);
        float e[1][TOK];
        clear(e);

        if constexpr (MODE == PRE_FWD) {
            each([&](int p) {
#pragma unroll
                for (int j = 0; j < TOK; ++j) e[0][j] += X[p][j] * X[p][j];
            });
            channel_sums(e, lds[0], waves);
            forget(X);
            float r[TOK];
            root(r, e[0]);
            each([&](int p) {
                const float k = wgt[p];
                float u[TOK];
#pragma unroll
                for (int j = 0; j < TOK; ++j) u[j] = k * (X[p][j] * r[j]);
                put(a.ou, a.su, p, u);
            });
        }
        if constexpr (MODE == POST_FWD) {
            // held in the place of z and g: the branch without its root, then y.  A z whose
            // square is infinite has a root of 0, and its product with gains and gate may be
            // infinite: it counts as 0 (an infinite z as NaN).
            float b[NP][TOK], r[TOK];
            auto branch = [&](int p) {
                const float k = wgt[p];
#pragma unroll
                for (int j = 0; j < TOK; ++j) {
                    float phi, slope;
                    gate(p, j, phi, slope);
                    const float z = Z[p][j];
                    b[p][j] = z * z < __builtin_inff() ? k * phi * z : 0.f * z;
                }
            };
            auto sum = [&](int p) {
#pragma unroll
                for (int j = 0; j < TOK; ++j) b[p][j] = __builtin_fmaf(b[p][j], r[j], X[p][j]);
            };
            each([&](int p) {
#pragma unroll
                for (int j = 0; j < TOK; ++j) e[0][j] += Z[p][j] * Z[p][j];
                if (PC) {
                    branch(p);
                    pin(b[p]);
                    pin(e[0]);
                }
            });
            channel_sums(e, lds[0], waves);
            forget(X);
            root(r, e[0]);
            float ry[TOK];
            if constexpr (NEXT) {
                clear(e);
                each([&](int p) {
                    if (!PC) branch(p);
                    sum(p);
                    if (PC) put_past(a.oy, a.sy, p, b[p]);
                    const bool is = kAll || ch[p] < a.c;
#pragma unroll
                    for (int j = 0; j < TOK; ++j) e[0][j] += is ? b[p][j] * b[p][j] : 0.f;
                    pin(b[p]);
                    pin(e[0]);
                });
                channel_sums(e, lds[1], waves);
                root(ry, e[0]);
            }
            each([&](int p) {
                if (!PC) branch(p);
                if (!PC || !NEXT) {
                    sum(p);
                    put_past(a.oy, a.sy, p, b[p]);
                }
                if constexpr (NEXT) {
                    const float k = nxt[p];
#pragma unroll
                    for (int j = 0; j < TOK; ++j) b[p][j] = k * (b[p][j] * ry[j]);
                    put(a.ou, a.su, p, b[p]);
                }
            });
        }
        if constexpr (kBwd) {
            float s[K][TOK];
            clear(s);
            each([&](int p) {
                const float k = kNext ? nxt[p] : 0.f;
#pragma unroll
                for (int j = 0; j < TOK; ++j) {
                    if constexpr (kPost) s[0][j] += Z[p][j] * Z[p][j];
                    if constexpr (kNext) {
                        const float y = Y[p][j];
                        s[K - 2][j] += y * y;
                        s[K - 1][j] += k * DU[p][j] * y;
                    }
                }
#pragma unroll
                for (int k = 0; k < K; ++k) pin(s[k]);
            });
            channel_sums(s, lds[0], waves);
            forget(X);
            if (kNext) {
                forget(Y);
                forget(DU);
            }
            if (kPost) forget(Z);
            if (GATED) forget(G);
            float ry[TOK], my[TOK], rz[TOK];
            if constexpr (kNext) {
                root(ry, s[K - 2]);
#pragma unroll
                for (int j = 0; j < TOK; ++j) my[j] = mean(s[K - 1][j], ry[j]);
            }
            if constexpr (kPost) root(rz, s[0]);
            // dY, and its part in the next norm's gain
            auto residual = [&](int p, float (&d)[TOK]) {
                const float k = kNext ? nxt[p] : 0.f;
                float n = 0.f;
#pragma unroll
                for (int j = 0; j < TOK; ++j) {
                    d[j] = X[p][j];
                    if constexpr (kNext) {
                        const float y = Y[p][j], du = DU[p][j];
                        d[j] += ry[j] * (k * du - y * my[j]);
                        n += du * (y * ry[j]);
                    }
                }
                return n;
            };
            auto add_n = [&](int p, float n) {
                asm volatile("" : "+v"(n));
                if constexpr (PC != 0) sum_n[p] += (double)n;
                else if (kNext) put_gain(0, ch[p], (double)n, more);
            };
            auto add_t = [&](int p, float q) {
                asm volatile("" : "+v"(q));
                if constexpr (PC != 0) sum_t[p] += (double)q;
                else put_gain(1, ch[p], (double)q, more);
            };
            if constexpr (!kPost) {
                each([&](int p) {
                    float d[TOK];
                    add_n(p, residual(p, d));
                    put_past(a.dx, a.sx, p, d);
                });
            } else {
                // e = dY s gamma phi, held in the place of what it is formed from; where
                // nothing is held, results wait for the last pass, which reads all again
                float E[NP][TOK], mz[TOK];
                constexpr bool kMaskDz = GATED || NEXT;  // or e is 0 at masked voxels
                auto middle = [&](int p, bool out) {
                    const float w = wgt[p];
                    const float n = residual(p, E[p]);
                    if (out) {
                        add_n(p, n);
                        if (kNext) put_past(a.dx, a.sx, p, E[p]);
                    }
                    float dg[TOK], q = 0.f;
#pragma unroll
                    for (int j = 0; j < TOK; ++j) {
                        float phi, slope;
                        gate(p, j, phi, slope);
                        const float d = is_live(p, j) ? E[p][j] : 0.f, zr = Z[p][j] * rz[j];
                        q += d * phi * zr;
                        dg[j] = d * w * zr * slope;
                        E[p][j] = kMaskDz || is_live(p, j) ? d * w * phi : 0.f;
                    }
                    if (out) {
                        add_t(p, q);
                        if (GATED) put(a.dg, a.sg, p, dg);
                    }
                };
                each([&](int p) {
                    middle(p, PC != 0);
#pragma unroll
                    for (int j = 0; j < TOK; ++j) e[0][j] += E[p][j] * Z[p][j];
                    pin(E[p]);
                    pin(e[0]);
                });
                channel_sums(e, lds[1], waves);
                forget(Z);
#pragma unroll
                for (int j = 0; j < TOK; ++j) mz[j] = mean(e[0][j], rz[j]);
                each([&](int p) {
                    if (!PC) middle(p, true);
#pragma unroll
                    for (int j = 0; j < TOK; ++j) E[p][j] = rz[j] * (E[p][j] - Z[p][j] * mz[j]);
                    if (kMaskDz) put(a.dz, a.sz, p, E[p]);
                    else put_bits(a.dz, a.sz, p, E[p], [](Words<T, TOK>&) {});
                });
            }
        }
        // the first sums are written again only behind the barrier of the second, the
        // second only behind that of the next first
        if constexpr (MODE == PRE_BWD) __syncthreads();
    };

    // backward: several tiles a workgroup, so that the gains' parts stay few
    const uint32_t t0 = a.base + (a.near ? xcd_remap(blockIdx.x, gridDim.x) : blockIdx.x);
    uint32_t t = t0;
    do {
        const uint32_t vol = t / a.tiles;
        tile(t != t0, vol, (int64_t)(t - vol * a.tiles) * TILE);
        t += gridDim.x;
    } while (kBwd && t < a.all);
    if constexpr (kBwd && PC != 0) {
#pragma unroll
        for (int p = 0; p < NP; ++p) {
            if (kNext) put_gain(0, grp + p * a.groups, sum_n[p], false);
            if (kPost) put_gain(1, grp + p * a.groups, sum_t[p], false);
        }
    }
}

// The gains' gradients: the parts of the workgroups added in float64, in a fixed order, of
// the gains from `gain` on that the call has written.
template <typename Part>
__global__ __launch_bounds__(256) void norm_gain_k(const Part* __restrict__ part, int parts, int c,
                                                   const float* gamma, const float* scale,
                                                   float* dnext, float* dgamma, float* dscale,
                                                   int gain, int accumulate) {
    __shared__ double red[4];
    const int ch = blockIdx.x, which = gain + blockIdx.y;  // 0: the norm du reads, 1: the branch's
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
// Tokens and channels a thread, and groups of threads along the channels (whole waves).
// Fewer tokens than 16 bytes hold,
//   half, where there are few tiles, so that one loads while another sums or stores: in
//   bfloat16 below two a CU (16 x 128 channels of 12x14x12 voxels 15.3 -> 12.5 us behind a
//   block, its gradient 34.9 -> 31.1, before a block 7.5 -> 6.5 and 16.4 -> 13.7; at 8 x 64
//   of 24x28x24, four tiles a CU, 18.4 -> 19.5 and 35.5 -> 36.9), in float32 up to one for
//   two CUs (16 x 256 channels of 252 voxels 13.1 -> 9.0 and 35.5 -> 19.0, before a block
//   15.5 -> 12.1; at 2 x 256 of 16128, two tiles a CU, 36.7 -> 39.8 behind a block);
//   half, with twice the channels, in the forward of more than 256 channels: 4 x 512
//   channels over 16128 voxels in float32 215 -> 150 us behind a block, 55 -> 41 before one
//   (bfloat16, also of up to 512 channels 215 -> 160 and 56 -> 52 over 2 x 64512 voxels);
//   half in the backward of more than 128 channels, where the registers of the full number
//   spill: in bfloat16 with twice the channels (4 x 256 channels over 64512 voxels 546 ->
//   280 us behind a block, 146 -> 136 before one), in float32 for the gradient behind a
//   block with a next norm and a mask, unwhole tiles or channels (4 x 256 channels over
//   16127 voxels 193 -> 154 us; over 16128 without a mask it does not gain, and neither do
//   the other gradients: 76 -> 85 without a next norm);
//   a quarter in the backward of 257 to 512 channels, where rows are no whole tiles (4 x 512
//   channels over 16127 voxels in float32 567 -> 399 us behind a block, 253 -> 149 before
//   one) or tiles are few (one of 400 channels and 27 voxels 92 -> 20 us), and in bfloat16
//   of 129 to 256 channels where tiles are few (one of 256 channels 24 -> 16 us).  Large
//   maps of whole tiles are read again instead: 4 x 512 over 16128 in float32 349 us
//   against 362, bfloat16 183 against 193, before a block 151 against 184 and 85 against 97.
// Channels that are read again have 64 groups, few rounds: 4 x 600 channels over 16128
// voxels in bfloat16 244 -> 235 us, before a block 135 -> 96, behind one 162 -> 116,
// against 16 groups.
// Kernels of 1024 threads have 128 registers, and some gradients behind a block with a next
// norm spill over them: two voxels of eight channels in bfloat16 65 registers where tiles are
// masked or unwhole (53 without a gate), 11 (9) on whole ones, four of four in float32 on
// whole tiles 18 (2), one of eight in float32 11, read again in bfloat16 13.
struct NormShape {
    int tok, pc, groups;
};
static NormShape norm_shape(const rat3d_norm_desc& d, NormMode mode, bool masked, bool next) {
    const int es = d.dtype == RAT3D_BF16 ? 2 : 4, tok = d.v < 16 / es ? 1 : 16 / es;
    const bool bwd = mode == PRE_BWD || mode == POST_BWD;
    const int64_t tiles = ceil_div(d.v, kLanes * tok) * d.n;
    const int64_t cus = device_cus();
    const bool few = tok == 8 ? tiles < 2 * cus : 2 * tiles <= cus, least = 4 * tiles < cus;
    // a group's rows are reached with 32 bits: at least 4 of them up to 2^28 tokens
    const int64_t most = ((int64_t)1 << 32) / (d.v * es);
    NormShape s = {tok, 4, 0};
    if (tok == 1) {
        if (d.c > 256) s.pc = 0;
    } else if (d.c > 512) {
        s.pc = 0;
    } else if (d.c > 256) {
        if (!bwd) s = {tok / 2, 8, 0};
        else if (least || d.v % 64) s = {tok / 4, 8, 0};
        else s.pc = 0;
    } else if (d.c <= 128 || !bwd) {
        if (few) s.tok = tok / 2;
    } else if (tok == 8) {
        s = least ? NormShape{2, 4, 0} : NormShape{4, 8, 0};
    } else if (few || (mode == POST_BWD && next && (masked || d.v % 64 || d.c % 16))) {
        s.tok = 2;
    }
    if (s.pc) s.groups = (int)ceil_div(d.c, 4 * s.pc) * 4;
    if (!s.pc || s.groups > most) s = {tok, 0, 64};
    while (s.groups > most) s.groups /= 2;
    return s;
}

static NormShape norm_plan(const rat3d_norm_desc& d, NormMode mode, bool masked, bool next,
                           NormArgs* a) {
    const int64_t packed = (int64_t)d.c * d.v;
    const NormShape shape = norm_shape(d, mode, masked, next);
    a->sx = d.x_stride ? d.x_stride : packed;
    a->sz = d.z_stride ? d.z_stride : packed;
    a->sg = d.g_stride ? d.g_stride : packed;
    a->sy = d.y_stride ? d.y_stride : packed;
    a->su = d.u_stride ? d.u_stride : packed;
    a->V = d.v;
    a->c = d.c;
    a->eps = d.eps;
    a->gate = d.gate;
    // Results larger than the memory-side cache (256 MB) do not wait there for their
    // reader; stored past it they leave it to the inputs (16 x 64 channels over 48x56x48:
    // 261 -> 255 us behind a block, its gradient 447 -> 434).
    a->stream = (double)d.n * d.c * d.v * (d.dtype == RAT3D_BF16 ? 2 : 4) > 256e6;
    a->groups = shape.groups;
    a->tiles = (uint32_t)ceil_div(d.v, kLanes * shape.tok);
    a->all = a->tiles * d.n;
    return shape;
}

// Backward: a few tiles a workgroup, so that the gains' parts stay few: two workgroups a CU,
// more of fewer than 256 threads (gradient before a block over 16 x 64 channels of
// 48x56x48 203 us with two, 217 with four; behind one over 16 x 32 251 and 225).
static uint32_t norm_grid(const NormArgs& a, NormMode mode) {
    if (mode == PRE_FWD || mode == POST_FWD) return a.all;
    const int threads = a.groups * kLanes;
    const uint32_t most = (threads < 256 ? 512 / threads : 2) * device_cus();
    return a.all > most ? most : a.all;
}

// The parts of the shape with the shortest tiles, and the most workgroups: of 64 channels
// on, and where 32 bits reach 16 groups, they have 256 threads or more.
size_t norm_ws_bytes(const rat3d_norm_desc& d) {
    const int full = d.dtype == RAT3D_BF16 ? 8 : 4, tok = d.v < full ? 1 : full / 4;
    const int64_t tiles = ceil_div(d.v, kLanes * tok) * d.n;
    const int64_t most = (d.c < 64 || d.v > 1 << 24 ? 8 : 2) * (int64_t)device_cus();
    return (size_t)(tiles < most ? tiles : most) * 2 * d.c * sizeof(double);
}

// Rows that begin inside a cache line: neighbouring tiles share lines, and one XCD's
// L2 should see both (16 x 64 channels of 129023 voxels: 407 -> 341 us behind a block,
// its gradient 692 -> 509; whole lines are 2 to 4 % faster dealt out).  Streaming stores
// would write the shared lines twice.
static void norm_lines(const rat3d_norm_desc& d, NormArgs* a) {
    const int64_t es = d.dtype == RAT3D_BF16 ? 2 : 4;
    uintptr_t any = (uintptr_t)(d.v * es);
    for (int64_t s : {a->sx, a->sz, a->sg, a->sy, a->su}) any |= (uintptr_t)(s * es);
    for (const void* p : {a->x, a->z, a->g, a->y, a->dy, a->du, (const void*)a->oy,
                          (const void*)a->ou, (const void*)a->dx, (const void*)a->dz,
                          (const void*)a->dg})
        any |= (uintptr_t)p;
    a->near = any % 128 != 0;
    if (a->near) a->stream = 0;
}

// False where no kernel is built for the shape: each is launched only where what it assumes
// holds.  dry: nothing is launched.
template <typename T, NormMode MODE, bool GATED, bool NEXT>
static bool norm_launch_t(const rat3d_norm_desc& d, const NormShape& shape, NormArgs a,
                          hipStream_t st, bool dry) {
    constexpr bool kBwd = MODE == PRE_BWD || MODE == POST_BWD;
    constexpr int TOK = 16 / (int)sizeof(T);
    const int threads = a.groups * kLanes;
    const bool all = !a.mask && d.v % (kLanes * shape.tok) == 0 &&
                     d.c % (a.groups * (shape.pc ? shape.pc : 1)) == 0;
#define RAT3D_NORM1(TOK, PC, ALL, THREADS)                                                     \
    do {                                                                                       \
        if ((ALL && !all) || threads > THREADS || (TOK) != shape.tok || (PC) != shape.pc ||    \
            ((PC) && (PC) * a.groups < d.c))                                                   \
            return false;                                                                      \
        if (!dry)                                                                              \
            block_norm_k<T, TOK, PC, MODE, GATED, NEXT, ALL, THREADS>                          \
                <<<grid, threads, 0, st>>>(a);                                                 \
    } while (0)
#define RAT3D_NORM(TOK, PC, THREADS)                  \
    do {                                              \
        if (all) RAT3D_NORM1(TOK, PC, true, THREADS); \
        else RAT3D_NORM1(TOK, PC, false, THREADS);    \
    } while (0)
    // a launch holds fewer than 2^32 threads; a workgroup at most as many as its kernel is
    // built for
    const uint32_t most = ((uint32_t)1 << 31) / (uint32_t)threads;
    for (uint32_t left = norm_grid(a, MODE); left; left -= left < most ? left : most) {
        const unsigned grid = left < most ? left : most;
        if (d.v < TOK) {
            if (shape.pc) RAT3D_NORM1(1, 4, false, 1024);
            else RAT3D_NORM1(1, 0, false, 1024);
        } else if (shape.pc == 0) {
            RAT3D_NORM(TOK, 0, 1024);
        } else if constexpr (!kBwd) {  // 128 registers are enough
            if (shape.tok == TOK) RAT3D_NORM(TOK, 4, 1024);
            else if (shape.pc == 4) RAT3D_NORM(TOK / 2, 4, 1024);
            else RAT3D_NORM(TOK / 2, 8, 1024);
        } else if (shape.tok == TOK) {
            if (threads <= 256) RAT3D_NORM(TOK, 4, 256);
            else if (TOK == 8 || threads <= 512) RAT3D_NORM(TOK, 4, 512);
            else if constexpr (TOK == 4 && MODE == POST_BWD && NEXT)
                RAT3D_NORM1(TOK, 4, true, 1024);  // norm_shape gives the others half the tokens
            else if constexpr (TOK == 4) RAT3D_NORM(TOK, 4, 1024);
        } else if (shape.tok == TOK / 2 && shape.pc == 4) {
            if (threads <= 256) RAT3D_NORM(TOK / 2, 4, 256);
            else if (TOK == 8 || threads <= 512) RAT3D_NORM(TOK / 2, 4, 512);
            else if constexpr (TOK == 4) RAT3D_NORM(TOK / 2, 4, 1024);
        } else if (shape.pc == 8) {
            if (shape.tok == TOK / 4) RAT3D_NORM(TOK / 4, 8, 1024);
            else if constexpr (TOK == 8) RAT3D_NORM(TOK / 2, 8, 512);
        } else if constexpr (TOK == 8) {
            RAT3D_NORM(TOK / 4, 4, 1024);
        } else {
            return false;
        }
        a.base += grid;
    }
    return true;
#undef RAT3D_NORM
#undef RAT3D_NORM1
}

template <NormMode MODE, bool GATED, bool NEXT>
static bool norm_launch_g(const rat3d_norm_desc& d, const NormShape& shape, const NormArgs& a,
                          hipStream_t st, bool dry) {
    return d.dtype == RAT3D_BF16 ? norm_launch_t<bf16, MODE, GATED, NEXT>(d, shape, a, st, dry)
                                 : norm_launch_t<float, MODE, GATED, NEXT>(d, shape, a, st, dry);
}
template <NormMode MODE>
static bool norm_launch(const rat3d_norm_desc& d, const NormShape& shape, NormArgs& a,
                        hipStream_t st, bool dry = false) {
    norm_lines(d, &a);
    if constexpr (MODE == PRE_FWD || MODE == PRE_BWD) {
        return norm_launch_g<MODE, false, MODE == PRE_BWD>(d, shape, a, st, dry);
    } else {
        if (d.gate && a.next) return norm_launch_g<MODE, true, true>(d, shape, a, st, dry);
        if (d.gate) return norm_launch_g<MODE, true, false>(d, shape, a, st, dry);
        if (a.next) return norm_launch_g<MODE, false, true>(d, shape, a, st, dry);
        return norm_launch_g<MODE, false, false>(d, shape, a, st, dry);
    }
}
static rat3d_status norm_none() {
    set_error("no kernel is built for this norm");
    return RAT3D_EUNSUPPORTED;
}

// Names of the measurement: channels held in registers (of 16, 8 or 4 bytes of tokens),
// read again for every sum, or single tokens.
static const char* norm_tag(const rat3d_norm_desc& d, const NormShape& s,
                            const char* const (&names)[5]) {
    const int full = d.dtype == RAT3D_BF16 ? 8 : 4;
    return names[d.v < full ? 4 : s.pc == 0 ? 3 : s.tok == full ? 0 : 2 * s.tok == full ? 1 : 2];
}
#define RAT3D_NORM_TAG(name) \
    norm_tag(d, shape, {name, name "_half", name "_quarter", name "_any", name "_one"})

static double norm_bytes(const rat3d_norm_desc& d, int tensors) {
    return (double)d.n * d.c * d.v * tensors * (d.dtype == RAT3D_BF16 ? 2 : 4);
}

rat3d_status pre_norm_fwd(const rat3d_norm_desc& d, const void* x, const float* gamma,
                          const uint8_t* mask, void* u, hipStream_t st) {
    NormArgs a = {};
    const NormShape shape = norm_plan(d, PRE_FWD, mask != nullptr, false, &a);
    a.x = x;
    a.gamma = gamma;
    a.mask = mask;
    a.ou = u;
    ProfScope ps(RAT3D_NORM_TAG("pre_norm_fwd"), st, 0.0, norm_bytes(d, 2));
    if (!norm_launch<PRE_FWD>(d, shape, a, st)) return norm_none();
    RAT3D_LAUNCH_CHECK();
    return RAT3D_OK;
}

rat3d_status post_norm_fwd(const rat3d_norm_desc& d, const void* x, const void* z, const void* g,
                           const float* gamma, const float* scale, const float* next,
                           const uint8_t* mask, void* y, void* u, hipStream_t st) {
    NormArgs a = {};
    const NormShape shape = norm_plan(d, POST_FWD, mask != nullptr, next != nullptr, &a);
    a.x = x;
    a.z = z;
    a.g = g;
    a.gamma = gamma;
    a.scale = scale;
    a.next = next;
    a.mask = mask;
    a.oy = y;
    a.ou = u;
    ProfScope ps(RAT3D_NORM_TAG("post_norm_fwd"), st, 0.0,
                 norm_bytes(d, 3 + (d.gate != 0) + (next != nullptr)));
    if (!norm_launch<POST_FWD>(d, shape, a, st)) return norm_none();
    RAT3D_LAUNCH_CHECK();
    return RAT3D_OK;
}

static rat3d_status norm_gains(const NormArgs& a, const NormShape& shape, NormMode mode,
                               float* dnext, float* dgamma, float* dscale, int accumulate,
                               hipStream_t st) {
    const int parts = (int)norm_grid(a, mode);
    const int gain = dnext ? 0 : 1, gains = (dgamma ? 2 : 1) - gain;
    ProfScope ps("norm_gain", st, 0.0, (shape.pc ? 4.0 : 8.0) * a.c * parts * gains);
    auto sum = [&](auto* part) {
        norm_gain_k<<<dim3(a.c, gains), 256, 0, st>>>(part, parts, a.c, a.gamma, a.scale, dnext,
                                                      dgamma, dscale, gain, accumulate);
    };
    if (shape.pc) sum((const NormPart<1>*)a.part);
    else sum((const NormPart<0>*)a.part);
    RAT3D_LAUNCH_CHECK();
    return RAT3D_OK;
}

rat3d_status pre_norm_bwd(const rat3d_norm_desc& d, const void* du, const void* x,
                          const float* gamma, const uint8_t* mask, const void* dres, void* dx,
                          float* dgamma, int accumulate, void* ws, hipStream_t st) {
    NormArgs a = {};
    const NormShape shape = norm_plan(d, PRE_BWD, mask != nullptr, true, &a);
    a.du = du;
    a.y = x;
    a.sy = a.sx;
    a.dy = dres;
    a.gamma = gamma;
    a.mask = mask;
    a.dx = dx;
    a.part = ws;
    {
        ProfScope ps(RAT3D_NORM_TAG("pre_norm_bwd"), st, 0.0,
                     norm_bytes(d, 3 + (dres != nullptr)));
        if (!norm_launch<PRE_BWD>(d, shape, a, st)) return norm_none();
        RAT3D_LAUNCH_CHECK();
    }
    return norm_gains(a, shape, PRE_BWD, dgamma, nullptr, nullptr, accumulate, st);
}

rat3d_status post_norm_bwd(const rat3d_norm_desc& d, const void* dy, const void* du, const void* y,
                           const void* z, const void* g, const float* gamma, const float* scale,
                           const float* next, const uint8_t* mask, void* dx, void* dz, void* dg,
                           float* dgamma, float* dscale, float* dnext, int accumulate, void* ws,
                           hipStream_t st) {
    NormArgs a = {};
    const NormShape shape = norm_plan(d, POST_BWD, mask != nullptr, next != nullptr, &a);
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
    a.part = ws;
    {
        ProfScope ps(RAT3D_NORM_TAG("post_norm_bwd"), st, 0.0,
                     norm_bytes(d, 3 + 2 * (d.gate != 0) + (next ? 3 : 0)));
        if (!norm_launch<POST_BWD>(d, shape, a, st)) return norm_none();
        RAT3D_LAUNCH_CHECK();
    }
    return norm_gains(a, shape, POST_BWD, dnext, dgamma, dscale, accumulate, st);
}

}  // namespace rat3d

// What a call is planned as, for the tests that keep every size on a kernel that is built for
// it.  pass: 0 and 1 forward and gradient before a block, 2 and 3 behind one.  Returns 0 where
// no kernel takes it, else 1 and out = {tokens a thread, channels a thread or 0, groups, tiles,
// workgroups}.
extern "C" int rat3d_norm_plan(const rat3d_norm_desc* desc, int pass, int masked, int next,
                               int64_t out[5]) {
    using namespace rat3d;
    if (!out || pass < 0 || pass > 3 || rat3d_norm_workspace_size(desc) == (size_t)-1) return 0;
    const NormMode modes[4] = {PRE_FWD, PRE_BWD, POST_FWD, POST_BWD};
    const NormMode mode = modes[pass];
    static const uint8_t mask = 1;
    static const float gain = 1.f;
    NormArgs a = {};
    const NormShape shape = norm_plan(*desc, mode, masked != 0, pass == 1 || next, &a);
    a.mask = masked ? &mask : nullptr;
    a.next = next ? &gain : nullptr;
    const bool built = mode == PRE_FWD   ? norm_launch<PRE_FWD>(*desc, shape, a, nullptr, true)
                       : mode == PRE_BWD ? norm_launch<PRE_BWD>(*desc, shape, a, nullptr, true)
                       : mode == POST_FWD
                           ? norm_launch<POST_FWD>(*desc, shape, a, nullptr, true)
                           : norm_launch<POST_BWD>(*desc, shape, a, nullptr, true);
    const int64_t o[5] = {shape.tok, shape.pc, shape.groups, a.all, norm_grid(a, mode)};
    for (int i = 0; i < 5; ++i) out[i] = o[i];
    return built;
}
