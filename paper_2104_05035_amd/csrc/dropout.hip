// Dropout whose mask is formed from a counter, in the forward and again in the
// backward, and never stored.
//
// Decision u takes the 16-bit number u % 8 of the Philox4x32-10 block (Salmon et
// al. 2011, "Parallel random numbers: as easy as 1, 2, 3") with counter
// (u / 8, step) and the seed as its key.  One block gives the eight decisions of
// one 16-byte unit of bfloat16 (of two of float32), so its ten rounds, twenty
// 32 x 32 -> 64 bit products, are paid once for eight elements: 2.5 quarter-rate
// instructions an element, fewer than the memory lets through.  Sixteen bits are
// the resolution of p; the scale is that of the rounded p, so the mean is kept.
//
// Bound: HBM, x (and the residual) read once and the result written once.
#include "kernels.hpp"
#include "prof.hpp"
#include "vec.hpp"

namespace rat3d {

struct Philox {
    uint32_t w[4];
    __device__ __forceinline__ Philox(uint64_t block, uint64_t step, uint64_t seed) {
        uint32_t c0 = (uint32_t)block, c1 = (uint32_t)(block >> 32);
        uint32_t c2 = (uint32_t)step, c3 = (uint32_t)(step >> 32);
        uint32_t k0 = (uint32_t)seed, k1 = (uint32_t)(seed >> 32);
#pragma unroll
        for (int r = 0; r < 10; ++r) {
            const uint64_t a = (uint64_t)0xD2511F53u * c0, b = (uint64_t)0xCD9E8D57u * c2;
            c0 = (uint32_t)(b >> 32) ^ c1 ^ k0;
            c1 = (uint32_t)b;
            c2 = (uint32_t)(a >> 32) ^ c3 ^ k1;
            c3 = (uint32_t)a;
            k0 += 0x9E3779B9u;
            k1 += 0xBB67AE85u;
        }
        w[0] = c0; w[1] = c1; w[2] = c2; w[3] = c3;
    }
    // the i-th of the eight 16-bit numbers (i may vary by lane)
    __device__ __forceinline__ uint32_t lot(int i) const {
        const uint32_t a = (i & 2) ? w[1] : w[0], b = (i & 2) ? w[3] : w[2];
        const uint32_t v = (i & 4) ? b : a;
        return (i & 1) ? v >> 16 : v & 0xffffu;
    }
};

// e / unit for 0 <= e < 2^53: the quotient by a reciprocal is off by at most one.
__device__ __forceinline__ int64_t unit_of(int64_t e, int64_t unit, double inv) {
    int64_t u = (int64_t)((double)e * inv);
    const int64_t r = e - u * unit;
    if (r < 0) --u;
    else if (r >= unit) ++u;
    return u;
}

// Eight elements per thread and turn.  ONE: every element has a decision of its
// own (one Philox block); otherwise all eight usually fall into one unit and share
// one, and where they do not each looks its own up.
template <typename T, bool ONE, bool RES>
__global__ __launch_bounds__(256) void dropout_k(int64_t count, int64_t unit, double inv,
                                                 uint32_t below, float scale, uint64_t seed,
                                                 uint64_t step,
                                                 const uint64_t* __restrict__ step_dev,
                                                 const T* x, const T* res, T* y) {
    constexpr int VEC = vec16<T>();
    if (step_dev) step += *step_dev;
    const int64_t turn = (int64_t)gridDim.x * 256;
    for (int64_t b = (int64_t)blockIdx.x * 256 + threadIdx.x; b * 8 < count; b += turn) {
        const int64_t e = b * 8;
        const bool whole = e + 8 <= count;
        float v[8 / VEC][VEC], r[8 / VEC][VEC];
#pragma unroll
        for (int i = 0; i < 8 / VEC; ++i) {
            if (whole) {
                vload<T, VEC>(x + e + i * VEC, v[i]);
                if (RES) vload<T, VEC>(res + e + i * VEC, r[i]);
            } else {
                vload_part<T, VEC>(x, e + i * VEC, count, v[i]);
                if (RES) vload_part<T, VEC>(res, e + i * VEC, count, r[i]);
            }
        }
        uint32_t keep = 0;  // bit j: element e + j stays
        if (ONE) {
            const Philox g((uint64_t)b, step, seed);
#pragma unroll
            for (int j = 0; j < 8; ++j) keep |= (g.lot(j) >= below ? 1u : 0u) << j;
        } else {
            int64_t u = unit_of(e, unit, inv);
            int64_t end = (u + 1) * unit - e;  // first element of the next unit, from e
            bool k = Philox((uint64_t)u / 8, step, seed).lot((int)(u & 7)) >= below;
            if (end >= 8) {
                keep = k ? 0xffu : 0u;
            } else {
                for (int j = 0; j < 8; ++j) {
                    if (j >= end) {
                        ++u;
                        end += unit;
                        k = Philox((uint64_t)u / 8, step, seed).lot((int)(u & 7)) >= below;
                    }
                    keep |= (k ? 1u : 0u) << j;
                }
            }
        }
#pragma unroll
        for (int i = 0; i < 8 / VEC; ++i) {
            float o[VEC];
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                // selected, not multiplied: a dropped NaN or infinity leaves nothing
                const float d = (keep >> (i * VEC + j)) & 1u ? v[i][j] * scale : 0.f;
                o[j] = RES ? r[i][j] + d : d;
            }
            if (whole) vstore<T, VEC>(y + e + i * VEC, o);
            else vstore_part<T, VEC>(y, e + i * VEC, count, o);
        }
    }
}

rat3d_status dropout(int64_t count, int64_t unit, double p, uint64_t seed, uint64_t step,
                     const uint64_t* step_dev, rat3d_dtype dt, const void* x, const void* res,
                     void* y, hipStream_t st) {
    const int64_t below = (int64_t)nearbyint(p * 65536.0);
    const float scale = below < 65536 ? (float)(65536.0 / (double)(65536 - below)) : 0.f;
    const int64_t blocks = ceil_div(count, 8 * 256);
    const unsigned grid = (unsigned)(blocks < (1 << 20) ? blocks : (1 << 20));
    const double inv = 1.0 / (double)unit;
    ProfScope ps("dropout", st, 0.0, (res ? 3.0 : 2.0) * (dt == RAT3D_BF16 ? 2.0 : 4.0) * count);
#define RAT3D_DROP(T, ONE, RES)                                                               \
    dropout_k<T, ONE, RES><<<grid, 256, 0, st>>>(count, unit, inv, (uint32_t)below, scale, seed, \
                                                 step, step_dev, (const T*)x, (const T*)res, (T*)y)
#define RAT3D_DROP_T(T)                                   \
    do {                                                  \
        if (unit == 1 && res) RAT3D_DROP(T, true, true);  \
        else if (unit == 1) RAT3D_DROP(T, true, false);   \
        else if (res) RAT3D_DROP(T, false, true);         \
        else RAT3D_DROP(T, false, false);                 \
    } while (0)
    if (dt == RAT3D_BF16) RAT3D_DROP_T(bf16);
    else RAT3D_DROP_T(float);
#undef RAT3D_DROP_T
#undef RAT3D_DROP
    RAT3D_LAUNCH_CHECK();
    return RAT3D_OK;
}

}  // namespace rat3d
