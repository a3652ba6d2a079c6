// A thread's neighbouring tokens of one channel's row, read and written in one access from
// any element on.
#pragma once

#include <type_traits>

#include "common.hpp"

namespace rat3d {

// A thread's tokens of one channel, as they lie.  A result may lie over an input that is
// read as other words or as elements: the compiler takes no two accesses for apart.
template <typename T, int TOK>
struct __attribute__((packed, aligned(sizeof(T)), may_alias)) Words {
    typename std::conditional<TOK * sizeof(T) < 4, uint16_t, uint32_t>::type
        w[TOK * sizeof(T) < 4 ? 1 : TOK * sizeof(T) / 4];
};
template <typename T, int TOK> struct Toks {
    static constexpr int N = sizeof(Words<T, TOK>) / sizeof(Words<T, TOK>::w[0]);
    Words<T, TOK> u;
    // all bits of the tokens whose bit is set
    __device__ __forceinline__ static Words<T, TOK> bits(uint32_t on) {
        Words<T, TOK> m;
        if constexpr (sizeof(T) == 4 || TOK == 1) {
#pragma unroll
            for (int j = 0; j < TOK; ++j) m.w[j] = 0u - (on >> j & 1u);
        } else {
#pragma unroll
            for (int j = 0; j < TOK; j += 2)
                m.w[j / 2] = (on >> j & 1u ? 0xffffu : 0u) | (on >> j & 2u ? 0xffff0000u : 0u);
        }
        return m;
    }
    __device__ __forceinline__ float operator[](int j) const {
        if constexpr (sizeof(T) == 4) return __uint_as_float(u.w[j]);
        else if constexpr (TOK == 1) return Elt<T>::from_bits(u.w[0]);
        else return __uint_as_float(j & 1 ? u.w[j / 2] & 0xffff0000u : u.w[j / 2] << 16);
    }
    // The tokens `off` bytes behind base, which is the same for a workgroup.
    __device__ __forceinline__ void load(const T* base, uint32_t off) {
        u = *reinterpret_cast<const Words<T, TOK>*>((const char*)base + off);
    }
    // The tokens from `over` (0 .. TOK) on.
    __device__ __forceinline__ void shift(int over) {
        if constexpr (TOK > 1) {
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
template <typename T, int TOK>
__device__ __forceinline__ void pack_tokens(Words<T, TOK>& u, const float (&o)[TOK]) {
#pragma unroll
    for (int j = 0; j < TOK; j += 4 / (int)sizeof(T)) {
        if constexpr (sizeof(T) == 4) u.w[j] = __float_as_uint(o[j]);
        else if constexpr (TOK == 1) u.w[0] = Elt<T>::to_bits(o[0]);
        else u.w[j / 2] = pack_bf16x2(o[j], o[j + 1]);
    }
}
// The first `left` tokens (ALL: each); `stream`: past the memory-side cache.
template <typename T, int TOK, bool ALL>
__device__ __forceinline__ void put_tokens(T* base, uint32_t off, int left,
                                           const float (&o)[TOK], bool stream) {
    T* p = (T*)((char*)base + off);
    if (ALL || left == TOK) {
        Words<T, TOK> u;
        pack_tokens<T, TOK>(u, o);
        if constexpr (TOK * sizeof(T) == 16) {
            if (stream) {
                typedef uint32_t __attribute__((ext_vector_type(4))) u4;
                typedef u4 __attribute__((aligned(2), may_alias)) u4_any;
                __builtin_nontemporal_store(u4{u.w[0], u.w[1], u.w[2], u.w[3]}, (u4_any*)p);
                return;
            }
        }
        *reinterpret_cast<Words<T, TOK>*>(p) = u;
    } else {
#pragma unroll
        for (int j = 0; j < TOK; ++j)
            if (j < left) Elt<T>::st(p + j, o[j]);
    }
}
// The same, the tokens changed by `edit` as words.
template <typename T, int TOK, bool ALL, typename F>
__device__ __forceinline__ void put_edited(T* base, uint32_t off, int left,
                                           const float (&o)[TOK], bool stream, F edit) {
    T* p = (T*)((char*)base + off);
    Words<T, TOK> u;
    pack_tokens<T, TOK>(u, o);
    edit(u);
    if (ALL || left == TOK) {
        if constexpr (TOK * sizeof(T) == 16) {
            if (stream) {
                typedef uint32_t __attribute__((ext_vector_type(4))) u4;
                typedef u4 __attribute__((aligned(2), may_alias)) u4_any;
                __builtin_nontemporal_store(u4{u.w[0], u.w[1], u.w[2], u.w[3]}, (u4_any*)p);
                return;
            }
        }
        *reinterpret_cast<Words<T, TOK>*>(p) = u;
    } else if constexpr (TOK > 1) {
#pragma unroll
        for (int j = 0; j < TOK; ++j)
            if (j < left) {
                Words<T, 1> e;
                e.w[0] = sizeof(T) == 4 ? u.w[j] : u.w[j / 2] >> (j & 1 ? 16 : 0);
                *reinterpret_cast<Words<T, 1>*>(p + j) = e;
            }
    }
}

}  // namespace rat3d
