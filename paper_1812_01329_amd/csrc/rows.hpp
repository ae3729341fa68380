// What the kernels that work on whole rows share: sums over a wave, and rows read
// in pieces of 16 bytes wherever they start.
#pragma once

#include "seq.hpp"

namespace janus {

__device__ __forceinline__ float wsum(float v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
    return v;
}
__device__ __forceinline__ float wmax(float v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor(v, o, 64));
    return v;
}
__device__ __forceinline__ double wsum(double v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
    return v;
}

template <typename T>
struct Piece {   // 16 bytes of a row
    static constexpr int VEC = 16 / sizeof(T);
    uint4 v;
    __device__ __forceinline__ float get(int j) const {
        const uint32_t* u = reinterpret_cast<const uint32_t*>(&v);
        if constexpr (sizeof(T) == 4) return __uint_as_float(u[j]);
        else return j & 1 ? hi2f(u[j / 2]) : lo2f(u[j / 2]);
    }
    __device__ __forceinline__ void set(int j, T x) {
        T t[VEC];
        __builtin_memcpy(t, &v, 16);
        t[j] = x;
        __builtin_memcpy(&v, t, 16);
    }
};

// Rows start at any element; a row is cut at 16-byte boundaries of memory, so
// only its first and last piece can be partial: those go element by element, and
// elements outside the row count as -inf.
template <typename T>
struct Row {
    static constexpr int VEC = 16 / sizeof(T);
    const T* base;   // first element's 16-byte boundary (not all of the first piece is the row's)
    int lo, hi;      // the row: elements [lo, hi) from base
    __device__ __forceinline__ Row(const T* p, int V) {
        const int mis = int(reinterpret_cast<uintptr_t>(p) % 16 / sizeof(T));
        base = p - mis, lo = mis, hi = mis + V;
    }
    __device__ __forceinline__ int pieces() const { return (hi + VEC - 1) / VEC; }
    __device__ __forceinline__ bool whole(int p) const { return p * VEC >= lo && p * VEC + VEC <= hi; }
    __device__ __forceinline__ Piece<T> load(int p) const {
        Piece<T> r;
        if (whole(p)) {
            r.v = *reinterpret_cast<const uint4*>(base + int64_t(p) * VEC);
        } else {
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                const int i = p * VEC + j;
                r.set(j, i >= lo && i < hi ? base[i] : out_f<T>(-INFINITY));
            }
        }
        return r;
    }
    // to another row with the same cut (or `same` false: element by element)
    __device__ __forceinline__ void store(T* out, bool same, int p, const float* f) const {
        if (same && whole(p)) {
            Chan<T, VEC>::store(out + int64_t(p) * VEC, f);
        } else {
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                const int i = p * VEC + j;
                if (i >= lo && i < hi) out[i] = out_f<T>(f[j]);
            }
        }
    }
};

}  // namespace janus
