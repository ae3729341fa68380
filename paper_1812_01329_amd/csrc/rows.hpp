// What the kernels that work on whole rows or blocks share: sums, scans and maxima over
// a wave, and rows read in pieces of 16 bytes wherever they start.
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

typedef unsigned long long u64;

// ---- sums, scans and maxima over a wave, by moves between neighbouring lanes and rows of 16
template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t moved(uint32_t old, uint32_t v) {
    return uint32_t(__builtin_amdgcn_update_dpp(int(old), int(v), CTRL, ROWS, 0xf, false));
}
template <int CTRL, int ROWS>
__device__ __forceinline__ u64 moved(u64 old, u64 v) {
    return u64(moved<CTRL, ROWS>(uint32_t(old), uint32_t(v))) |
           u64(moved<CTRL, ROWS>(uint32_t(old >> 32), uint32_t(v >> 32))) << 32;
}
template <int CTRL, int ROWS>
__device__ __forceinline__ float moved(float old, float v) {
    return __uint_as_float(moved<CTRL, ROWS>(__float_as_uint(old), __float_as_uint(v)));
}
// f(... f(first, second) ..., this lane's); `none`: what f leaves as it is
template <typename S, typename F>
__device__ __forceinline__ S wave_scan(S v, S none, F f) {
    v = f(v, moved<0x111, 0xf>(none, v));   // from 1, 2, 4, 8 lanes before in the row
    v = f(v, moved<0x112, 0xf>(none, v));
    v = f(v, moved<0x114, 0xf>(none, v));
    v = f(v, moved<0x118, 0xf>(none, v));
    v = f(v, moved<0x142, 0xa>(none, v));   // the row's last to the next row (rows 1 and 3)
    v = f(v, moved<0x143, 0xc>(none, v));   // lane 31 to the upper half
    return v;
}
__device__ __forceinline__ u64 up_to(u64 v) { return wave_scan(v, u64(0), [](u64 a, u64 b) { return a + b; }); }
__device__ __forceinline__ uint32_t up_to(uint32_t v) { return wave_scan(v, 0u, [](uint32_t a, uint32_t b) { return a + b; }); }
__device__ __forceinline__ uint32_t last_lane(uint32_t v) { return uint32_t(__builtin_amdgcn_readlane(int(v), 63)); }
__device__ __forceinline__ u64 last_lane(u64 v) { return u64(last_lane(uint32_t(v))) | u64(last_lane(uint32_t(v >> 32))) << 32; }
__device__ __forceinline__ float last_lane(float v) { return __uint_as_float(last_lane(__float_as_uint(v))); }
__device__ __forceinline__ float wave_max(float v) {
    return last_lane(wave_scan(v, -INFINITY, [](float a, float b) { return fmaxf(a, b); }));
}
__device__ __forceinline__ float wave_sum(float v) {
    return last_lane(wave_scan(v, 0.f, [](float a, float b) { return a + b; }));
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
