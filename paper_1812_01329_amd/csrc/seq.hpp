// What the convolution and the scan over variable-length sequences share:
// argument checks, lengths passed to kernels by value, and loads and stores of
// a few channels at once.
#pragma once

#include <algorithm>

#include "device.hpp"
#include "runtime.hpp"

namespace janus {

// Up to kSlice sequences and their lengths as a kernel argument: no upload, no
// device buffer, and a captured launch keeps its own copy.  Larger batches
// take one launch per slice.  The longest come first: workgroups start in that
// order, and a short sequence at the end leaves less of the chip idle than a
// long one.
constexpr int kSlice = 256;
struct SeqSlice {
    int32_t b0;               // first sequence of the slice
    int32_t len[kSlice];
    uint8_t at[kSlice];       // entry i is sequence b0 + at[i]
};

// The sequence of entry i (a byte comes through a vector register: made uniform again)
__device__ __forceinline__ int seq_of(const SeqSlice& s, int i) {
    return s.b0 + __builtin_amdgcn_readfirstlane(int(s.at[i]));
}

inline janus_status check_lengths(int32_t B, int32_t T, const int32_t* lengths) {
    if (lengths)
        for (int32_t b = 0; b < B; ++b)
            if (lengths[b] < 0 || lengths[b] > T) return JANUS_ERR_LENGTH;
    return JANUS_OK;
}

// Sequences [b0, b0 + kSlice) of the batch; returns how many there are.
inline int fill_slice(SeqSlice& s, int32_t b0, int32_t B, int32_t T, const int32_t* lengths) {
    const int n = std::min(kSlice, B - b0);
    s.b0 = b0;
    for (int i = 0; i < n; ++i) s.at[i] = uint8_t(i);
    if (lengths) std::stable_sort(s.at, s.at + n, [&](uint8_t i, uint8_t j) { return lengths[b0 + i] > lengths[b0 + j]; });
    for (int i = 0; i < n; ++i) s.len[i] = lengths ? lengths[b0 + s.at[i]] : T;
    return n;
}

inline bool aligned(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

// float -> bf16, round to nearest even (v_cvt_pk_bf16_f32)
typedef float f32x2_t __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t pack2(float a, float b) {
    const f32x2_t v = {a, b};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2_t));
}
template <typename T> __device__ __forceinline__ T out_f(float v);
template <> __device__ __forceinline__ float out_f<float>(float v) { return v; }
template <> __device__ __forceinline__ bf16_t out_f<bf16_t>(float v) { return __builtin_bit_cast(bf16_t, (__bf16)v); }

// VEC consecutive channels in one access (the pointer is aligned to it)
template <typename T, int VEC> struct Chan;
template <> struct Chan<float, 1> {
    float v;
    __device__ __forceinline__ void load(const float* p) { v = *p; }
    __device__ __forceinline__ void get(float* f) const { f[0] = v; }
    __device__ __forceinline__ static void store(float* p, const float* f) { *p = f[0]; }
};
template <> struct Chan<float, 4> {
    float4 v;
    __device__ __forceinline__ void load(const float* p) { v = *reinterpret_cast<const float4*>(p); }
    __device__ __forceinline__ void get(float* f) const { f[0] = v.x, f[1] = v.y, f[2] = v.z, f[3] = v.w; }
    __device__ __forceinline__ static void store(float* p, const float* f) {
        *reinterpret_cast<float4*>(p) = make_float4(f[0], f[1], f[2], f[3]);
    }
};
template <> struct Chan<bf16_t, 1> {
    bf16_t v;
    __device__ __forceinline__ void load(const bf16_t* p) { v = *p; }
    __device__ __forceinline__ void get(float* f) const { f[0] = bf2f(v); }
    __device__ __forceinline__ static void store(bf16_t* p, const float* f) { *p = out_f<bf16_t>(f[0]); }
};
// two bf16 of one word, and back
__device__ __forceinline__ float lo2f(uint32_t u) { return __uint_as_float(u << 16); }
__device__ __forceinline__ float hi2f(uint32_t u) { return __uint_as_float(u & 0xffff0000u); }
template <> struct Chan<bf16_t, 2> {
    uint32_t v;
    __device__ __forceinline__ void load(const bf16_t* p) { v = *reinterpret_cast<const uint32_t*>(p); }
    __device__ __forceinline__ void get(float* f) const { f[0] = lo2f(v), f[1] = hi2f(v); }
    __device__ __forceinline__ static void store(bf16_t* p, const float* f) {
        *reinterpret_cast<uint32_t*>(p) = pack2(f[0], f[1]);
    }
};
template <> struct Chan<bf16_t, 4> {
    uint2 v;
    __device__ __forceinline__ void load(const bf16_t* p) { v = *reinterpret_cast<const uint2*>(p); }
    __device__ __forceinline__ void get(float* f) const {
        f[0] = lo2f(v.x), f[1] = hi2f(v.x), f[2] = lo2f(v.y), f[3] = hi2f(v.y);
    }
    __device__ __forceinline__ static void store(bf16_t* p, const float* f) {
        *reinterpret_cast<uint2*>(p) = make_uint2(pack2(f[0], f[1]), pack2(f[2], f[3]));
    }
};
template <> struct Chan<bf16_t, 8> {
    uint4 v;
    __device__ __forceinline__ void load(const bf16_t* p) { v = *reinterpret_cast<const uint4*>(p); }
    __device__ __forceinline__ void get(float* f) const {
        f[0] = lo2f(v.x), f[1] = hi2f(v.x), f[2] = lo2f(v.y), f[3] = hi2f(v.y);
        f[4] = lo2f(v.z), f[5] = hi2f(v.z), f[6] = lo2f(v.w), f[7] = hi2f(v.w);
    }
    __device__ __forceinline__ static void store(bf16_t* p, const float* f) {
        *reinterpret_cast<uint4*>(p) =
            make_uint4(pack2(f[0], f[1]), pack2(f[2], f[3]), pack2(f[4], f[5]), pack2(f[6], f[7]));
    }
};

}  // namespace janus
