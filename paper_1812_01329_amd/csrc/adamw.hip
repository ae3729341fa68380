// AdamW on many tensors in one call, with states of 32 or of 8 bits.
//
//   norm^2 = sum g^2,  s = min(1, max_norm / (norm + 1e-6)),  g <- s g
//   m <- b1 m + (1 - b1) g,   v <- b2 v + (1 - b2) g^2
//   p <- p - lr decay p - lr / (1 - b1^t) m / (sqrt(v) / sqrt(1 - b2^t) + eps)
//
// Two passes, both bound by memory: the norm has to be known before the first
// parameter moves (nothing moves when it is not finite), so the gradients are read
// twice.  Tensors are cut into tiles of 4096 elements, which the workgroups of a
// launch take in turn; the second pass takes them in the opposite order, for the last
// gradients of the first one are then still in the 256 MB cache before the HBM.
//
// 8-bit states: 256 elements are one access of four a lane in a wave, whose
// largest the lanes find among themselves.  With E the exponent that makes the largest
// at most 1.75 2^E, codes are e4m3 floats of x 2^(8 - E): exact but for the rounding
// of the mantissa to 3 bits, which adds 16 random bits below them and cuts off.
// sqrt(v) is kept in v's place: its range is half of v's in powers of two (e4m3
// reaches 2^-18 of the largest), and half of v's relative step.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "seq.hpp"

namespace janus {
namespace {

constexpr int kThreads = 256;
constexpr int kTile = 4096;      // elements
constexpr int kBlocks = 1024;    // workgroups a launch at most
constexpr int kTable = 40;       // tensors a launch

// The tensors of a launch of the first pass, passed by value: tile t belongs to the
// last tensor that starts at t or before.
struct NormTable {
    int n;
    int64_t tile[kTable + 1];
    const float* g[kTable];
    int64_t size[kTable];
};
struct AdamTable {
    int n, first;                // first: the place of tensor 0 in the call
    int64_t tile[kTable + 1];
    janus_adamw_tensor t[kTable];
};
static_assert(sizeof(AdamTable) < 3600, "kernel arguments hold 4 KB");

// What the first pass leaves for the second, behind the block sums of the norm
struct Control {
    int64_t t;                   // this step's number
    float rate, root;            // lr / (1 - b1^t), 1 / sqrt(1 - b2^t)
    float lr;
    uint32_t key;                // of this step's random bits
};

struct AdamArgs {
    float b1, b2, c1, c2;        // c = 1 - b
    float eps, max_norm, lr;
    uint32_t seed;
    int n_sums;
    double* sums;
    Control* ctl;
    int64_t* step;
    const float* lr_dev;
    const uint32_t* hold;
    float* stats;
};

template <typename Table>
__device__ __forceinline__ int tensor_of(const Table& t, int64_t tile) {
    int lo = 0, hi = t.n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (t.tile[mid] <= tile) lo = mid;
        else hi = mid;
    }
    return lo;
}

// 32 random bits a number
__host__ __device__ __forceinline__ uint32_t mix(uint32_t a) {
    a ^= a >> 16;
    a *= 0x6A09E667u;
    a ^= a >> 15;
    a *= 0xBB67AE85u;
    return a ^ (a >> 16);
}

__device__ __forceinline__ double block_sum(double v, double* red) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    if (lane == 0) red[wave] = v;
    __syncthreads();
    double s = 0.0;
    for (int w = 0; w < kThreads / 64; ++w) s += red[w];
    return s;
}

// Pass one: a workgroup's sum of squares; the first of the first launch also forms
// what depends on the step's number alone.
__global__ __launch_bounds__(kThreads) void adamw_norm_kernel(NormTable t, AdamArgs a, double* sums, bool first) {
    __shared__ double red[kThreads / 64];
    const int tid = threadIdx.x;
    if (first && blockIdx.x == 0 && tid == 0) {
        Control c;
        c.t = *a.step + 1;
        c.lr = a.lr_dev ? *a.lr_dev : a.lr;
        c.rate = float(double(c.lr) / (1.0 - pow(double(a.b1), double(c.t))));
        c.root = float(1.0 / sqrt(1.0 - pow(double(a.b2), double(c.t))));
        c.key = mix(mix(a.seed) ^ uint32_t(c.t));
        *a.ctl = c;
    }
    double acc = 0.0;
    for (int64_t tile = blockIdx.x; tile < t.tile[t.n]; tile += gridDim.x) {
        const int i = tensor_of(t, tile);
        const int64_t at = (tile - t.tile[i]) * kTile;
        const int64_t left = t.size[i] - at;
        const int len = int(left < kTile ? left : kTile);
        const float* g = t.g[i] + at;
        // elements before the first 16-byte boundary, then float4s, then the rest
        const int head = min(len, int((16u - (reinterpret_cast<uintptr_t>(g) & 15u)) & 15u) / 4);
        const int n4 = (len - head) / 4;
        const float4* g4 = reinterpret_cast<const float4*>(g + head);
#pragma unroll
        for (int u = 0; u < kTile / 4 / kThreads; ++u) {
            const int k = tid + u * kThreads;
            if (k < n4) {
                const float4 v = g4[k];
                acc += double(v.x) * v.x + double(v.y) * v.y + double(v.z) * v.z + double(v.w) * v.w;
            }
        }
        const int rest = head + 4 * n4 + tid;
        if (tid < head) acc += double(g[tid]) * g[tid];
        if (rest < len) acc += double(g[rest]) * g[rest];
    }
    const double s = block_sum(acc, red);
    if (tid == 0) sums[blockIdx.x] = s;
}

// One element: the moments and the parameter.  Every product and sum is rounded by
// itself (contracted, the codes of 8 bits would depend on how the compiler paired them).
struct Step {
    float b1, b2, c1, c2, eps, s, rate, root, shrink;
    __device__ __forceinline__ void moments(float g, float& m, float& v) const {
#pragma clang fp contract(off)
        g = g * s;
        m = m * b1 + g * c1;
        v = v * b2 + (g * g) * c2;
    }
    __device__ __forceinline__ float parameter(float p, float m, float r) const {
        return p - p * shrink - rate * m / (r * root + eps);
    }
};

// Four elements at p, of which `k` are there; whole vectors where they are aligned.
template <typename T>
__device__ __forceinline__ void load4(const T* p, int k, bool vec, float* f) {
    if (vec && k == 4) {
        Chan<T, 4> v;
        v.load(p);
        v.get(f);
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) f[j] = j < k ? to_f(p[j]) : 0.f;
    }
}
template <typename T>
__device__ __forceinline__ void store4(T* p, int k, bool vec, const float* f) {
    if (vec && k == 4) {
        Chan<T, 4>::store(p, f);
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (j < k) p[j] = out_f<T>(f[j]);
    }
}
__device__ __forceinline__ uint32_t load_codes(const uint8_t* p, int k, bool vec) {
    if (vec && k == 4) return *reinterpret_cast<const uint32_t*>(p);
    uint32_t v = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (j < k) v |= uint32_t(p[j]) << (8 * j);
    return v;
}
__device__ __forceinline__ void store_codes(uint8_t* p, int k, bool vec, uint32_t v) {
    if (vec && k == 4) {
        *reinterpret_cast<uint32_t*>(p) = v;
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (j < k) p[j] = uint8_t(v >> (8 * j));
    }
}

typedef float f32x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ void decode(uint32_t codes, float scale, float* f) {
    const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8(int(codes), false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(int(codes), true);
    f[0] = lo.x * scale, f[1] = lo.y * scale, f[2] = hi.x * scale, f[3] = hi.y * scale;
}

// |x| of a wave's 256 elements as codes and the power of two that goes with them;
// rnd: 16 random bits an element.
constexpr float kLargest = 1.75f * 0x1p127f;
__device__ __forceinline__ uint32_t encode(const float* f, const uint32_t* rnd, float& scale) {
    float a[4], top = 0.f;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        a[j] = fminf(fabsf(f[j]), kLargest);
        top = fmaxf(top, a[j]);
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor(top, o, 64));
    // (the exponent goes up by one where the mantissa is past 1.75)
    const uint32_t E = max((__float_as_uint(top) + 0x1FFFFFu) >> 23, 9u);
    scale = __uint_as_float((E - 8u) << 23);
    const float inv = __uint_as_float((262u - E) << 23);
    uint32_t out = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const float t = a[j] * inv;                       // at most 448, exact
        const uint32_t bits = __float_as_uint(t), r = rnd[j] << 4;
        const uint32_t code = bits >= (121u << 23) ? ((bits + r) >> 20) - 960u            // from 2^-6 on: 3 bits of mantissa
                                                   : (uint32_t(t * 0x1p29f) + r) >> 20;   // steps of 2^-9
        out |= (code | (f[j] < 0.f ? 0x80u : 0u)) << (8 * j);
    }
    return out;
}

// What every thread of the second pass needs of the first, or false when nothing may change
__device__ bool form_step(const AdamArgs& a, Step& st, Control& c, bool report) {
    __shared__ double red[kThreads / 64];
    double acc = 0.0;
    for (int k = threadIdx.x; k < a.n_sums; k += kThreads) acc += a.sums[k];
    const double norm = sqrt(block_sum(acc, red));
    c = *a.ctl;
    const bool go = isfinite(norm) && isfinite(c.lr) && !(a.hold && *a.hold);
    double s = 1.0;
    if (!go) s = 0.0;
    else if (a.max_norm > 0.f && isfinite(a.max_norm)) s = fmin(1.0, double(a.max_norm) / (norm + 1e-6));
    if (report && threadIdx.x == 0) {
        if (a.stats) a.stats[0] = float(norm), a.stats[1] = float(s);
        if (go) *a.step = c.t;   // (the other workgroups have it from the control word)
    }
    st.b1 = a.b1, st.b2 = a.b2, st.c1 = a.c1, st.c2 = a.c2, st.eps = a.eps;
    st.s = float(s), st.rate = c.rate, st.root = c.root, st.shrink = 0.f;
    return go;
}

__device__ __forceinline__ bool aligned4(const void* p, unsigned a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

template <typename T, bool Q>
__device__ __forceinline__ void adamw_tile(const janus_adamw_tensor& t, const Step& st, uint32_t key, int64_t at) {
    const int64_t left = t.size - at;
    const int len = int(left < kTile ? left : kTile);
    const float* g = t.g + at;
    T* p = static_cast<T*>(t.p) + at;
    float* w = t.master ? t.master + at : nullptr;
    const bool vg = aligned4(g, 16), vp = aligned4(p, 4 * sizeof(T)), vw = aligned4(w, 16);
#pragma unroll 2
    for (int u = 0; u < kTile / 4 / kThreads; ++u) {
        const int e = (threadIdx.x + u * kThreads) * 4;
        if ((e & ~255) >= len) break;                    // (256 elements are a wave's: it goes on as a whole)
        const int k = min(max(len - e, 0), 4);
        float gf[4], pf[4], m[4], v[4], r[4];
        load4(g + e, k, vg, gf);
        if (w) load4(w + e, k, vw, pf);
        else load4(p + e, k, vp, pf);
        if constexpr (Q) {
            uint8_t *mc = static_cast<uint8_t*>(t.m) + at + e, *vc = static_cast<uint8_t*>(t.v) + at + e;
            const bool vm = aligned4(t.m, 4), vv = aligned4(t.v, 4);
            float2* sp = reinterpret_cast<float2*>(t.scale + (at + e) / 256 * 2);
            const float2 sc = *sp;
            decode(load_codes(mc, k, vm), sc.x, m);
            decode(load_codes(vc, k, vv), sc.y, v);
            uint32_t rm[4], rv[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                v[j] = v[j] * v[j];
                st.moments(gf[j], m[j], v[j]);
                r[j] = __fsqrt_rn(v[j]);
                const uint32_t x = mix(uint32_t(at + e + j) ^ key);
                rm[j] = x & 0xffffu, rv[j] = x >> 16;
            }
            float sm, sv;
            const uint32_t cm = encode(m, rm, sm), cv = encode(r, rv, sv);
            store_codes(mc, k, vm, cm);
            store_codes(vc, k, vv, cv);
            if ((threadIdx.x & 63) == 0) *sp = make_float2(sm, sv);
        } else {
            float *mp = static_cast<float*>(t.m) + at + e, *vp_ = static_cast<float*>(t.v) + at + e;
            const bool vm = aligned4(t.m, 16), vv = aligned4(t.v, 16);
            load4(mp, k, vm, m);
            load4(vp_, k, vv, v);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                st.moments(gf[j], m[j], v[j]);
                r[j] = sqrtf(v[j]);
            }
            store4(mp, k, vm, m);
            store4(vp_, k, vv, v);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) pf[j] = st.parameter(pf[j], m[j], r[j]);
        if (w) store4(w + e, k, vw, pf);
        store4(p + e, k, vp, pf);
    }
}

template <bool Q>
__global__ __launch_bounds__(kThreads) void adamw_update_kernel(AdamTable t, AdamArgs a, bool report) {
    Step st;
    Control c;
    if (!form_step(a, st, c, report && blockIdx.x == 0)) return;
    for (int64_t tile = t.tile[t.n] - 1 - blockIdx.x; tile >= 0; tile -= gridDim.x) {
        const int i = tensor_of(t, tile);
        const janus_adamw_tensor& x = t.t[i];
        st.shrink = c.lr * x.decay;
        const uint32_t key = mix(c.key ^ uint32_t(t.first + i));
        const int64_t at = (tile - t.tile[i]) * kTile;
        if (x.dtype == JANUS_BF16) adamw_tile<bf16_t, Q>(x, st, key, at);
        else adamw_tile<float, Q>(x, st, key, at);
    }
}

constexpr int chunks(int n) { return (n + kTable - 1) / kTable; }
size_t adamw_carve(AdamArgs& a, int n, void* ws) {
    Carver c(ws);
    a.ctl = c.take<Control>(1);
    a.sums = c.take<double>(size_t(chunks(n)) * kBlocks);
    return c.off;
}

bool adamw_desc_ok(const janus_adamw_desc* d) {
    return d && d->n >= 1 && std::isfinite(d->lr) && d->beta1 >= 0.f && d->beta1 < 1.f && d->beta2 >= 0.f &&
           d->beta2 < 1.f && std::isfinite(d->eps) && d->eps > 0.f && !std::isnan(d->max_norm);
}

janus_status adamw_check(const janus_adamw_desc* d, const janus_adamw_tensor* tensors) {
    const bool q = d->states == JANUS_ADAMW_8BIT;
    for (int i = 0; i < d->n; ++i) {
        const janus_adamw_tensor& t = tensors[i];
        if (!dtype_ok(t.dtype)) return JANUS_ERR_UNSUPPORTED;
        if (t.size < 0 || !std::isfinite(t.decay) || (t.master && t.dtype == JANUS_F32)) return JANUS_ERR_INVALID_ARG;
        if (t.size > (q ? (int64_t(1) << 32) : (int64_t(1) << 40))) return JANUS_ERR_UNSUPPORTED;
        if (t.size > 0 && (!t.p || !t.g || !t.m || !t.v || (q && !t.scale))) return JANUS_ERR_INVALID_ARG;
        if (!aligned(t.p, dtype_size(t.dtype)) || !aligned(t.g, 4) || !aligned(t.master, 4) ||
            (q ? !aligned(t.scale, 8) : !aligned(t.m, 4) || !aligned(t.v, 4)))
            return JANUS_ERR_INVALID_ARG;
    }
    return JANUS_OK;
}

}  // namespace
}  // namespace janus

using namespace janus;

extern "C" size_t janus_adamw_workspace_bytes(const janus_adamw_desc* d) {
    if (!adamw_desc_ok(d) || (d->states != JANUS_ADAMW_F32 && d->states != JANUS_ADAMW_8BIT)) return 0;
    AdamArgs a{};
    return adamw_carve(a, d->n, nullptr);
}

extern "C" janus_status janus_adamw_update(const janus_adamw_desc* d, const janus_adamw_tensor* tensors, int64_t* step,
                                           const float* lr, float* stats, const uint32_t* hold, void* ws,
                                           size_t ws_bytes, void* stream) {
    if (!adamw_desc_ok(d) || !tensors || !step) return JANUS_ERR_INVALID_ARG;
    if (d->states != JANUS_ADAMW_F32 && d->states != JANUS_ADAMW_8BIT) return JANUS_ERR_UNSUPPORTED;
    if (!aligned(step, 8) || !aligned(lr, 4) || !aligned(stats, 4) || !aligned(hold, 4)) return JANUS_ERR_INVALID_ARG;
    janus_status e = adamw_check(d, tensors);
    if (e != JANUS_OK) return e;
    AdamArgs a{};
    const size_t need = adamw_carve(a, d->n, ws);
    if (!ws || ws_bytes < need || !aligned(ws, 256)) return JANUS_ERR_WORKSPACE;
    a.b1 = d->beta1, a.b2 = d->beta2;
    a.c1 = float(1.0 - double(d->beta1)), a.c2 = float(1.0 - double(d->beta2));
    a.eps = d->eps, a.max_norm = d->max_norm, a.lr = d->lr, a.seed = d->seed;
    a.step = step, a.lr_dev = lr, a.hold = hold, a.stats = stats;
    hipStream_t st = static_cast<hipStream_t>(stream);
    const bool q = d->states == JANUS_ADAMW_8BIT;
    auto tiles = [](int64_t size) { return (size + kTile - 1) / kTile; };
    double* sums = a.sums;
    for (int c = 0; c < chunks(d->n); ++c) {
        NormTable t{};
        const int i0 = c * kTable;
        t.n = std::min(d->n - i0, kTable);
        for (int i = 0; i < t.n; ++i) {
            t.g[i] = tensors[i0 + i].g, t.size[i] = tensors[i0 + i].size;
            t.tile[i + 1] = t.tile[i] + tiles(t.size[i]);
        }
        const int blocks = int(std::max<int64_t>(1, std::min<int64_t>(kBlocks, t.tile[t.n])));
        TraceScope trace("adamw_norm", 2.0 * kTile * double(t.tile[t.n]), 4.0 * kTile * double(t.tile[t.n]), st);
        hipLaunchKernelGGL(adamw_norm_kernel, dim3(blocks), dim3(kThreads), 0, st, t, a, sums, c == 0);
        JANUS_LAUNCH_CHECK();
        sums += blocks;
        a.n_sums += blocks;
    }
    for (int c = 0; c < chunks(d->n); ++c) {
        AdamTable t{};
        const int i0 = c * kTable;
        t.n = std::min(d->n - i0, kTable), t.first = i0;
        double bytes = 0.0;
        for (int i = 0; i < t.n; ++i) {
            t.t[i] = tensors[i0 + i];
            t.tile[i + 1] = t.tile[i] + tiles(t.t[i].size);
            bytes += double(t.t[i].size) * (4 + 2 * double(dtype_size(t.t[i].dtype)) + (q ? 4 : 16) + (t.t[i].master ? 8 : 0));
        }
        const int blocks = int(std::max<int64_t>(1, std::min<int64_t>(kBlocks, t.tile[t.n])));
        TraceScope trace("adamw_update", 16.0 * kTile * double(t.tile[t.n]), bytes, st);
        // (the last launch reports: every other one has read the step's number by then)
        const bool report = c == chunks(d->n) - 1;
        if (q) hipLaunchKernelGGL(adamw_update_kernel<true>, dim3(blocks), dim3(kThreads), 0, st, t, a, report);
        else hipLaunchKernelGGL(adamw_update_kernel<false>, dim3(blocks), dim3(kThreads), 0, st, t, a, report);
        JANUS_LAUNCH_CHECK();
    }
    return JANUS_OK;
}
