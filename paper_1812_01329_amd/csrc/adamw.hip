// AdamW on many tensors in one call, with states of 32 or of 8 bits.
//
//   norm^2 = sum g^2,  s = min(1, max_norm / (norm + 1e-6)),  g <- s g
//   m <- b1 m + (1 - b1) g,   v <- b2 v + (1 - b2) g^2
//   p <- p - lr decay p - lr / (1 - b1^t) m / (sqrt(v) / sqrt(1 - b2^t) + eps)
//
// Two passes, both bound by memory: the norm has to be known before the first
// parameter moves (nothing moves when it is not finite), so the gradients are read
// twice.  Tensors are cut into tiles of 1024 or 4096 elements, which the workgroups of a
// launch take in turn; the second pass takes them in the opposite order, for the last
// gradients of the first one are then still in the 256 MB cache before the HBM.  A
// table of the tensors goes to the kernels by value; one of more than 52 is written to the
// workspace by launches that have a part of it each, and each pass stays one launch.
//
// 8-bit states: 256 elements are one access of four a lane in a wave, whose
// largest the lanes find among themselves.  With E the exponent that makes the largest
// at most 1.75 2^E, codes are e4m3 floats of x 2^(8 - E): exact but for the rounding
// of the mantissa to 3 bits, which adds 16 random bits below them and cuts off.
// sqrt(v) is kept in v's place: its range is half of v's in powers of two (e4m3
// reaches 2^-18 of the largest), and half of v's relative step.  Where a root was kept as 0,
// the parameter's step takes one of at least sqrt(b2) 2^-9 of its block's power, the least that
// the block could have held: m has a power of its own and may be left, and m / eps is a step of
// 470 lr half of a block's gradients of N(0, 1) after a single one of 1e-4 (so: 2.3).
//
// 19.8 M float32 parameters with 32-bit states: the norm 14.7 us (5.4 TB/s, partly from
// the cache), the update 88 (6.3 TB/s with gradients in the cache; 108 us a call, where a
// copy of the same bytes takes 117).  71 M of bf16 with masters and 8-bit states: 45 and 215 us
// (257 a call, 273).  10 small tensors: 3.2 and 4.7 us, latency.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "rows.hpp"

namespace janus {
namespace {

constexpr int kThreads = 256;
constexpr int kBlocks = 1024;    // workgroups a launch at most
constexpr int kTable = 52;       // tensors of a table passed by value
constexpr int kStarts = 1024;    // tensors whose tiles are looked up in LDS

// Tensors and their tiles: tile t belongs to the last tensor that starts at t or before.
struct TensorTable {
    int n, first;                // first: the place of tensor 0 in the call
    int64_t tile[kTable + 1];
    janus_adamw_tensor t[kTable];
};
static_assert(sizeof(TensorTable) < 3800, "kernel arguments hold 4 KB");
struct Tensors {                 // the same in the workspace
    int n;
    const int64_t* tile;
    const janus_adamw_tensor* t;
};

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
    float least;                 // sqrt(b2) 2^-9: a root of 0 in 8 bits in the next step, of its power of two
    uint32_t seed;
    int n_sums;
    double* sums;
    Control* ctl;
    int64_t* step;
    const float* lr_dev;
    const uint32_t* hold;
    float* stats;
};

// Tiles' tensors are found by a copy of their starts in LDS; a table passed by value has so
// few that it is read in its place.
__device__ __forceinline__ void prepare(const TensorTable&, int64_t*) {}
__device__ __forceinline__ int64_t start(const TensorTable& t, const int64_t*, int i) { return t.tile[i]; }
__device__ __forceinline__ void prepare(const Tensors& t, int64_t* lds) {
    if (t.n <= kStarts)
        for (int i = threadIdx.x; i <= t.n; i += kThreads) lds[i] = t.tile[i];
    __syncthreads();
}
__device__ __forceinline__ int64_t start(const Tensors& t, const int64_t* lds, int i) {
    return t.n <= kStarts ? lds[i] : t.tile[i];
}
template <typename Table>
__device__ __forceinline__ int tensor_of(const Table& t, const int64_t* lds, int64_t tile) {
    int lo = 0, hi = t.n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (start(t, lds, mid) <= tile) lo = mid;
        else hi = mid;
    }
    return __builtin_amdgcn_readfirstlane(lo);
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

__global__ void adamw_table_kernel(TensorTable v, int64_t* tile, janus_adamw_tensor* t) {
    const int i = threadIdx.x;
    if (i <= v.n) tile[v.first + i] = v.tile[i];   // (the next part's first again, or the end)
    if (i < v.n) t[v.first + i] = v.t[i];
}

// Pass one: a workgroup's sum of squares; the first one also forms what depends on the
// step's number alone.
template <int TILE, typename Table>
__global__ __launch_bounds__(kThreads) void adamw_norm_kernel(Table t, AdamArgs a) {
    __shared__ double red[kThreads / 64];
    __shared__ int64_t lds[kStarts + 1];
    prepare(t, lds);
    const int tid = threadIdx.x;
    if (blockIdx.x == 0 && tid == 0) {
        Control c;
        c.t = *a.step + 1;
        c.lr = a.lr_dev ? *a.lr_dev : a.lr;
        c.rate = float(double(c.lr) / (1.0 - pow(double(a.b1), double(c.t))));
        c.root = float(1.0 / sqrt(1.0 - pow(double(a.b2), double(c.t))));
        c.key = mix(mix(a.seed) ^ uint32_t(c.t));
        *a.ctl = c;
    }
    // the next tile is on its way while one is added up
    constexpr int U = TILE / 4 / kThreads;
    struct Part {
        float4 v[U];
        float edge[2];
    };
    auto load = [&](int64_t tile, Part& x) {
        const int i = tensor_of(t, lds, tile);
        const int64_t at = (tile - start(t, lds, i)) * TILE;
        const int64_t left = t.t[i].size - at;
        const int len = int(left < TILE ? left : TILE);
        const float* g = t.t[i].g + at;
        // elements before the first 16-byte boundary, then float4s, then the rest
        const int head = min(len, int((16u - (reinterpret_cast<uintptr_t>(g) & 15u)) & 15u) / 4);
        const int n4 = (len - head) / 4;
        const float4* g4 = reinterpret_cast<const float4*>(g + head);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int k = tid + u * kThreads;
            x.v[u] = k < n4 ? g4[k] : make_float4(0.f, 0.f, 0.f, 0.f);
        }
        const int rest = head + 4 * n4 + tid;
        x.edge[0] = tid < head ? g[tid] : 0.f;
        x.edge[1] = rest < len ? g[rest] : 0.f;
    };
    double acc = 0.0;
    auto add = [&](const Part& x) {
#pragma unroll
        for (int u = 0; u < U; ++u)
            acc += double(x.v[u].x) * x.v[u].x + double(x.v[u].y) * x.v[u].y + double(x.v[u].z) * x.v[u].z + double(x.v[u].w) * x.v[u].w;
        acc += double(x.edge[0]) * x.edge[0] + double(x.edge[1]) * x.edge[1];
    };
    const int64_t tiles = start(t, lds, t.n);
    int64_t tile = blockIdx.x;
    if (tile < tiles) {
        Part x, y;
        load(tile, x);
        while (true) {
            if ((tile += gridDim.x) >= tiles) {
                add(x);
                break;
            }
            load(tile, y);
            add(x);
            if ((tile += gridDim.x) >= tiles) {
                add(y);
                break;
            }
            load(tile, x);
            add(y);
        }
    }
    const double s = block_sum(acc, red);
    if (tid == 0) a.sums[blockIdx.x] = s;
}

// One element: the moments and the parameter.  Every product and sum is rounded by
// itself (contracted, the codes of 8 bits would depend on how the compiler paired them).
struct Step {
    float b1, b2, c1, c2, eps, s, rate, root, shrink, least;
    __device__ __forceinline__ void moments(float g, float& m, float& v) const {
#pragma clang fp contract(off)
        g = g * s;
        m = m * b1 + g * c1;
        v = v * b2 + (g * g) * c2;
    }
    __device__ __forceinline__ float parameter(float p, float m, float r) const {
        // (off by an ulp of the step; eps is 2^-126 at least, whose reciprocal is finite)
        return p - p * shrink - rate * (m * __builtin_amdgcn_rcpf(r * root + eps));
    }
};

// Four elements at p: SOME, `k` of them are there; ALL, one access wherever it starts, and the
// loads go out without a branch between them; PAST, one access that starts at a multiple of its
// size and goes past the caches: what the update reads and writes is not met again before the next step, and leaves the gradients of the first
// pass their place (19.8 M float32 parameters: 108 us a call, 130 without; 71 M
// of bf16 with masters and 8-bit states 269 and 320 when it was tried; the first pass's own
// loads: slower so).
enum How { SOME, ALL, PAST };
template <typename T> struct Access;
template <> struct Access<float> {
    typedef float V __attribute__((ext_vector_type(4)));
};
template <> struct Access<bf16_t> {
    typedef uint32_t V __attribute__((ext_vector_type(2)));
};
template <> struct Access<uint8_t> {
    typedef uint32_t V;
};
template <How HOW, typename T>
__device__ __forceinline__ typename Access<T>::V fetch(const T* p) {
    typedef typename Access<T>::V V;
    if constexpr (HOW == PAST) return __builtin_nontemporal_load(reinterpret_cast<const V*>(p));
    V v;
    __builtin_memcpy(&v, p, sizeof(V));
    return v;
}
template <How HOW, typename T>
__device__ __forceinline__ void put(T* p, typename Access<T>::V v) {
    if constexpr (HOW == PAST) __builtin_nontemporal_store(v, reinterpret_cast<typename Access<T>::V*>(p));
    else __builtin_memcpy(p, &v, sizeof(v));
}
template <How HOW, typename T>
__device__ __forceinline__ void load4(const T* p, int k, float* f) {
    if (HOW != SOME || k == 4) {
        Chan<T, 4> v;
        const typename Access<T>::V x = fetch<HOW>(p);
        __builtin_memcpy(&v.v, &x, sizeof(x));
        v.get(f);
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) f[j] = j < k ? to_f(p[j]) : 0.f;
    }
}
template <How HOW, typename T>
__device__ __forceinline__ void store4(T* p, int k, const float* f) {
    if (HOW != SOME || k == 4) {
        alignas(16) T v[4];
        Chan<T, 4>::store(v, f);
        typename Access<T>::V x;
        __builtin_memcpy(&x, v, sizeof(x));
        put<HOW>(p, x);
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (j < k) p[j] = out_f<T>(f[j]);
    }
}
template <How HOW>
__device__ __forceinline__ uint32_t load_codes(const uint8_t* p, int k) {
    if (HOW != SOME || k == 4) return fetch<HOW>(p);
    uint32_t v = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (j < k) v |= uint32_t(p[j]) << (8 * j);
    return v;
}
template <How HOW>
__device__ __forceinline__ void store_codes(uint8_t* p, int k, uint32_t v) {
    if (HOW != SOME || k == 4) {
        put<HOW>(p, v);
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (j < k) p[j] = uint8_t(v >> (8 * j));
    }
}

// sqrt(v), rounded correctly, as the codes' definition has it: the machine's root is off by its last
// bit at times; of it and its neighbours the one that v lies next to
__device__ __forceinline__ float root_of(float v) {
    if (!(v >= 0x1p-64f && v < INFINITY)) return sqrtf(v);   // (the products below would leave float32)
    const float s = __builtin_amdgcn_sqrtf(v);
    const float down = __uint_as_float(__float_as_uint(s) - 1u), up = __uint_as_float(__float_as_uint(s) + 1u);
    // the borders are the squares of the means: (s - ulp / 2)^2 = s down + ulp^2 / 4
    if (fmaf(-down, s, v) <= 0.f) return down;
    return fmaf(-up, s, v) > 0.f ? up : s;
}

// sqrt v to an ulp; the instruction takes subnormal ones for 0
__device__ __forceinline__ float near_root(float v) {
    const bool low = v < 0x1p-96f;
    return __builtin_amdgcn_sqrtf(low ? v * 0x1p64f : v) * (low ? 0x1p-32f : 1.f);
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
    top = wave_max(top);
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
    st.s = float(s), st.rate = c.rate, st.root = c.root, st.shrink = 0.f, st.least = a.least;
    return go;
}

// Four elements of a tensor, from element e on: k of them are there.
template <typename T, bool Q>
__device__ __forceinline__ bool even(const janus_adamw_tensor& t) {
    auto at = [](const void* p) { return uint32_t(reinterpret_cast<uintptr_t>(p)); };
    return ((at(t.p) & (4 * sizeof(T) - 1)) | (at(t.g) & 15u) | (at(t.master) & 15u) | ((at(t.m) | at(t.v)) & (Q ? 3u : 15u))) == 0;
}
template <typename T, bool Q>
struct Four {
    float g[4], p[4], m[4], v[4];
    uint32_t mc, vc;
    float2 scale;
    int k;
    template <How HOW>
    __device__ __forceinline__ void load(const janus_adamw_tensor& t, int64_t e) {
        k = HOW != SOME ? 4 : int(min(max(t.size - e, int64_t(0)), int64_t(4)));
        load4<HOW>(t.g + e, k, g);
        if (t.master) load4<HOW>(t.master + e, k, p);
        else load4<HOW>(static_cast<const T*>(t.p) + e, k, p);
        if constexpr (Q) {
            mc = load_codes<HOW>(static_cast<const uint8_t*>(t.m) + e, k);
            vc = load_codes<HOW>(static_cast<const uint8_t*>(t.v) + e, k);
            scale = *reinterpret_cast<const float2*>(t.scale + e / 256 * 2);
        } else {
            load4<HOW>(static_cast<const float*>(t.m) + e, k, m);
            load4<HOW>(static_cast<const float*>(t.v) + e, k, v);
        }
    }
    template <How HOW>
    __device__ __forceinline__ void finish(const janus_adamw_tensor& t, int64_t e, const Step& st, uint32_t key) {
        float r[4];
        if constexpr (Q) {
            decode(mc, scale.x, m);
            decode(vc, scale.y, v);
            uint32_t rm[4], rv[4];
            float least[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                least[j] = v[j] == 0.f ? st.least * scale.y : 0.f;
                v[j] = v[j] * v[j];
                st.moments(g[j], m[j], v[j]);
                r[j] = root_of(v[j]);
                const uint32_t x = mix(uint32_t(e + j) ^ key);
                rm[j] = x & 0xffffu, rv[j] = x >> 16;
            }
            float2 s;
            const uint32_t cm = encode(m, rm, s.x), cv = encode(r, rv, s.y);
            store_codes<HOW>(static_cast<uint8_t*>(t.m) + e, k, cm);
            store_codes<HOW>(static_cast<uint8_t*>(t.v) + e, k, cv);
            if ((threadIdx.x & 63) == 0) *reinterpret_cast<float2*>(t.scale + e / 256 * 2) = s;
#pragma unroll
            for (int j = 0; j < 4; ++j) r[j] = r[j] < least[j] ? least[j] : r[j];   // (a NaN stays)
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                st.moments(g[j], m[j], v[j]);
                r[j] = near_root(v[j]);
            }
            store4<HOW>(static_cast<float*>(t.m) + e, k, m);
            store4<HOW>(static_cast<float*>(t.v) + e, k, v);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) p[j] = st.parameter(p[j], m[j], r[j]);
        if (t.master) store4<HOW>(t.master + e, k, p);
        store4<HOW>(static_cast<T*>(t.p) + e, k, p);
    }
};

// A tile; form() gives the step, and false when nothing may change: after the tile's first loads
// went out.  PAST: the tile is whole, and so are its accesses.
template <typename T, bool Q, How HOW, int TILE, typename F>
__device__ __forceinline__ bool adamw_tile(const janus_adamw_tensor& t, int64_t at, F form) {
    constexpr int U = TILE / 4 / kThreads, W = U < 2 ? U : 2;
    Step st{};
    uint32_t key = 0;
#pragma unroll 1
    for (int u = 0; u < U; u += W) {
        Four<T, Q> x[W];
        int64_t e[W], end[W];   // end: of the wave's 256 elements
#pragma unroll
        for (int w = 0; w < W; ++w) {
            e[w] = at + int64_t(threadIdx.x + (u + w) * kThreads) * 4, end[w] = (e[w] & ~int64_t(255)) + 256;
            if (HOW == PAST) x[w].template load<PAST>(t, e[w]);
            else if (end[w] <= t.size) x[w].template load<ALL>(t, e[w]);
            else if (end[w] - 256 < t.size) x[w].template load<SOME>(t, e[w]);
        }
        if (u == 0 && !form(st, key)) return false;
#pragma unroll
        for (int w = 0; w < W; ++w) {
            if (HOW == PAST) x[w].template finish<PAST>(t, e[w], st, key);
            else if (end[w] <= t.size) x[w].template finish<ALL>(t, e[w], st, key);
            else if (end[w] - 256 < t.size) x[w].template finish<SOME>(t, e[w], st, key);
        }
    }
    return true;
}

template <bool Q, int TILE, typename Table>
__global__ __launch_bounds__(kThreads) void adamw_update_kernel(Table t, AdamArgs a) {
    __shared__ int64_t lds[kStarts + 1];
    prepare(t, lds);
    Step st;
    Control c;
    bool formed = false, go = false;
    for (int64_t tile = start(t, lds, t.n) - 1 - blockIdx.x; tile >= 0 || !formed; tile -= gridDim.x) {
        if (tile < 0) {   // (nothing to do but to say so)
            form_step(a, st, c, blockIdx.x == 0);
            return;
        }
        const int i = tensor_of(t, lds, tile);
        const janus_adamw_tensor x = t.t[i];
        auto form = [&](Step& s, uint32_t& key) {
            if (!formed) go = form_step(a, st, c, blockIdx.x == 0);
            formed = true;
            st.shrink = c.lr * x.decay;
            key = mix(c.key ^ uint32_t(i));
            s = st;
            return go;
        };
        const int64_t at = (tile - start(t, lds, i)) * TILE;
        const bool there = at + TILE <= x.size;
        const bool done = x.dtype == JANUS_BF16 ? (there && even<bf16_t, Q>(x) ? adamw_tile<bf16_t, Q, PAST, TILE>(x, at, form)
                                                                      : adamw_tile<bf16_t, Q, SOME, TILE>(x, at, form))
                                                : (there && even<float, Q>(x) ? adamw_tile<float, Q, PAST, TILE>(x, at, form)
                                                                     : adamw_tile<float, Q, SOME, TILE>(x, at, form));
        if (!done) return;
    }
}

size_t adamw_carve(AdamArgs& a, Tensors& t, int n, void* ws) {
    Carver c(ws);
    a.ctl = c.take<Control>(1);
    a.sums = c.take<double>(kBlocks);
    t.n = n;
    if (n > kTable) t.tile = c.take<int64_t>(n + 1), t.t = c.take<janus_adamw_tensor>(n);
    return c.off;
}

// Calls of up to this many elements are cut in tiles of 1024, for there to be more of them.
// With tiles of 1024 and of 4096: 2^18 elements 8.0 and 9.4 us (8-bit states 8.5 and 12.7),
// 2^21 16.6 and 16.7 (16.7 and 15.5), 2^22 29.6 and 26.5 (26.3 and 22.2).
constexpr int64_t kSmallTotal = 1 << 21;

// The two passes, over a table by value or in the workspace
template <bool Q, typename Table>
janus_status adamw_run(const Table& t, const AdamArgs& a, bool small, double total, double bytes, hipStream_t st) {
    const dim3 blocks(a.n_sums), threads(kThreads);
    {
        TraceScope trace("adamw_norm", 2.0 * total, 4.0 * total, st);
        if (small) hipLaunchKernelGGL((adamw_norm_kernel<1024, Table>), blocks, threads, 0, st, t, a);
        else hipLaunchKernelGGL((adamw_norm_kernel<4096, Table>), blocks, threads, 0, st, t, a);
        JANUS_LAUNCH_CHECK();
    }
    TraceScope trace("adamw_update", 16.0 * total, bytes, st);
    if (small) hipLaunchKernelGGL((adamw_update_kernel<Q, 1024, Table>), blocks, threads, 0, st, t, a);
    else hipLaunchKernelGGL((adamw_update_kernel<Q, 4096, Table>), blocks, threads, 0, st, t, a);
    JANUS_LAUNCH_CHECK();
    return JANUS_OK;
}

bool adamw_desc_ok(const janus_adamw_desc* d) {
    return d && d->n >= 1 && std::isfinite(d->lr) && d->beta1 >= 0.f && d->beta1 < 1.f && d->beta2 >= 0.f &&
           d->beta2 < 1.f && std::isfinite(d->eps) && d->eps >= 0x1p-126f && !std::isnan(d->max_norm);
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
    Tensors t;
    return adamw_carve(a, t, d->n, nullptr);
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
    Tensors big;
    const size_t need = adamw_carve(a, big, d->n, ws);
    if (!ws || ws_bytes < need || !aligned(ws, 256)) return JANUS_ERR_WORKSPACE;
    a.b1 = d->beta1, a.b2 = d->beta2;
    a.c1 = float(1.0 - double(d->beta1)), a.c2 = float(1.0 - double(d->beta2));
    a.eps = d->eps, a.max_norm = d->max_norm, a.lr = d->lr, a.seed = d->seed;
    a.least = float(std::sqrt(double(d->beta2)) * 0x1p-9);
    a.step = step, a.lr_dev = lr, a.hold = hold, a.stats = stats;
    hipStream_t st = static_cast<hipStream_t>(stream);
    const bool q = d->states == JANUS_ADAMW_8BIT;
    int64_t total = 0;
    double bytes = 0.0;
    for (int i = 0; i < d->n; ++i) {
        const janus_adamw_tensor& x = tensors[i];
        total += x.size;
        bytes += double(x.size) * (4 + 2 * double(dtype_size(x.dtype)) + (q ? 4 : 16) + (x.master ? 8 : 0));
    }
    const bool small = total <= kSmallTotal;
    const int64_t tile = small ? 1024 : 4096;
    TensorTable t{};
    int64_t tiles = 0;
    for (int i = 0; i < d->n; i += kTable) {
        t.n = std::min(d->n - i, kTable), t.first = i;
        t.tile[0] = tiles;
        for (int k = 0; k < t.n; ++k) {
            t.t[k] = tensors[i + k];
            t.tile[k + 1] = tiles += (t.t[k].size + tile - 1) / tile;
        }
        if (d->n > kTable) {
            TraceScope trace("adamw_table", 0.0, double(sizeof(TensorTable)), st);
            hipLaunchKernelGGL(adamw_table_kernel, dim3(1), dim3(64), 0, st, t, const_cast<int64_t*>(big.tile),
                               const_cast<janus_adamw_tensor*>(big.t));
            JANUS_LAUNCH_CHECK();
        }
    }
    a.n_sums = int(std::max<int64_t>(1, std::min<int64_t>(kBlocks, tiles)));
    if (d->n > kTable) return q ? adamw_run<true>(big, a, small, double(total), bytes, st)
                                : adamw_run<false>(big, a, small, double(total), bytes, st);
    return q ? adamw_run<true>(t, a, small, double(total), bytes, st) : adamw_run<false>(t, a, small, double(total), bytes, st);
}
