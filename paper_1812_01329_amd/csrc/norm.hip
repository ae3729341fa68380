// Layer norm over rows, with the residual sum before it; forward and backward.
//
//   h = x + r,  mu = sum h / D,  rstd = (sum (h - mu)^2 / D + eps)^(-1/2)
//   y = (h - mu) rstd gamma + beta
//   xh = (h - mu) rstd,  g = dy gamma
//   dx = rstd (g - sum g / D - xh sum(g xh) / D) + dh
//   dgamma = sum dy xh,  dbeta = sum dy   (over rows)
//
// A row belongs to a group of 16 to 1024 threads, 8 elements a thread where that
// suffices, and stays in registers from its mean to its result, so every tensor is read
// and written once (up to 16384 elements; float32 in the backward up to 8192: past that
// registers spill, and a row is read again for every pass).  In the backward a thread
// has the same columns in every row it meets and adds up their dgamma and dbeta;
// workgroups' sums go to the workspace, and a second kernel adds them up in their order.
// Everything between loads and stores is float32; the variance is that of the
// differences from the mean (a mean of squares less the square of the mean loses what a
// large mean has in common).
//
// Bound by memory: training 65536 rows of 2048 bf16 with a residual, the forward takes
// 201 us (5.3 TB/s of four tensors) and the backward 215 (5.0 TB/s); 25600 rows of 1024 27
// and 32 us, partly from the last-level cache.  Few rows are bound by latency: 20 rows of
// 1300 take 3.8 us, 1021 of 301 float32 4.2 and 4.9.
#include <cmath>

#include "rows.hpp"

namespace janus {
namespace {

struct NormArgs {
    int32_t rows, D;
    float eps, width;      // D as a float: sums are divided by it (the mean of a constant row is its value)
    int64_t ldx, ldh, ldy;
    const void *x, *r;     // (backward: x is h)
    const float *gamma, *beta;
    void *h, *y;
    float *mean, *rstd;
    const void *dy, *dh;
    void* dx;
    float* part;           // [gridDim.x][2][D] sums of dgamma and dbeta, or NULL
};

constexpr int kThreads = 256;   // of a workgroup, or a row's where that is more

// N sums over the LANES threads of a row (a power of two; above 64 a workgroup's)
template <int LANES, int N>
__device__ __forceinline__ void row_sum(float (&v)[N], float* red) {
    constexpr int W = LANES < 64 ? LANES : 64;
#pragma unroll
    for (int o = W / 2; o > 0; o >>= 1)
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] += __shfl_xor(v[k], o, 64);
    if constexpr (LANES > 64) {
        constexpr int WAVES = LANES / 64;
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, first = threadIdx.x / LANES * WAVES;
        __syncthreads();   // (the sums before have been read)
        if (lane == 0)
#pragma unroll
            for (int k = 0; k < N; ++k) red[wave * N + k] = v[k];
        __syncthreads();
#pragma unroll
        for (int k = 0; k < N; ++k) {
            v[k] = 0.f;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) v[k] += red[(first + w) * N + k];
        }
    }
}

// VEC elements at p.  ODD: wherever they start, and of the last ones only `left` (one at least) are
// there; the others are read as 0, or with SAME as the first of them.
template <typename T, int VEC, bool ODD>
struct Span {
    Chan<T, VEC> c;
    template <bool SAME = false>
    __device__ __forceinline__ void load(const T* p, int left) {
        if constexpr (!ODD) {
            c.load(p);
        } else if (left >= VEC) {
            __builtin_memcpy(&c.v, p, sizeof(c.v));
        } else if constexpr (sizeof(T) == 2) {
            const uint32_t none = SAME ? p[0] : 0;
            c.v = make_uint2(word(p, 0, left, none), word(p, 2, left, none));
        } else {
            const float none = SAME ? p[0] : 0.f;
            c.v = make_float4(p[0], left > 1 ? p[1] : none, left > 2 ? p[2] : none, none);
        }
    }
    __device__ __forceinline__ void get(float* f) const { c.get(f); }
    __device__ __forceinline__ static void store(T* p, const float* f, int left) {
        if constexpr (!ODD) {
            Chan<T, VEC>::store(p, f);
        } else if (left >= VEC) {
            Chan<T, VEC> o;
            if constexpr (sizeof(T) == 2) o.v = make_uint2(pack2(f[0], f[1]), pack2(f[2], f[3]));
            else o.v = make_float4(f[0], f[1], f[2], f[3]);
            __builtin_memcpy(p, &o.v, sizeof(o.v));
        } else {
#pragma unroll
            for (int j = 0; j < VEC; ++j)
                if (j < left) p[j] = out_f<T>(f[j]);
        }
    }

  private:
    __device__ __forceinline__ static uint32_t word(const T* p, int j, int left, uint32_t none) {
        return (j < left ? uint32_t(p[j]) : none) | (j + 1 < left ? uint32_t(p[j + 1]) : none) << 16;
    }
};
template <int VEC, bool ODD>
__device__ __forceinline__ void load_f(const float* p, float* f, int left) {
    constexpr int ONE = VEC < 4 ? 1 : 4;
#pragma unroll
    for (int j = 0; j < VEC; j += ONE) {
        Span<float, ONE, ODD> v;
        v.load(p + j, left);
        v.get(f + j);
    }
}

// LANES threads a row, P accesses of VEC elements each; P = 0: rows longer than that,
// read three times (for the mean, the variance, the result).
template <typename T, int VEC, bool ODD, int LANES, int P>
__global__ __launch_bounds__(LANES > kThreads ? LANES : kThreads) void norm_fwd_kernel(NormArgs a) {
    constexpr int THREADS = LANES > kThreads ? LANES : kThreads, ROWS = THREADS / LANES;
    __shared__ float red[THREADS / 64];
    const int tid = threadIdx.x % LANES;
    const int64_t r0 = int64_t(blockIdx.x) * ROWS + threadIdx.x / LANES;
    const bool there = r0 < a.rows;   // (only rows of less than a workgroup can be missing)
    const int64_t row = there ? r0 : a.rows - 1;
    const T* x = static_cast<const T*>(a.x) + row * a.ldx;
    const T* r = a.r ? static_cast<const T*>(a.r) + row * a.ldh : nullptr;
    T* h = a.h && there ? static_cast<T*>(a.h) + row * a.ldh : nullptr;
    T* y = static_cast<T*>(a.y) + row * a.ldy;
    auto load = [&](int c, float* f) {
        Span<T, VEC, ODD> v;
        v.load(x + c, a.D - c);
        v.get(f);
        if (r) {
            float s[VEC];
            v.load(r + c, a.D - c);
            v.get(s);
#pragma unroll
            for (int j = 0; j < VEC; ++j) f[j] = to_f(out_f<T>(f[j] + s[j]));
        }
    };
    auto result = [&](int c, const float* f, float mean, float rstd) {
        float g[VEC], o[VEC];
#pragma unroll
        for (int j = 0; j < VEC; ++j) o[j] = (f[j] - mean) * rstd;
        if (a.gamma) {
            load_f<VEC, ODD>(a.gamma + c, g, a.D - c);
#pragma unroll
            for (int j = 0; j < VEC; ++j) o[j] *= g[j];
        }
        if (a.beta) {
            load_f<VEC, ODD>(a.beta + c, g, a.D - c);
#pragma unroll
            for (int j = 0; j < VEC; ++j) o[j] += g[j];
        }
        if (there) Span<T, VEC, ODD>::store(y + c, o, a.D - c);
    };
    float s[1] = {0.f}, q[1] = {0.f};
    if constexpr (P > 0) {
        float v[P][VEC];
#pragma unroll
        for (int i = 0; i < P; ++i) {
            const int c = (tid + i * LANES) * VEC;
            if (c < a.D) {
                load(c, v[i]);
            } else {
#pragma unroll
                for (int j = 0; j < VEC; ++j) v[i][j] = 0.f;
            }
        }
#pragma unroll
        for (int i = 0; i < P; ++i)
#pragma unroll
            for (int j = 0; j < VEC; ++j) s[0] += v[i][j];
        row_sum<LANES>(s, red);
        const float mean = s[0] / a.width;
#pragma unroll
        for (int i = 0; i < P; ++i)
            if ((tid + i * LANES) * VEC < a.D)
#pragma unroll
                for (int j = 0; j < VEC; ++j)
                    if (!ODD || (tid + i * LANES) * VEC + j < a.D) q[0] = fmaf(v[i][j] - mean, v[i][j] - mean, q[0]);
        row_sum<LANES>(q, red);
        const float rstd = 1.f / sqrtf(q[0] / a.width + a.eps);
        if (tid == 0 && there) {
            if (a.mean) a.mean[row] = mean;
            if (a.rstd) a.rstd[row] = rstd;
        }
#pragma unroll
        for (int i = 0; i < P; ++i) {
            const int c = (tid + i * LANES) * VEC;
            if (c < a.D) {
                if (h) Span<T, VEC, ODD>::store(h + c, v[i], a.D - c);
                result(c, v[i], mean, rstd);
            }
        }
    } else {
        float v[VEC];
        const int64_t end = a.D;
        for (int64_t c = int64_t(tid) * VEC; c < end; c += LANES * VEC) {
            load(c, v);
#pragma unroll
            for (int j = 0; j < VEC; ++j) s[0] += v[j];
        }
        row_sum<LANES>(s, red);
        const float mean = s[0] / a.width;
        for (int64_t c = int64_t(tid) * VEC; c < end; c += LANES * VEC) {
            load(c, v);
#pragma unroll
            for (int j = 0; j < VEC; ++j)
                if (!ODD || c + j < end) q[0] = fmaf(v[j] - mean, v[j] - mean, q[0]);
        }
        row_sum<LANES>(q, red);
        const float rstd = 1.f / sqrtf(q[0] / a.width + a.eps);
        if (tid == 0) {
            if (a.mean) a.mean[row] = mean;
            if (a.rstd) a.rstd[row] = rstd;
        }
        for (int64_t c = int64_t(tid) * VEC; c < end; c += LANES * VEC) {
            load(c, v);   // (before h is written: h may be r or x)
            if (h) Span<T, VEC, ODD>::store(h + c, v, int(end - c));
            result(c, v, mean, rstd);
        }
    }
}

// As the forward; a workgroup takes every gridDim.x-th group of rows.  65536 rows of 2048
// bf16 take 215 us, a row in 256 threads; with a row in a wave, 32 elements a thread, 305
// (registers leave too few waves).  P = 0: dx alone, by two reads of a row.  Past a row's end dy is
// read as 0 and h as an element of the row: 0 may be further from the mean than float32
// reaches, and 0 * inf would be in the row's sums (elements left out instead: registers
// spilled, 14444 rows of 12001 bf16 4650 us instead of 481).
constexpr int kBwdThreads = 512;   // (the fewer workgroups, the fewer sums of dgamma and dbeta)
template <typename T, int VEC, bool ODD, int LANES, int P>
__global__ __launch_bounds__(LANES > kBwdThreads ? LANES : kBwdThreads) void norm_bwd_kernel(NormArgs a) {
    constexpr int THREADS = LANES > kBwdThreads ? LANES : kBwdThreads, ROWS = THREADS / LANES, E = P * VEC;
    __shared__ float red[2 * THREADS / 64];
    const int tid = threadIdx.x % LANES, at = threadIdx.x / LANES;
    if constexpr (P > 0) {
        float dg[E ? E : 1] = {}, db[E ? E : 1] = {};
        for (int64_t r0 = int64_t(blockIdx.x) * ROWS; r0 < a.rows; r0 += int64_t(gridDim.x) * ROWS) {
            const bool there = r0 + at < a.rows;
            const int64_t row = there ? r0 + at : a.rows - 1;
            const T* h = static_cast<const T*>(a.x) + row * a.ldh;
            const T* dy = static_cast<const T*>(a.dy) + row * a.ldy;
            const float mean = a.mean[row], rstd = a.rstd[row];
            Span<T, VEC, ODD> hv[P], dv[P];
#pragma unroll
            for (int i = 0; i < P; ++i) {
                const int c = (tid + i * LANES) * VEC;
                if (c < a.D) hv[i].template load<true>(h + c, a.D - c), dv[i].load(dy + c, a.D - c);
            }
            float xh[P][VEC], g[P][VEC], s[2] = {0.f, 0.f};
#pragma unroll
            for (int i = 0; i < P; ++i) {
                const int c = (tid + i * LANES) * VEC;
                if (c < a.D) {
                    hv[i].get(xh[i]);
                    dv[i].get(g[i]);
                    float w[VEC];
                    if (a.gamma) load_f<VEC, ODD>(a.gamma + c, w, a.D - c);
#pragma unroll
                    for (int j = 0; j < VEC; ++j) {
                        xh[i][j] = (xh[i][j] - mean) * rstd;
                        if (there) {
                            dg[i * VEC + j] = fmaf(g[i][j], xh[i][j], dg[i * VEC + j]);
                            db[i * VEC + j] += g[i][j];
                        }
                        if (a.gamma) g[i][j] *= w[j];
                        s[0] += g[i][j];
                        s[1] = fmaf(g[i][j], xh[i][j], s[1]);
                    }
                }
            }
            row_sum<LANES>(s, red);
            if (!a.dx || !there) continue;
            const float m0 = s[0] / a.width, m1 = s[1] / a.width;
            T* dx = static_cast<T*>(a.dx) + row * a.ldx;
            const T* dh = a.dh ? static_cast<const T*>(a.dh) + row * a.ldh : nullptr;
#pragma unroll
            for (int i = 0; i < P; ++i) {
                const int c = (tid + i * LANES) * VEC;
                if (c < a.D) {
                    float o[VEC];
#pragma unroll
                    for (int j = 0; j < VEC; ++j) o[j] = (g[i][j] - m0 - xh[i][j] * m1) * rstd;
                    if (dh) {
                        Span<T, VEC, ODD> e;
                        float f[VEC];
                        e.load(dh + c, a.D - c);
                        e.get(f);
#pragma unroll
                        for (int j = 0; j < VEC; ++j) o[j] += f[j];
                    }
                    Span<T, VEC, ODD>::store(dx + c, o, a.D - c);
                }
            }
        }
        if (!a.part) return;
        // the workgroup's groups of lanes together
        float* to = a.part + int64_t(blockIdx.x) * 2 * a.D;
        if constexpr (ROWS == 1) {
#pragma unroll
            for (int i = 0; i < P; ++i)
#pragma unroll
                for (int j = 0; j < VEC; ++j) {
                    const int c = (tid + i * LANES) * VEC + j;
                    if (c < a.D) to[c] = dg[i * VEC + j], to[a.D + c] = db[i * VEC + j];
                }
        } else {
            __shared__ float sums[THREADS * E];
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                __syncthreads();
#pragma unroll
                for (int e = 0; e < E; ++e) sums[(at * E + e) * LANES + tid] = k ? db[e] : dg[e];
                __syncthreads();
                for (int t = threadIdx.x; t < LANES * E; t += THREADS) {
                    const int e = t / LANES, c = (t % LANES + (e / VEC) * LANES) * VEC + e % VEC;
                    float v = 0.f;
#pragma unroll 8
                    for (int n = 0; n < ROWS; ++n) v += sums[n * LANES * E + t];
                    if (c < a.D) to[k * a.D + c] = v;
                }
            }
        }
    } else {
        const int64_t row = blockIdx.x, end = a.D;
        const T* h = static_cast<const T*>(a.x) + row * a.ldh;
        const T* dy = static_cast<const T*>(a.dy) + row * a.ldy;
        T* dx = static_cast<T*>(a.dx) + row * a.ldx;
        const T* dh = a.dh ? static_cast<const T*>(a.dh) + row * a.ldh : nullptr;
        const float mean = a.mean[row], rstd = a.rstd[row];
        float xh[VEC], g[VEC], s[2] = {0.f, 0.f};
        auto load = [&](int64_t c) {
            Span<T, VEC, ODD> v;
            const int left = int(end - c);
            v.template load<true>(h + c, left);
            v.get(xh);
            v.load(dy + c, left);
            v.get(g);
#pragma unroll
            for (int j = 0; j < VEC; ++j) xh[j] = (xh[j] - mean) * rstd;
            if (a.gamma) {
                float w[VEC];
                load_f<VEC, ODD>(a.gamma + c, w, left);
#pragma unroll
                for (int j = 0; j < VEC; ++j) g[j] *= w[j];
            }
        };
        for (int64_t c = int64_t(tid) * VEC; c < end; c += LANES * VEC) {
            load(c);
#pragma unroll
            for (int j = 0; j < VEC; ++j) s[0] += g[j], s[1] = fmaf(g[j], xh[j], s[1]);
        }
        row_sum<LANES>(s, red);
        const float m0 = s[0] / a.width, m1 = s[1] / a.width;
        for (int64_t c = int64_t(tid) * VEC; c < end; c += LANES * VEC) {
            load(c);
            float o[VEC];
#pragma unroll
            for (int j = 0; j < VEC; ++j) o[j] = (g[j] - m0 - xh[j] * m1) * rstd;
            if (dh) {
                Span<T, VEC, ODD> e;
                float f[VEC];
                e.load(dh + c, int(end - c));
                e.get(f);
#pragma unroll
                for (int j = 0; j < VEC; ++j) o[j] += f[j];
            }
            Span<T, VEC, ODD>::store(dx + c, o, int(end - c));
        }
    }
}

// dgamma and dbeta of rows longer than registers hold: a thread has a column, a
// workgroup (blockIdx.y) every gridDim.y-th row.
template <typename T>
__global__ __launch_bounds__(kThreads) void norm_cols_kernel(NormArgs a) {
    const int64_t c = int64_t(blockIdx.x) * kThreads + threadIdx.x;
    if (c >= a.D) return;
    float dg = 0.f, db = 0.f;
    for (int64_t row = blockIdx.y; row < a.rows; row += gridDim.y) {
        const float h = to_f(static_cast<const T*>(a.x)[row * a.ldh + c]);
        const float g = to_f(static_cast<const T*>(a.dy)[row * a.ldy + c]);
        dg = fmaf(g, (h - a.mean[row]) * a.rstd[row], dg);
        db += g;
    }
    float* to = a.part + int64_t(blockIdx.y) * 2 * a.D;
    to[c] = dg;
    to[a.D + c] = db;
}

// The workgroups' sums, added up: 64 columns of dgamma or dbeta a workgroup, four of
// them and every 64th sum a thread.  512 sums of 2048 columns take 4.2 us, 1024 of them 23
// and 2048 48: why the backward has 512 workgroups at most.
__global__ __launch_bounds__(1024) void norm_sum_kernel(const float* part, int n, int D, float* dgamma, float* dbeta) {
    __shared__ float4 red[64][16];
    const int col = threadIdx.x & 15, from = threadIdx.x >> 4;
    const int64_t width = 2 * int64_t(D), c = int64_t(blockIdx.x) * 64 + 4 * col;
    float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
    if (D % 4 == 0) {
        if (c < width) {
#pragma unroll 4
            for (int k = from; k < n; k += 64) {
                const float4 v = *reinterpret_cast<const float4*>(part + k * width + c);
                s.x += v.x, s.y += v.y, s.z += v.z, s.w += v.w;
            }
        }
    } else {
        float f[4] = {};
        for (int k = from; k < n; k += 64)
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (c + j < width) f[j] += part[k * width + c + j];
        s = make_float4(f[0], f[1], f[2], f[3]);
    }
    red[from][col] = s;
    __syncthreads();
    // a wave a quarter of the columns, 16 of the 64 sums a lane
    if (threadIdx.x >= 256) return;
    const int at = threadIdx.x >> 2;   // the column
    float v = 0.f;
#pragma unroll
    for (int k = 0; k < 16; ++k) v += reinterpret_cast<const float*>(&red[(threadIdx.x & 3) * 16 + k][at >> 2])[at & 3];
    v += __shfl_xor(v, 1, 64);
    v += __shfl_xor(v, 2, 64);
    const int64_t to = int64_t(blockIdx.x) * 64 + at;
    if ((threadIdx.x & 3) || to >= width) return;
    if (to < D) {
        if (dgamma) dgamma[to] = v;
    } else if (dbeta) {
        dbeta[to - D] = v;
    }
}
__global__ __launch_bounds__(kThreads) void norm_zero_kernel(float* dgamma, float* dbeta, int D) {
    const int64_t c = int64_t(blockIdx.x) * kThreads + threadIdx.x;
    if (c >= D) return;
    if (dgamma) dgamma[c] = 0.f;
    if (dbeta) dbeta[c] = 0.f;
}

// A backward of at most this many workgroups: two of 512 threads on each CU.
constexpr int kNormBlocks = 512;
// Rows of more elements than this never fit the registers (16 elements a thread).
constexpr int kMostHeld = 1024 * 16;

// Workgroups of norm_cols_kernel over the rows
int cols_parts(int32_t rows, int32_t D) {
    const int64_t cols = (int64_t(D) + kThreads - 1) / kThreads;
    return int(std::max<int64_t>(1, std::min<int64_t>({rows, kNormBlocks, 8192 / cols})));
}
// Sums of dgamma and dbeta in the workspace, at most
int norm_parts(const janus_norm_desc* d) {
    return d->D > kMostHeld ? std::min(d->rows, cols_parts(d->rows, d->D)) : std::min(d->rows, kNormBlocks);
}
size_t norm_ws_bytes(const janus_norm_desc* d) { return size_t(norm_parts(d)) * 2 * size_t(d->D) * sizeof(float); }

bool norm_desc_ok(const janus_norm_desc* d) {
    auto stride = [&](int64_t ld) { return ld == 0 || ld >= d->D; };
    return d && d->rows >= 0 && d->D > 0 && stride(d->ldx) && stride(d->ldh) && stride(d->ldy) &&
           std::isfinite(d->eps) && d->eps >= 0.f;
}
bool norm_built(const janus_norm_desc* d) {
    return dtype_ok(d->dtype) && d->rows <= (1 << 30) && d->D <= (1 << 24);
}

NormArgs norm_args(const janus_norm_desc* d) {
    NormArgs a{};
    a.rows = d->rows, a.D = d->D, a.eps = d->eps, a.width = float(d->D);
    a.ldx = d->ldx ? d->ldx : d->D, a.ldh = d->ldh ? d->ldh : d->D, a.ldy = d->ldy ? d->ldy : d->D;
    return a;
}

// Elements an aligned access: the most that rows' starts and ends allow.
// Where that is fewer than four, the forward takes four wherever they start (ODD): 14444 rows of
// 1409 bf16 27 us, by single elements 64; of 5946, by pairs, 144 and 165; of 1409 float32 34 and 37.
// The backward does so for single bf16 alone (14444 rows of 12001: 484 us, by single elements 935).
// Rows of 5946 bf16 take 188 us by pairs and 208 by four from anywhere, of 5946 float32 267 by
// single elements (no multiple of four) and 299 by four from anywhere.
int norm_vec(const NormArgs& a, size_t es, std::initializer_list<const void*> rows, std::initializer_list<int64_t> lds) {
    int vec = int(16 / es);
    for (; vec > 1; vec /= 2) {
        if (es == 4 && vec == 2) continue;
        bool ok = a.D % vec == 0 && aligned(a.gamma, vec >= 4 ? 16 : 4) && aligned(a.beta, vec >= 4 ? 16 : 4);
        for (const void* p : rows) ok = ok && aligned(p, vec * es);
        for (int64_t ld : lds) ok = ok && (ld % vec == 0);
        if (ok) break;
    }
    return vec;
}

// A launch holds fewer than 2^32 threads: more rows take several.
template <typename T, int VEC, bool ODD, int LANES, int P>
void fwd_launch(NormArgs a, hipStream_t st) {
    constexpr int THREADS = LANES > kThreads ? LANES : kThreads, ROWS = THREADS / LANES;
    constexpr int64_t kMost = int64_t((1 << 30) / THREADS) * ROWS;
    const int64_t rows = a.rows, es = sizeof(T);
    for (int64_t r0 = 0; r0 < rows; r0 += kMost) {
        NormArgs b = a;
        b.rows = int32_t(std::min(kMost, rows - r0));
        auto on = [&](const void* p, int64_t ld) { return p ? static_cast<const char*>(p) + r0 * ld * es : nullptr; };
        b.x = on(a.x, a.ldx), b.r = on(a.r, a.ldh), b.h = const_cast<char*>(on(a.h, a.ldh));
        b.y = const_cast<char*>(on(a.y, a.ldy));
        if (a.mean) b.mean = a.mean + r0;
        if (a.rstd) b.rstd = a.rstd + r0;
        hipLaunchKernelGGL((norm_fwd_kernel<T, VEC, ODD, LANES, P>), dim3(unsigned((b.rows + ROWS - 1) / ROWS)), dim3(THREADS), 0,
                           st, b);
    }
}
template <typename T, int VEC, bool ODD, int LANES, int P, int... MORE>
bool fwd_lanes(const NormArgs& a, int64_t n, hipStream_t st) {
    if (n <= LANES * P) {
        fwd_launch<T, VEC, ODD, LANES, P>(a, st);
        return true;
    }
    if constexpr (sizeof...(MORE) > 0) return fwd_lanes<T, VEC, ODD, LANES, MORE...>(a, n, st);
    else return false;
}
// From this many rows on a forward gives a bf16 row of up to 2048 elements a wave, which waits for no
// other one: 65536 rows of 2048 with a residual 204 us, in workgroups 216 (float32 rows hold twice the
// registers: 25600 of 2048 81 and 73 us).  Fewer rows leave the chip idle that way: 20 rows of 1300
// take 3.9 us in workgroups of 256, and 5.1.
constexpr int kWaveRows = 4096;
template <typename T, int VEC, bool ODD>
void fwd_vec(const NormArgs& a, hipStream_t st) {
    const int64_t n = (int64_t(a.D) + VEC - 1) / VEC;   // accesses a row
    constexpr int P = 8 / VEC;
    if (fwd_lanes<T, VEC, ODD, 16, P>(a, n, st)) return;
    if constexpr (sizeof(T) == 2)
        if (a.rows >= kWaveRows && fwd_lanes<T, VEC, ODD, 64, P, 2 * P, 4 * P>(a, n, st)) return;
    if (fwd_lanes<T, VEC, ODD, 64, P>(a, n, st) || fwd_lanes<T, VEC, ODD, 128, P>(a, n, st) ||
        fwd_lanes<T, VEC, ODD, 256, P>(a, n, st) || fwd_lanes<T, VEC, ODD, 512, P>(a, n, st) ||
        fwd_lanes<T, VEC, ODD, 1024, P, 2 * P>(a, n, st))
        return;
    fwd_launch<T, VEC, ODD, 1024, 0>(a, st);
}

template <typename T, int VEC, bool ODD, int LANES, int P>
int bwd_launch(const NormArgs& a, hipStream_t st) {
    constexpr int THREADS = LANES > kBwdThreads ? LANES : kBwdThreads, ROWS = THREADS / LANES;
    // A workgroup's sums cost as much as three or four rows, but few rows spread over the
    // CUs gain more: 64 at least instead of 256 takes 11.2 us instead of 9.9 for 1500 rows of
    // 301 float32 and 13.9 instead of 12.9 for 1500 of 2048 bf16.
    const int64_t groups = (int64_t(a.rows) + ROWS - 1) / ROWS;
    const int blocks = int(std::min<int64_t>(groups, std::min<int64_t>(std::max<int64_t>(256, groups / 4), kNormBlocks)));
    hipLaunchKernelGGL((norm_bwd_kernel<T, VEC, ODD, LANES, P>), dim3(blocks), dim3(THREADS), 0, st, a);
    return blocks;
}
template <typename T, int VEC, bool ODD, int LANES, int P, int... MORE>
int bwd_lanes(const NormArgs& a, int64_t n, hipStream_t st) {
    if (n <= LANES * P) return bwd_launch<T, VEC, ODD, LANES, P>(a, st);
    if constexpr (sizeof...(MORE) > 0) return bwd_lanes<T, VEC, ODD, LANES, MORE...>(a, n, st);
    else return 0;
}
// Launches the pass over the rows; returns the number of its sums in a.part.
template <typename T, int VEC, bool ODD>
int bwd_vec(NormArgs a, hipStream_t st) {
    const int64_t n = (int64_t(a.D) + VEC - 1) / VEC;
    int k;
    constexpr int P = 8 / VEC;
    if ((k = bwd_lanes<T, VEC, ODD, 16, P>(a, n, st))) return k;
    if ((k = bwd_lanes<T, VEC, ODD, 64, P>(a, n, st))) return k;
    if ((k = bwd_lanes<T, VEC, ODD, 128, P>(a, n, st))) return k;
    if ((k = bwd_lanes<T, VEC, ODD, 256, P>(a, n, st))) return k;
    if ((k = bwd_lanes<T, VEC, ODD, 512, P>(a, n, st))) return k;
    if ((k = bwd_lanes<T, VEC, ODD, 1024, P>(a, n, st))) return k;
    if constexpr (sizeof(T) == 2)   // (float32: 404 registers spilled)
        if ((k = bwd_lanes<T, VEC, ODD, 1024, 2 * P>(a, n, st))) return k;
    if (a.dx) {   // (a launch holds fewer than 2^32 threads)
        constexpr int64_t kMost = (1 << 30) / 1024;
        const int64_t rows = a.rows, es = sizeof(T);
        for (int64_t r0 = 0; r0 < rows; r0 += kMost) {
            NormArgs b = a;
            b.rows = int32_t(std::min(kMost, rows - r0));
            b.x = static_cast<const char*>(a.x) + r0 * a.ldh * es, b.dy = static_cast<const char*>(a.dy) + r0 * a.ldy * es;
            if (a.dh) b.dh = static_cast<const char*>(a.dh) + r0 * a.ldh * es;
            b.dx = static_cast<char*>(a.dx) + r0 * a.ldx * es;
            b.mean = a.mean + r0, b.rstd = a.rstd + r0;
            hipLaunchKernelGGL((norm_bwd_kernel<T, VEC, ODD, 1024, 0>), dim3(unsigned(b.rows)), dim3(1024), 0, st, b);
        }
    }
    if (!a.part) return 0;
    const int parts = cols_parts(a.rows, a.D);
    hipLaunchKernelGGL(norm_cols_kernel<T>, dim3((a.D + kThreads - 1) / kThreads, parts), dim3(kThreads), 0, st, a);
    return parts;
}

}  // namespace
}  // namespace janus

using namespace janus;

extern "C" size_t janus_layer_norm_workspace_bytes(const janus_norm_desc* d) {
    return norm_desc_ok(d) && norm_built(d) ? norm_ws_bytes(d) : 0;
}

extern "C" janus_status janus_layer_norm_fwd(const janus_norm_desc* d, const void* x, const void* r,
                                             const float* gamma, const float* beta, void* h, void* y, float* mean,
                                             float* rstd, void* stream) {
    if (!norm_desc_ok(d) || (d->rows > 0 && (!x || !y)) || (h && !r)) return JANUS_ERR_INVALID_ARG;
    if (!norm_built(d)) return JANUS_ERR_UNSUPPORTED;
    const size_t es = dtype_size(d->dtype);
    for (const void* p : {x, r, static_cast<const void*>(h), static_cast<const void*>(y)})
        if (!aligned(p, es)) return JANUS_ERR_INVALID_ARG;
    for (const float* p : {gamma, beta, static_cast<const float*>(mean), static_cast<const float*>(rstd)})
        if (!aligned(p, 4)) return JANUS_ERR_INVALID_ARG;
    NormArgs a = norm_args(d);
    if (y && (y == x || y == r || y == h)) return JANUS_ERR_INVALID_ARG;
    if (h && h == x && a.ldh != a.ldx) return JANUS_ERR_INVALID_ARG;
    if (d->rows == 0) return JANUS_OK;
    a.x = x, a.r = r, a.gamma = gamma, a.beta = beta, a.h = h, a.y = y, a.mean = mean, a.rstd = rstd;
    const int vec = norm_vec(a, es, {x, r, h, y}, {a.ldx, r ? a.ldh : 0, a.ldy});
    hipStream_t st = static_cast<hipStream_t>(stream);
    const double el = double(d->rows) * d->D;
    TraceScope trace("norm_fwd", 8.0 * el, el * es * (2 + (r ? 1 : 0) + (h ? 1 : 0)), st);
    if (d->dtype == JANUS_BF16) {
        if (vec == 8) fwd_vec<bf16_t, 8, false>(a, st);
        else if (vec == 4) fwd_vec<bf16_t, 4, false>(a, st);
        else fwd_vec<bf16_t, 4, true>(a, st);
    } else if (vec == 4) {
        fwd_vec<float, 4, false>(a, st);
    } else {
        fwd_vec<float, 4, true>(a, st);
    }
    JANUS_LAUNCH_CHECK();
    return JANUS_OK;
}

extern "C" janus_status janus_layer_norm_bwd(const janus_norm_desc* d, const void* h, const float* gamma,
                                             const float* mean, const float* rstd, const void* dy, const void* dh,
                                             void* dx, float* dgamma, float* dbeta, void* ws, size_t ws_bytes,
                                             void* stream) {
    if (!norm_desc_ok(d) || (d->rows > 0 && (!h || !mean || !rstd || !dy))) return JANUS_ERR_INVALID_ARG;
    if (!norm_built(d)) return JANUS_ERR_UNSUPPORTED;
    const size_t es = dtype_size(d->dtype);
    for (const void* p : {h, dy, dh, static_cast<const void*>(dx)})
        if (!aligned(p, es)) return JANUS_ERR_INVALID_ARG;
    for (const float* p : {gamma, mean, rstd, static_cast<const float*>(dgamma), static_cast<const float*>(dbeta)})
        if (!aligned(p, 4)) return JANUS_ERR_INVALID_ARG;
    NormArgs a = norm_args(d);
    if (dx && (dx == h || dx == dy || (dx == dh && a.ldh != a.ldx))) return JANUS_ERR_INVALID_ARG;
    const bool sums = dgamma || dbeta;
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (d->rows == 0) {
        if (!sums) return JANUS_OK;
        TraceScope trace("norm_zero", 0.0, 8.0 * d->D, st);
        hipLaunchKernelGGL(norm_zero_kernel, dim3((d->D + kThreads - 1) / kThreads), dim3(kThreads), 0, st, dgamma,
                           dbeta, d->D);
        JANUS_LAUNCH_CHECK();
        return JANUS_OK;
    }
    if (sums && (!ws || ws_bytes < norm_ws_bytes(d) || !aligned(ws, 256))) return JANUS_ERR_WORKSPACE;
    if (!sums && !dx) return JANUS_OK;
    a.x = h, a.gamma = gamma, a.mean = const_cast<float*>(mean), a.rstd = const_cast<float*>(rstd);
    a.dy = dy, a.dh = dx ? dh : nullptr, a.dx = dx, a.part = sums ? static_cast<float*>(ws) : nullptr;
    const int vec = norm_vec(a, es, {h, dy, a.dh, dx}, {a.ldh, a.ldy, dx ? a.ldx : 0});
    int parts = 0;
    {
        const double el = double(d->rows) * d->D;
        TraceScope trace("norm_bwd", 14.0 * el, el * es * (2 + (a.dh ? 1 : 0) + (dx ? 1 : 0)), st);
        if (d->dtype == JANUS_BF16) {
            if (vec == 8) parts = bwd_vec<bf16_t, 8, false>(a, st);
            else if (vec == 4) parts = bwd_vec<bf16_t, 4, false>(a, st);
            else if (vec == 2) parts = bwd_vec<bf16_t, 2, false>(a, st);
            else parts = bwd_vec<bf16_t, 4, true>(a, st);
        } else if (vec == 4) {
            parts = bwd_vec<float, 4, false>(a, st);
        } else {
            parts = bwd_vec<float, 1, false>(a, st);
        }
        JANUS_LAUNCH_CHECK();
    }
    if (sums) {
        TraceScope trace("norm_sum", 2.0 * parts * d->D, 8.0 * parts * double(d->D), st);
        hipLaunchKernelGGL(norm_sum_kernel, dim3(unsigned((2 * int64_t(d->D) + 63) / 64)), dim3(1024), 0, st,
                           static_cast<const float*>(ws), parts, d->D, dgamma, dbeta);
        JANUS_LAUNCH_CHECK();
    }
    return JANUS_OK;
}
