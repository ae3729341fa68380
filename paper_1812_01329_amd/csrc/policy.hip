// Clipped policy loss from logits: rows' log-probabilities and entropies, the
// loss with its KL and entropy terms, and the gradient of the logits.
//
//   M = max x,  t = (x - M) log2(e),  S = sum 2^t,  E = sum t 2^t
//   l = (t[a] - log2 S) ln 2,   H = (log2 S - E / S) ln 2,   p_j = 2^t_j / S
//   row  = -min(r adv, clip(r) adv) + beta (exp(u) - 1 - u) - eta H,   r = exp(l - old), u = ref - l
//   c    = d row / d l = -r adv [r adv <= clip(r) adv] - beta (exp(u) - 1)
//   dx_j = w / W (c (1[j = a] - p_j) + eta p_j (log p_j + H)),   W = sum w
//
// One workgroup a row, which it holds in registers from the maximum to the
// gradient, so the logits are read once and the gradient written once; rows
// past 65533 float32 or 131065 bf16 are read three times (16384 pieces of 16 bytes,
// one of them for a row that starts inside one).  Bound by memory: 16384 rows
// of 32768 bf16 logits 416 us (2.15 GB: 5.2 TB/s; a large copy reaches 4.8);
// workgroups of 1024 threads, one a CU, took 860.  700 rows of 10000: 12 us, of
// which 6 are bytes.  2^28 logits in all, gradient and scoring: 4.9 and 5.7 TB/s in
// rows of 65528 bf16, but 3.5 and 2.9 of 65536 (1024 threads a row from there on),
// 3.0 and 2.8 of 131072 (read three times); float32 5.2 and 4.4 in rows of 32768,
// 5.0 and 5.1 of 65528, 3.0 and 3.5 of 131072.  Sums are float32 (float64 over the
// rows) in a fixed order.
#include <cmath>
#include <type_traits>

#include "seq.hpp"

namespace janus {
namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kFarBelow = -200.f;   // exp is 0 there: keeps 0 * -inf out of the sums

struct PolicyArgs {
    int32_t rows, V;
    int32_t row0;         // first row of the launch
    int64_t ld;
    const void* logits;
    const int32_t* actions;
    const float *old_logp, *adv, *ref, *weights;
    void* dlogits;        // NULL: scoring
    float *logp, *entropy;
    float* W;             // sum of the weights that count
    bool own_W;           // the rows' workgroups form it
    float4* terms;        // [rows] weighted first term, KL, H, clipped
    float lo, hi, beta, eta;
};

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

// A product that stays rounded: contracted into the sum it goes into, c w / W
// would leave its rounding error where the gradient is 0 (p = 1 at the action)
__device__ __forceinline__ float rounded_mul(float a, float b) {
#pragma clang fp contract(off)
    return a * b;
}

// exp(u) - 1 - u without the cancellation near 0 (infinite for an infinite u, also a positive one)
__device__ __forceinline__ float kl_term(float u) {
    if (fabsf(u) < 0.5f)
        return u * u *
               (0.5f + u * (1.f / 6 + u * (1.f / 24 + u * (1.f / 120 + u * (1.f / 720 + u * (1.f / 5040 + u / 40320))))));
    const float v = expm1f(u);
    return v == INFINITY ? v : v - u;
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

// S = sum 2^t and E = sum t 2^t
struct Soft {
    float s = 0.f, e = 0.f;
    __device__ __forceinline__ void add(float t) {
        const float v = __builtin_amdgcn_exp2f(t);
        s += v;
        e = fmaf(v, fmaxf(t, kFarBelow), e);   // (0 * -inf for a forbidden action)
    }
};

// A thread's share of the weights that count, eight rows' loads at once
template <int THREADS, typename S>
__device__ __forceinline__ S part_of_weights(const PolicyArgs& a) {
    constexpr int U = 8;
    S s = 0;
    for (int r0 = threadIdx.x; r0 < a.rows; r0 += U * THREADS) {
        int act[U];
        float w[U];
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const int r = min(r0 + i * THREADS, a.rows - 1);
            act[i] = a.actions[r];
            w[i] = a.weights ? a.weights[r] : 1.f;
        }
#pragma unroll
        for (int i = 0; i < U; ++i)
            if (r0 + i * THREADS < a.rows && act[i] >= 0) s += w[i];
    }
    return s;
}

// N sums over a workgroup of 1024, in thread 0
template <int N>
__device__ __forceinline__ void sum_up(double (&s)[N]) {
    __shared__ double red[N][16];
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int k = 0; k < N; ++k) {
        s[k] = wsum(s[k]);
        if (lane == 0) red[k][threadIdx.x >> 6] = s[k];
    }
    __syncthreads();
    if (threadIdx.x >= 64) return;
#pragma unroll
    for (int k = 0; k < N; ++k) {
        s[k] = red[k][lane & 15];
#pragma unroll
        for (int o = 8; o > 0; o >>= 1) s[k] += __shfl_xor(s[k], o, 64);
    }
}

// One workgroup a row.  PIECES 16-byte pieces of the row a thread holds; 0: the row is
// read three times (for its maximum, the sums, the gradient).
template <typename T, int PIECES, int THREADS>
__global__ __launch_bounds__(THREADS, 4) void policy_row_kernel(PolicyArgs a) {
    constexpr int VEC = 16 / sizeof(T), WAVES = THREADS / 64;
    __shared__ float red[4][WAVES];
    const int r = a.row0 + blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const bool score = !a.dlogits;
    const int act = a.actions[r];
    const float w = !score && a.weights ? a.weights[r] : 1.f;
    const Row<T> row(static_cast<const T*>(a.logits) + r * a.ld, a.V);
    const int np = row.pieces();
    T* out = nullptr;
    bool same = false;
    if (!score) {
        T* p = static_cast<T*>(a.dlogits) + r * a.ld;
        same = int(reinterpret_cast<uintptr_t>(p) % 16 / sizeof(T)) == row.lo;
        out = p - row.lo;
    }
    auto no_gradient = [&] {
        if (score) return;
        if (tid == 0) a.terms[r] = make_float4(0.f, 0.f, 0.f, 0.f);
        const float zero[VEC] = {};
        for (int p = tid; p < np; p += THREADS) row.store(out, same, p, zero);
    };
    auto answer = [&](float l, float H) {
        if (tid == 0 && a.logp) a.logp[r] = l;
        if (tid == 0 && a.entropy) a.entropy[r] = H;
    };
    if (act < 0 || (w == 0.f && !a.logp && !a.entropy)) {
        answer(0.f, 0.f);
        no_gradient();
        return;
    }
    float old = 0.f, adv = 0.f, ref = 0.f;   // (on their way with the row)
    if (!score) {
        old = a.old_logp[r], adv = a.adv[r];
        if (a.ref) ref = a.ref[r];
    }
    const float xa = act < a.V ? to_f(static_cast<const T*>(a.logits)[r * a.ld + act]) : NAN;

    // the row, a piece at a time: from registers, or from memory again
    Piece<T> x[PIECES ? PIECES : 1], none;
#pragma unroll
    for (int j = 0; j < VEC; ++j) none.set(j, out_f<T>(-INFINITY));
    if constexpr (PIECES > 0) {
        // (rows of whole pieces: loads without a branch between them go out together)
        if (row.lo == 0 && row.hi % VEC == 0) {
#pragma unroll
            for (int i = 0; i < PIECES; ++i)
                x[i].v = reinterpret_cast<const uint4*>(row.base)[min(tid + i * THREADS, np - 1)];
#pragma unroll
            for (int i = 0; i < PIECES; ++i)
                if (tid + i * THREADS >= np) x[i] = none;
        } else {
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            const int p = tid + i * THREADS;
            if (p < np) {
                x[i] = row.load(p);
            } else {
                x[i] = none;
            }
        }
        }
    }
    auto each = [&](auto f) {
        if constexpr (PIECES > 0) {
#pragma unroll
            for (int i = 0; i < PIECES; ++i) {
                // (converted again in each pass: the compiler would hold the row as float32)
                asm volatile("" : "+v"(x[i].v.x), "+v"(x[i].v.y), "+v"(x[i].v.z), "+v"(x[i].v.w));
                f(x[i], tid + i * THREADS);
            }
        } else {
            for (int p = tid; p < np; p += THREADS) f(row.load(p), p);
        }
    };
    float m = -INFINITY, W = 0.f;
    if (!score) {
        if (a.own_W) {   // few rows: every workgroup adds the weights up, in the same order
            W = wsum(part_of_weights<THREADS, float>(a));
            if (lane == 0) red[3][wave] = W;
        }
    }
    each([&](const Piece<T>& v, int) {
#pragma unroll
        for (int j = 0; j < VEC; ++j) m = fmaxf(m, v.get(j));
    });
    m = wmax(m);
    if (lane == 0) red[0][wave] = m;
    __syncthreads();
    m = red[0][0];
#pragma unroll
    for (int i = 1; i < WAVES; ++i) m = fmaxf(m, red[0][i]);
    if (!score) {
        if (a.own_W) {
            W = 0.f;
#pragma unroll
            for (int i = 0; i < WAVES; ++i) W += red[3][i];
        } else {
            W = *a.W;
        }
    }
    bool bad = act >= a.V;
    if (m == -INFINITY) {   // nothing to choose from, or NaN and -inf
        bool nan = false;
        each([&](const Piece<T>& v, int) {
#pragma unroll
            for (int j = 0; j < VEC; ++j) nan = nan || v.get(j) != v.get(j);
        });
        bad = __syncthreads_or(nan) || bad;
        if (!bad) {
            answer(-INFINITY, 0.f);
            no_gradient();
            return;
        }
    }
    // (x - M first: the action's own exponent is then exactly 0 where it is the maximum)
    auto exponent = [&](float v) { return (v - m) * kLog2e; };
    Soft f;
    each([&](const Piece<T>& v, int) {
#pragma unroll
        for (int j = 0; j < VEC; ++j) f.add(exponent(v.get(j)));
    });
    const float s1 = wsum(f.s), e1 = wsum(f.e);
    if (lane == 0) red[1][wave] = s1, red[2][wave] = e1;
    __syncthreads();
    float S = 0.f, E = 0.f;
#pragma unroll
    for (int i = 0; i < WAVES; ++i) S += red[1][i], E += red[2][i];
    const float L2 = __builtin_amdgcn_logf(S), inv = 1.f / S;
    float l = (exponent(xa) - L2) * kLn2, H = (L2 - E * inv) * kLn2;
    if (bad) l = H = NAN;
    answer(l, H);
    if (score) return;
    if (w == 0.f) {
        no_gradient();
        return;
    }

    const float ratio = expf(l - old);
    const float free_ = ratio * adv, cut = fminf(fmaxf(ratio, 1.f - a.lo), 1.f + a.hi) * adv;
    const bool off = free_ > cut;
    float c = off ? 0.f : -free_, kl = 0.f;
    if (a.ref) {
        const float u = ref - l;
        kl = kl_term(u);
        if (a.beta != 0.f) c -= a.beta * expm1f(u);   // (0 * inf: u of a forbidden action)
    }
    if (tid == 0) a.terms[r] = make_float4(w * -(off ? cut : free_), w * kl, w * H, off ? w : 0.f);
    // gradient p (es (log p + H) - cs), and cs more at the action
    const float scale = w / W, cs = bad ? NAN : rounded_mul(c, scale), es = a.eta * scale;
    const float g0 = (es * (H - L2 * kLn2) - cs) * inv, g1 = es * kLn2 * inv;
    const int ai = row.lo + (bad ? 0 : act), ap = ai / VEC;
    auto grad = [&](const Piece<T>& v, int p, auto entropy) {
        if (p >= np) return;
        float g[VEC];
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
            const float t = exponent(v.get(j)), e = __builtin_amdgcn_exp2f(t);
            g[j] = e * (entropy.value ? fmaf(g1, fmaxf(t, kFarBelow), g0) : g0);
        }
        if (p == ap) {
#pragma unroll
            for (int j = 0; j < VEC; ++j)
                if (p * VEC + j == ai) g[j] += cs;
        }
        row.store(out, same, p, g);
    };
    if (es != 0.f) each([&](const Piece<T>& v, int p) { grad(v, p, std::true_type{}); });
    else each([&](const Piece<T>& v, int p) { grad(v, p, std::false_type{}); });
}

__global__ __launch_bounds__(1024) void policy_weight_kernel(PolicyArgs a) {
    double s[1] = {part_of_weights<1024, double>(a)};
    sum_up(s);
    if (threadIdx.x == 0) *a.W = float(s[0]);
}

// the statistics, one workgroup
__global__ __launch_bounds__(1024) void policy_stats_kernel(PolicyArgs a, float* stats) {
    double s[5] = {};
    constexpr int U = 4;
    for (int r0 = threadIdx.x; r0 < a.rows; r0 += U * 1024) {
        float4 t[U];
#pragma unroll
        for (int i = 0; i < U; ++i) t[i] = a.terms[min(r0 + i * 1024, a.rows - 1)];
#pragma unroll
        for (int i = 0; i < U; ++i)
            if (r0 + i * 1024 < a.rows) s[0] += t[i].x, s[1] += t[i].y, s[2] += t[i].z, s[3] += t[i].w;
    }
    if (a.own_W) s[4] = part_of_weights<1024, double>(a);
    sum_up(s);
    if (threadIdx.x == 0) {
        const double W = a.own_W ? s[4] : *a.W;
        for (int k = 0; k < 4; ++k) s[k] = W > 0.0 ? s[k] / W : 0.0;
        stats[0] = float(s[0] + (a.ref && a.beta != 0.f ? double(a.beta) * s[1] : 0.0) - (a.eta != 0.f ? double(a.eta) * s[2] : 0.0));
        for (int k = 0; k < 4; ++k) stats[1 + k] = float(s[k]);
        stats[5] = float(W);
    }
}

bool policy_desc_ok(const janus_policy_desc* d) {
    return d && d->rows > 0 && d->V > 0 && (d->ld == 0 || d->ld >= d->V) && std::isfinite(d->clip_low) &&
           d->clip_low >= 0.f && std::isfinite(d->clip_high) && d->clip_high >= 0.f && std::isfinite(d->kl_coef) &&
           std::isfinite(d->ent_coef);
}
size_t policy_carve(PolicyArgs& a, int rows, void* ws) {
    Carver c(ws);
    a.W = c.take<float>(1);
    a.terms = c.take<float4>(rows);
    return c.off;
}

// Up to this many rows each workgroup adds the weights up itself: a launch less.
// Calls on bf16 rows of 10000, workgroups of their own against a launch: 64 rows 11
// and 13 us, 700 15 and 17, 2048 26 and 28, 3000 34 and 32, 8192 95 and 75.
constexpr int kOwnWeightRows = 2048;

// A launch holds fewer than 2^32 threads: more rows take several.
template <typename T, int PIECES, int THREADS>
void row_launch(PolicyArgs a, hipStream_t st) {
    constexpr int kMost = (1 << 30) / THREADS * 2;
    for (; a.row0 < a.rows; a.row0 += kMost)
        hipLaunchKernelGGL((policy_row_kernel<T, PIECES, THREADS>), dim3(std::min(kMost, a.rows - a.row0)),
                           dim3(THREADS), 0, st, a);
}
// The fewest pieces a thread that hold a row (which may touch one piece more
// than its length fills), since every pass works on all of them: small
// workgroups as long as 17 pieces do, for several of them on a CU load, sum and
// store at different times.
template <typename T, int P, int... MORE>
void row_small(int64_t np, const PolicyArgs& a, hipStream_t st) {
    if (np <= 256 * P) return row_launch<T, P, 256>(a, st);
    if constexpr (sizeof...(MORE) > 0) row_small<T, MORE...>(np, a, st);
}
template <typename T>
void row_dispatch(const PolicyArgs& a, hipStream_t st) {
    const int64_t np = (int64_t(a.V) + 16 / sizeof(T) - 2) / (16 / sizeof(T)) + 1;
    if (np <= 256 * 17) row_small<T, 1, 2, 3, 4, 5, 6, 8, 10, 13, 17>(np, a, st);
    else if (np <= 512 * 12) row_launch<T, 12, 512>(a, st);
    else if (np <= 512 * 16) row_launch<T, 16, 512>(a, st);
    else if (np <= 1024 * 12) row_launch<T, 12, 1024>(a, st);
    else if (np <= 1024 * 16) row_launch<T, 16, 1024>(a, st);
    else row_launch<T, 0, 1024>(a, st);
}

}  // namespace
}  // namespace janus

using namespace janus;

extern "C" size_t janus_policy_workspace_bytes(const janus_policy_desc* d) {
    if (!policy_desc_ok(d) || !dtype_ok(d->dtype)) return 0;
    PolicyArgs a{};
    return policy_carve(a, d->rows, nullptr);
}

extern "C" janus_status janus_policy_loss(const janus_policy_desc* d, const void* logits, const int32_t* actions,
                                          const float* old_logp, const float* adv, const float* ref_logp,
                                          const float* weights, void* dlogits, float* logp, float* entropy,
                                          float* stats, void* ws, size_t ws_bytes, void* stream) {
    if (!policy_desc_ok(d) || !logits || !actions) return JANUS_ERR_INVALID_ARG;
    if (!dtype_ok(d->dtype) || d->V > (1 << 30) || d->rows > (1 << 30)) return JANUS_ERR_UNSUPPORTED;
    const bool score = !dlogits;
    if (score ? (old_logp || adv || stats) : (!old_logp || !adv)) return JANUS_ERR_INVALID_ARG;
    const size_t es = dtype_size(d->dtype);
    if (!aligned(logits, es) || !aligned(dlogits, es) || !aligned(actions, 4)) return JANUS_ERR_INVALID_ARG;
    for (const float* p : {old_logp, adv, ref_logp, weights, static_cast<const float*>(logp),
                           static_cast<const float*>(entropy), static_cast<const float*>(stats)})
        if (!aligned(p, 4)) return JANUS_ERR_INVALID_ARG;
    PolicyArgs a{};
    const size_t need = policy_carve(a, d->rows, ws);
    if (!score && (!ws || ws_bytes < need || !aligned(ws, 256))) return JANUS_ERR_WORKSPACE;
    a.rows = d->rows, a.V = d->V, a.ld = d->ld ? d->ld : d->V;
    a.logits = logits, a.actions = actions, a.old_logp = old_logp, a.adv = adv, a.ref = ref_logp, a.weights = weights;
    a.dlogits = dlogits, a.logp = logp, a.entropy = entropy;
    a.lo = d->clip_low, a.hi = d->clip_high, a.beta = d->kl_coef, a.eta = d->ent_coef;
    hipStream_t st = static_cast<hipStream_t>(stream);
    const double el = double(d->rows) * d->V;
    a.own_W = d->rows <= kOwnWeightRows;
    if (!score && !a.own_W) {
        TraceScope trace("policy_weight", double(d->rows), 8.0 * d->rows, st);
        hipLaunchKernelGGL(policy_weight_kernel, dim3(1), dim3(1024), 0, st, a);
        JANUS_LAUNCH_CHECK();
    }
    {
        TraceScope trace("policy_row", 9.0 * el, (score ? 1.0 : 2.0) * el * es, st);
        if (d->dtype == JANUS_BF16) row_dispatch<bf16_t>(a, st);
        else row_dispatch<float>(a, st);
        JANUS_LAUNCH_CHECK();
    }
    if (stats) {
        TraceScope trace("policy_stats", 4.0 * d->rows, 16.0 * d->rows, st);
        hipLaunchKernelGGL(policy_stats_kernel, dim3(1), dim3(1024), 0, st, a, stats);
        JANUS_LAUNCH_CHECK();
    }
    return JANUS_OK;
}
