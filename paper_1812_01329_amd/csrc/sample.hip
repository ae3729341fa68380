// One token from each row of logits by a given uniform number, under temperature,
// top-k, top-p and min-p.
//
//   w_j = 2^((x_j - M) log2(e) / T),  M = max x
//   kept: in the order of (x falling, index rising) the first k, of those the
//         shortest run with p of their weight, of those the ones with w >= min_p
//   token: the first i with  sum_{j <= i, kept} w_j > u sum_{kept} w_j
//
// Which token that is hangs on single bits where a sum meets its border, so weights are
// formed in float64 (relative error 4e-14) and rounded to integers of 38 to 50 bits:
// their sums in 64 bits are exact in any order, and the answer does not depend on how
// threads share the row.
//
// One workgroup a row.  Where the run ends is found without sorting: the logits'
// range is cut in 1024 bins, whose counts (or weights) tell the bin in which the run
// ends; its elements are ranked among themselves if they are few, else cut in bins
// again.  Elements are in the order of their index by wave, by slot, by lane, so the
// border of the draw is found in one wave of the workgroup.
#include <cmath>

#include "rows.hpp"

namespace janus {
namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr int kBins = 1024, kList = 256;

struct SampleArgs {
    int32_t rows, V;
    int32_t row0;         // first row of the launch
    int64_t ld;
    const void* logits;
    const float *u, *T_, *p_, *minp_;
    const int32_t* k_;
    float T, p, minp;
    int32_t k, bits;      // weights are integers, the largest 2^bits
    int32_t* tokens;
    float *logp, *draw_logp;
    int32_t* kept;
};

typedef unsigned long long u64;

// Order of floats as integers (-0 as 0; no NaN)
__device__ __forceinline__ uint32_t key_of(float x) {
    const uint32_t b = __float_as_uint(x + 0.f);
    return b ^ (uint32_t(int32_t(b) >> 31) | 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t k) {
    return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k);
}

// 2^bits 2^((x - M) c), rounded to an integer.  2^f on [-1/2, 1/2] by the polynomial
// through 9 Chebyshev nodes of (2^f - 1) / f.
struct Weight {
    double m, c;
    int bits;
    __device__ __forceinline__ u64 operator()(float x) const {
        const double e = (double(x) - m) * c;
        if (!(e >= -double(bits + 1))) return 0;   // (also -inf, and 0 * inf)
        const double n = rint(e), f = e - n;
        double q = 0x1.b63880c66a8f1p-24;
        q = fma(q, f, 0x1.63d136367c2cdp-20);
        q = fma(q, f, 0x1.ffcb951593518p-17);
        q = fma(q, f, 0x1.4308ac85aa724p-13);
        q = fma(q, f, 0x1.5d87fe86fe886p-10);
        q = fma(q, f, 0x1.3b2ab7181b757p-7);
        q = fma(q, f, 0x1.c6b08d7047e52p-5);
        q = fma(q, f, 0x1.ebfbdff823cedp-3);
        q = fma(q, f, 0x1.62e42fefa39efp-1);
        q = ldexp(fma(q, f, 1.0), int(n) + bits) + 0x1p52;   // (the sum rounds)
        return u64(__double_as_longlong(q)) & 0xfffffffffffffull;
    }
};

__device__ __forceinline__ u64 wave_total(u64 v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
    return v;
}
// sum over this and the lanes before
template <typename S>
__device__ __forceinline__ S wscan(S v) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const S w = __shfl_up(v, o, 64);
        if (lane >= o) v += w;
    }
    return v;
}

template <int WAVES>
struct Shared {
    uint32_t count[kBins];
    u64 mass[kBins];
    uint32_t key[kList];
    int32_t idx[kList];
    u64 w[kList];
    float f[3][WAVES];
    u64 sum[WAVES];
    u64 before;
    uint32_t lo, hi, n, bin;
    int32_t at;
};

// The elements of a run from the front of the order: all of a key above `key`, and those of
// that key up to index `last`.
struct Run {
    uint32_t key = 0;
    int32_t last = 0x7fffffff;
    __device__ __forceinline__ bool has(uint32_t k, int i) const { return k > key || (k == key && i <= last); }
};

template <typename T, int THREADS>
struct Sampler {
    static constexpr int VEC = 16 / sizeof(T), WAVES = THREADS / 64;
    const Row<T> row;
    Shared<WAVES>& sh;
    int slots, first;     // 64 pieces a slot; this wave's first piece
    float m = 0.f, low = 0.f;
    Weight weight;

    __device__ Sampler(const T* p, int V, Shared<WAVES>& s) : row(p, V), sh(s) {
        const int np = row.pieces();
        slots = (np + THREADS - 1) / THREADS;
        first = (threadIdx.x >> 6) * slots * 64 + (threadIdx.x & 63);
    }
    // f(value, index) for the lane's elements of a slot (-inf outside the row)
    template <typename F>
    __device__ __forceinline__ void slot(int i, F f) const {
        const int p = first + i * 64;
        if (p >= row.pieces()) return;
        const Piece<T> v = row.load(p);
#pragma unroll
        for (int j = 0; j < VEC; ++j) f(v.get(j), p * VEC + j - row.lo);
    }
    template <typename F>
    __device__ __forceinline__ void each(F f) const {
#pragma unroll 2
        for (int i = 0; i < slots; ++i) slot(i, f);
    }
    // sum over the workgroup of a number a wave has (in all its lanes)
    __device__ __forceinline__ u64 over_waves(u64 v, u64& before) const {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
        __syncthreads();
        if (lane == 0) sh.sum[wave] = v;
        __syncthreads();
        u64 s = 0;
        before = 0;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            if (w == wave) before = s;
            s += sh.sum[w];
        }
        return s;
    }

    // Index of the n-th (from 1) live element with this key
    __device__ int nth(uint32_t key, u64 n) {
        int c = 0;
        each([&](float x, int) { c += x > -INFINITY && key_of(x) == key; });
        u64 before;
        const u64 own = wave_total(u64(c));
        over_waves(own, before);
        if (before < n && n <= before + own) {
            u64 left = n - before;
            for (int i = 0; i < slots; ++i) {
                int k = 0;
                slot(i, [&](float x, int) { k += x > -INFINITY && key_of(x) == key; });
                const int up = wscan(k), all = __shfl(up, 63, 64);
                if (u64(all) >= left) {
                    if (u64(up) >= left && u64(up - k) < left) {
                        u64 seen = u64(up - k);
                        slot(i, [&](float x, int j) {
                            if (x > -INFINITY && key_of(x) == key && ++seen == left) sh.at = j;
                        });
                    }
                    break;
                }
                left -= u64(all);
            }
        }
        __syncthreads();
        const int at = sh.at;
        __syncthreads();
        return at;
    }

    // Shortens the run to its first `need` elements, or (MASS) to the shortest one with the
    // share p of its weight.
    template <bool MASS>
    __device__ void shorten(Run& run, u64 need, float p) {
        constexpr int PER = kBins / THREADS;
        const int tid = threadIdx.x;
        uint32_t lo = 0, hi = 0xffffffffu;   // keys among which the run's end is
        const float scale = m > low ? float(kBins) / (m - low) : 0.f;
        for (int level = 0;; ++level) {
            const int sft = level ? max(0, 32 - __clz(int(hi - lo)) - 10) : 0;
            auto member = [&](float x, uint32_t k, int j) { return x > -INFINITY && k >= lo && k <= hi && run.has(k, j); };
            auto bin = [&](float x, uint32_t k) {
                if (level) return int((hi - k) >> sft);
                const float b = (m - x) * scale;
                return b < float(kBins - 1) ? int(b) : kBins - 1;   // (inf * 0 of far values: the last)
            };
#pragma unroll
            for (int t = 0; t < PER; ++t) {
                sh.count[tid + t * THREADS] = 0;
                if (MASS) sh.mass[tid + t * THREADS] = 0;
            }
            __syncthreads();
            each([&](float x, int j) {
                const uint32_t k = key_of(x);
                if (!member(x, k, j)) return;
                const int b = bin(x, k);
                atomicAdd(&sh.count[b], 1u);
                if (MASS) atomicAdd(&sh.mass[b], weight(x));
            });
            __syncthreads();
            // a thread has PER bins; `own` what they hold
            u64 own = 0;
#pragma unroll
            for (int t = 0; t < PER; ++t) own += MASS ? sh.mass[tid * PER + t] : u64(sh.count[tid * PER + t]);
            const u64 up = wscan(own), wave_all = __shfl(up, 63, 64);
            u64 before;
            const u64 all = over_waves(wave_all, before);
            before += up - own;
            if (MASS && level == 0) {
                const double t = ceil(double(p) * double(all));
                need = t < 1.0 ? 1 : t > double(all) ? all : u64(t);
            }
#pragma unroll
            for (int t = 0; t < PER; ++t) {
                const u64 v = MASS ? sh.mass[tid * PER + t] : u64(sh.count[tid * PER + t]);
                if (before < need && need <= before + v) {
                    sh.bin = tid * PER + t, sh.before = before;
                    sh.n = 0, sh.lo = 0xffffffffu, sh.hi = 0;
                }
                before += v;
            }
            __syncthreads();
            const int b = sh.bin;
            const uint32_t n = sh.count[b];
            need -= sh.before;
            auto inside = [&](float x, uint32_t k, int j) { return member(x, k, j) && bin(x, k) == b; };
            if (n <= uint32_t(kList)) {
                each([&](float x, int j) {
                    const uint32_t k = key_of(x);
                    if (!inside(x, k, j)) return;
                    const uint32_t at = atomicAdd(&sh.n, 1u);
                    sh.key[at] = k, sh.idx[at] = j;
                    if (MASS) sh.w[at] = weight(x);
                });
                __syncthreads();
                for (uint32_t t = tid; t < n; t += THREADS) {
                    const uint32_t k = sh.key[t];
                    const int j = sh.idx[t];
                    u64 ahead = 0;
                    for (uint32_t o = 0; o < n; ++o)
                        if (sh.key[o] > k || (sh.key[o] == k && sh.idx[o] < j)) ahead += MASS ? sh.w[o] : 1;
                    if (ahead < need && need <= ahead + (MASS ? sh.w[t] : 1)) sh.lo = k, sh.at = j;
                }
                __syncthreads();
                run.key = sh.lo, run.last = sh.at;
                __syncthreads();
                return;
            }
            uint32_t a = 0xffffffffu, z = 0;
            each([&](float x, int j) {
                const uint32_t k = key_of(x);
                if (inside(x, k, j)) a = min(a, k), z = max(z, k);
            });
#pragma unroll
            for (int o = 32; o > 0; o >>= 1) a = min(a, uint32_t(__shfl_xor(int(a), o, 64))), z = max(z, uint32_t(__shfl_xor(int(z), o, 64)));
            if ((tid & 63) == 0) atomicMin(&sh.lo, a), atomicMax(&sh.hi, z);
            __syncthreads();
            lo = sh.lo, hi = sh.hi;
            __syncthreads();
            if (lo == hi) {   // many equal ones: the first by index
                u64 r = need;
                if (MASS) {
                    const u64 w = weight(value_of(lo));
                    r = (need + w - 1) / w;
                }
                run.last = nth(lo, r);
                run.key = lo;
                return;
            }
        }
    }
};

template <typename T, int THREADS>
__global__ __launch_bounds__(THREADS) void sample_kernel(SampleArgs a) {
    constexpr int WAVES = THREADS / 64;
    __shared__ Shared<WAVES> sh;
    const int r = a.row0 + blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const T* logits = static_cast<const T*>(a.logits) + r * a.ld;
    Sampler<T, THREADS> s(logits, a.V, sh);
    const float temp = a.T_ ? a.T_[r] : a.T, p = a.p_ ? a.p_[r] : a.p, minp = a.minp_ ? a.minp_[r] : a.minp, u = a.u[r];
    const int k = a.k_ ? a.k_[r] : a.k;
    auto answer = [&](int token, float logp, float drawn, int kept) {
        a.tokens[r] = token;
        if (a.logp) a.logp[r] = logp;
        if (a.draw_logp) a.draw_logp[r] = drawn;
        if (a.kept) a.kept[r] = kept;
    };

    // the largest and the smallest logit, and how many are live
    float m = -INFINITY, low = INFINITY;
    int live = 0;
    bool nan = false;
    s.each([&](float x, int) {
        m = fmaxf(m, x);
        nan = nan || x != x;
        if (x > -INFINITY) low = fminf(low, x), ++live;
    });
    m = wmax(m), low = -wmax(-low);
    float cnt = float(live);   // (V is below 2^24)
    cnt = wsum(cnt);
    if (lane == 0) sh.f[0][wave] = m, sh.f[1][wave] = low, sh.f[2][wave] = cnt;
    nan = __syncthreads_or(nan);
    cnt = 0.f;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) m = fmaxf(m, sh.f[0][w]), low = fminf(low, sh.f[1][w]), cnt += sh.f[2][w];
    live = int(cnt);
    __syncthreads();
    if (nan || m == INFINITY || !(temp >= 0.f) || p != p || minp != minp || u != u) {
        if (tid == 0) answer(-1, NAN, NAN, 0);
        return;
    }
    if (live == 0) {
        if (tid == 0) answer(-1, -INFINITY, -INFINITY, 0);
        return;
    }
    s.m = m, s.low = low;
    s.weight = Weight{double(m), 1.4426950408889634074 / double(temp), a.bits};

    // log of the sum of exp(x - m)
    float lse = 0.f;
    if (a.logp) {
        float e = 0.f;
        s.each([&](float x, int) { e += __builtin_amdgcn_exp2f((x - m) * kLog2e); });
        e = wsum(e);
        if (lane == 0) sh.f[0][wave] = e;
        __syncthreads();
        e = 0.f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) e += sh.f[0][w];
        lse = __builtin_amdgcn_logf(e);
        __syncthreads();
    }
    auto logp_of = [&](float x) { return fmaf(-lse, kLn2, x - m); };   // (lse: a binary logarithm)

    if (temp == 0.f) {   // the first of the largest
        const int j = s.nth(key_of(m), 1);
        if (tid == 0) answer(j, logp_of(m), 0.f, 1);
        return;
    }
    Run run;
    if (k > 0 && k < live) s.template shorten<false>(run, u64(k), 0.f);
    if (p < 1.f) s.template shorten<true>(run, 0, p);
    if (minp > 0.f && temp < INFINITY) {
        const uint32_t least = key_of(__double2float_ru(double(m) + double(temp) * log(fmin(double(minp), 1.0))));
        if (least > run.key) run.key = least, run.last = 0x7fffffff;
    }

    auto kept = [&](float x, int j) { return x > -INFINITY && run.has(key_of(x), j); };
    u64 own = 0;
    int n = 0;
    s.each([&](float x, int j) {
        if (kept(x, j)) own += s.weight(x), ++n;
    });
    own = wave_total(own);
    u64 before, nb;
    const u64 all = s.over_waves(own, before);
    const int count = int(s.over_waves(wave_total(u64(n)), nb));
    const double t = double(fminf(fmaxf(u, 0.f), 1.f)) * double(all);
    const u64 border = min(u64(t), all - 1);
    if (!(before <= border && border < before + own)) return;
    u64 left = border - before;
    for (int i = 0; i < s.slots; ++i) {
        u64 w = 0;
        s.slot(i, [&](float x, int j) {
            if (kept(x, j)) w += s.weight(x);
        });
        const u64 up = wscan(w), sum = __shfl(up, 63, 64);
        if (left < sum) {
            if (up - w <= left && left < up) {
                u64 c = up - w;
                bool found = false;
                s.slot(i, [&](float x, int j) {
                    if (found || !kept(x, j)) return;
                    const u64 v = s.weight(x);
                    c += v;
                    if (c > left) {
                        found = true;
                        answer(j, logp_of(x), float(log(double(v) / double(all))), count);
                    }
                });
            }
            return;
        }
        left -= sum;
    }
}

bool sample_desc_ok(const janus_sample_desc* d) {
    return d && d->rows > 0 && d->V > 0 && (d->ld == 0 || d->ld >= d->V) && d->temperature >= 0.f &&
           !std::isnan(d->top_p) && !std::isnan(d->min_p);
}

// Rows of up to this many pieces of 16 bytes take workgroups of 256 threads.
constexpr int kSmallRow = 1024;

// A launch holds fewer than 2^32 threads: more rows take several.
template <typename T, int THREADS>
void sample_launch(SampleArgs a, hipStream_t st) {
    constexpr int kMost = (1 << 30) / THREADS * 2;
    for (; a.row0 < a.rows; a.row0 += kMost)
        hipLaunchKernelGGL((sample_kernel<T, THREADS>), dim3(std::min(kMost, a.rows - a.row0)), dim3(THREADS), 0, st, a);
}
template <typename T>
void sample_dispatch(const SampleArgs& a, hipStream_t st) {
    if (int64_t(a.V) * sizeof(T) <= kSmallRow * 16) sample_launch<T, 256>(a, st);
    else sample_launch<T, 1024>(a, st);
}

}  // namespace
}  // namespace janus

using namespace janus;

extern "C" size_t janus_sample_workspace_bytes(const janus_sample_desc*) { return 0; }

extern "C" janus_status janus_sample(const janus_sample_desc* d, const void* logits, const float* u,
                                     const float* temperature, const int32_t* top_k, const float* top_p,
                                     const float* min_p, int32_t* tokens, float* logp, float* draw_logp, int32_t* kept,
                                     void* ws, size_t ws_bytes, void* stream) {
    if (!sample_desc_ok(d) || !logits || !u || !tokens) return JANUS_ERR_INVALID_ARG;
    if (!dtype_ok(d->dtype) || d->V > (1 << 24) || d->rows > (1 << 30)) return JANUS_ERR_UNSUPPORTED;
    const size_t es = dtype_size(d->dtype);
    if (!aligned(logits, es)) return JANUS_ERR_INVALID_ARG;
    for (const void* p : {static_cast<const void*>(u), static_cast<const void*>(temperature), static_cast<const void*>(top_k),
                          static_cast<const void*>(top_p), static_cast<const void*>(min_p),
                          static_cast<const void*>(tokens), static_cast<const void*>(logp),
                          static_cast<const void*>(draw_logp), static_cast<const void*>(kept)})
        if (!aligned(p, 4)) return JANUS_ERR_INVALID_ARG;
    (void)ws, (void)ws_bytes;
    SampleArgs a{};
    a.rows = d->rows, a.V = d->V, a.ld = d->ld ? d->ld : d->V;
    a.logits = logits, a.u = u, a.T_ = temperature, a.k_ = top_k, a.p_ = top_p, a.minp_ = min_p;
    a.T = d->temperature, a.k = d->top_k, a.p = d->top_p, a.minp = d->min_p;
    int log2V = 0;
    while ((int64_t(1) << log2V) < d->V) ++log2V;
    a.bits = std::min(50, 62 - log2V);   // (a row's sum stays below 2^63)
    a.tokens = tokens, a.logp = logp, a.draw_logp = draw_logp, a.kept = kept;
    hipStream_t st = static_cast<hipStream_t>(stream);
    const double el = double(d->rows) * d->V;
    TraceScope trace("sample", 6.0 * el, el * es, st);
    if (d->dtype == JANUS_BF16) sample_dispatch<bf16_t>(a, st);
    else sample_dispatch<float>(a, st);
    JANUS_LAUNCH_CHECK();
    return JANUS_OK;
}
