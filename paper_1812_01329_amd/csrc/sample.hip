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
// One workgroup a row, which it holds in LDS, a thread a run of neighbours.  Three ways to
// the token:
//   a short list  With top-k the k-th largest of the threads' own maxima is a value that
//         at least k logits reach and few more; with min-p the border is known.  What
//         reaches it is listed, compared pair by pair (or, past 256, sorted), cut and
//         drawn from: only the list needs weights (top-p without top-k: one sum of all).
//   cut in bins   Otherwise the run's end is found without sorting: the logits' range
//         is cut in 1024 bins, whose counts (or weights) tell the bin in which the run
//         ends; its elements are ranked among themselves if they are few, else cut in
//         bins again.
//   the whole row  What is kept and not listed is added up by thread; the draw's border is
//         then among one thread's elements.  Min-p alone goes this way too.
//
// Few rows are bound by the chain of passes and scans between lanes: 20 rows of 10000 bf16
// with top-k and top-p 9.6 us, 37 of 20001 float32 with min-p 11.1.  Many spend their time in the
// vector units and in turns: a CU has room for one row past 16384 bf16, which it
// loads, waits for at barriers and works on one after another.  1024 rows of 65536 bf16 with
// nothing filtered take 85 us (1.6 TB/s): 32 vector instructions a logit, most of them a
// weight's in float64, keep the units busy for 62 % of it (91 us with the weights of
// four elements in turn).  2000 rows of 32768 bf16 with min-p take 72 us (1.8 TB/s; with the
// log-probability the units are busy for 57 %, LDS for 6 %), 2000 of 40000 with top-p alone
// 272: 96 instructions a logit, 76 %, and LDS with its atomics 16 %.  A row in
// registers instead of LDS needs every pass unrolled, which the instruction cache does not
// hold: 45 us for 37 rows where LDS took 20.
#include <cmath>
#include <mutex>

#include "rows.hpp"

namespace janus {
namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr int kBins = 1024, kPairs = 256;

struct SampleArgs {
    int32_t rows, V;
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

// Order of floats as integers (-0 as 0; no NaN)
__device__ __forceinline__ uint32_t key_of(float x) {
    const uint32_t b = __float_as_uint(x + 0.f);
    return b ^ (uint32_t(int32_t(b) >> 31) | 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t k) {
    return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k);
}

// f v of a float in [0, 1], rounded down; `more`: something was cut off.  Exact: half of
// an even number of equal weights is half of them.
__device__ __forceinline__ u64 fraction(float f, u64 v, bool& more) {
    const uint32_t b = __float_as_uint(f);
    const int shift = 150 - max(int(b >> 23), 1);           // f = mantissa 2^-shift, shift 23 at least
    const u64 man = (b & 0x7fffffu) | (b >> 23 ? 0x800000u : 0u);
    const u64 hi = __umul64hi(man, v), lo = man * v;
    if (shift >= 64) {
        const int s = shift - 64;
        more = lo != 0 || (s < 64 ? hi & ((1ull << s) - 1) : hi) != 0;
        return s < 64 ? hi >> s : 0;
    }
    more = (lo & ((1ull << shift) - 1)) != 0;
    return (hi << (64 - shift)) | (lo >> shift);
}

// 2^f on [-1/2, 1/2] by the polynomial through 9 Chebyshev nodes of (2^f - 1) / f (off by 4e-14)
__device__ __forceinline__ double power_of_2(double f) {
    double q = 0x1.b63880c66a8f1p-24;
    q = fma(q, f, 0x1.63d136367c2cdp-20);
    q = fma(q, f, 0x1.ffcb951593518p-17);
    q = fma(q, f, 0x1.4308ac85aa724p-13);
    q = fma(q, f, 0x1.5d87fe86fe886p-10);
    q = fma(q, f, 0x1.3b2ab7181b757p-7);
    q = fma(q, f, 0x1.c6b08d7047e52p-5);
    q = fma(q, f, 0x1.ebfbdff823cedp-3);
    q = fma(q, f, 0x1.62e42fefa39efp-1);
    return fma(q, f, 1.0);
}
// log r of a positive r from 2^-180 on: from the float32 logarithm y, r 2^-y is 1 + e with a small e,
// and log(1 + e) = e - e^2 / 2
__device__ __forceinline__ double log_of(double r) {
    const float shift = r < 0x1p-90 ? 96.f : 0.f;   // (float32 has no smaller ones)
    const float y = __builtin_amdgcn_logf(float(ldexp(r, int(shift)))) - shift, n = rintf(y);
    const double e = ldexp(r, -int(n)) * power_of_2(double(n - y)) - 1.0;
    return double(y) * 0.69314718055994530942 + (e - 0.5 * e * e);
}

// 2^bits 2^((x - M) c), rounded to an integer
struct Weight {
    double m, c, least, magic;    // least: an exponent that rounds to 0
    // kOne + the weight: in the low 52 bits of a float64 that has 2^52 added (which rounds it)
    static constexpr u64 kOne = 0x4330000000000000ull;
    __device__ __forceinline__ void set(float largest, float T, int bits) {
        m = double(largest), c = 1.4426950408889634074 / double(T);
        least = -double(bits + 2), magic = 0x1.8p52 + double(bits);
    }
    __device__ __forceinline__ u64 raw(float x) const {
        const double e = fmax((double(x) - m) * c, least);      // (-inf, and NaN from 0 * inf, go to `least`)
        const double z = e + magic, f = e - (z - magic);        // z: e + bits rounded, in its low bits
        return u64(__double_as_longlong(ldexp(power_of_2(f), int(uint32_t(__double_as_longlong(z)))) + 0x1p52));
    }
    __device__ __forceinline__ u64 operator()(float x) const { return raw(x) - kOne; }
};

// An entry of a list: key and index in one number that falls in the run's order, and a weight
struct Entry {
    u64 at, w;
};
__device__ __forceinline__ u64 place_of(uint32_t key, int j) { return u64(key) << 32 | uint32_t(~j); }

template <int THREADS>
struct Shared {
    u64 mass[kBins];      // weights of bins; sums of pairs; a sort's exchange
    uint32_t count[kBins];
    Entry list[kBins];
    float f[3][THREADS / 64];
    u64 sum[THREADS / 64];
    u64 before, total, kept_total;
    double depth;
    uint32_t lo, hi, n, bin, kept, live;
    uint32_t bins[65];
    int32_t at;
};
extern __shared__ uint4 held_row[];

// The elements of a run from the front of the order: all of a key above `key`, and those of
// that key up to index `last`.
struct Run {
    uint32_t key = 0;
    int32_t last = 0x7fffffff;
    __device__ __forceinline__ bool has(uint32_t k, int i) const { return k > key || (k == key && i <= last); }
};

// Pieces of 16 bytes of a row that LDS holds beside the rest (29 of a CU's 160 KB): in a
// workgroup of 1024 threads, in one of 256 and in one of 512.  Smaller workgroups wait less
// at their barriers, and more of them share a CU.  With top-k and top-p, 300 rows of 4000
// bf16 take 11.4, 11.7 and 19.8 us in 256, 512 and 1024 threads, 2000 rows 24, 35 and 64;
// 300 and 2000 rows of 16000 13.3 and 44 us in 512, 21.4 and 73 in 1024.
constexpr int kHeld = 8192, kHeldSmall = 512, kHeldMiddle = 2048;
// In a row that is not held, up to this many elements that min-p alone keeps are listed: marks are
// met again in memory, by their weights and by the border.  Rows of 50257 float32 by list and by
// marks: 20 rows that keep 12 14.7 and 20.3 us, 96 16.4 and 20.6, 200 21.1 and 20.9, 900 31.7 and 23.3;
// 2000 rows 175, 188, 226 and 320 by list, 207, 211, 212 and 227 by marks (counting them is
// 1 to 3 % on top).
constexpr uint32_t kFewMarked = 128;
template <int THREADS> constexpr int kSlots = THREADS == 256 ? 2 : THREADS == 512 ? 4 : 8;   // a thread's at most
constexpr size_t held_bytes(int64_t np) { return size_t(np + 8) * 16; }  // (the last thread's pieces are turned as well)

// HELD: the row is in LDS, a thread has `slots` pieces one after another; else a wave
// has 64 `slots` of them, which its lanes read from memory in every pass, 64 at a time.
template <typename T, int THREADS, bool HELD>
struct Sampler {
    static constexpr int VEC = 16 / sizeof(T), WAVES = THREADS / 64;
    const T* row;
    Shared<THREADS>& sh;
    int V, np, slots, first, turn;   // V elements in np pieces
    float m = 0.f;
    Weight weight;

    __device__ __forceinline__ Sampler(const T* p, int n, Shared<THREADS>& s) : row(p), sh(s), V(n) {
        np = (V + VEC - 1) / VEC;
        slots = (np + THREADS - 1) / THREADS;
        first = HELD ? int(threadIdx.x) * slots : int(threadIdx.x >> 6) * slots * 64 + int(threadIdx.x & 63);
        turn = HELD ? turn_of(threadIdx.x) : 0;
    }
    // Where thread t's piece i lies in LDS: its pieces are turned by some, so that 8 lanes
    // which read theirs at once meet 8 different sets of banks.
    __device__ __forceinline__ int turn_of(int t) const {
        const int g = slots & 1 ? 1 : slots & 2 ? 2 : slots & 4 ? 4 : 8;   // (of 8 banks' sets, how many lanes meet in one)
        return (t * g >> 3) & (g - 1);
    }
    __device__ __forceinline__ int held_at(int start, int t, int i) const {
        const int q = i + t;
        return start + (q >= slots ? q - slots : q);
    }
    // f(value, index) for the elements of a piece (-inf outside the row)
    template <typename F>
    __device__ __forceinline__ void elements(const Piece<T>& v, int p, F f) const {
#pragma unroll
        for (int j = 0; j < VEC; ++j) f(v.get(j), p * VEC + j);
    }
    __device__ __forceinline__ bool ragged() const { return V % VEC != 0; }   // the last piece has less
    // 16 bytes from where any element starts
    __device__ __forceinline__ uint4 whole_piece(int p) const {
        typedef uint32_t Words __attribute__((ext_vector_type(4), aligned(2)));
        const Words w = *reinterpret_cast<const Words*>(row + int64_t(p) * VEC);
        return make_uint4(w.x, w.y, w.z, w.w);
    }
    // (the last piece may have less: by its elements)
    __device__ __forceinline__ Piece<T> from_memory(int p) const {
        Piece<T> r;
        if (p < np - 1 || !ragged()) {
            r.v = whole_piece(p);
        } else {
#pragma unroll
            for (int j = 0; j < VEC; ++j) r.set(j, p * VEC + j < V ? row[p * VEC + j] : out_f<T>(-INFINITY));
        }
        return r;
    }
    __device__ __forceinline__ bool piece(int i, int& p, Piece<T>& v) const {
        p = HELD ? first + i : first + i * 64;
        if (p >= np) return false;
        if constexpr (HELD) v.v = held_row[held_at(first, turn, i)];
        else v = from_memory(p);
        return true;
    }
    template <typename F>
    __device__ __forceinline__ void slot(int i, F f) const {
        int p;
        Piece<T> v;
        if (piece(i, p, v)) elements(v, p, f);
    }
    // The same for all of the thread's elements.  Loops stay loops: a pass is run once or
    // twice a row, and what is unrolled waits for its instructions to be fetched.
    template <typename F>
    __device__ __forceinline__ void each(F f) const {
#pragma unroll 1
        for (int i = 0; i < slots; ++i) slot(i, f);
    }
    // The row's pieces tid, tid + THREADS, ... on their way to registers, but a ragged one
    __device__ __forceinline__ void fetch(uint4 (&v)[kSlots<THREADS>]) const {
        const int last = V / VEC - 1;
#pragma unroll
        for (int k = 0; k < kSlots<THREADS>; ++k)
            if (k < slots && last >= 0) v[k] = whole_piece(min(int(threadIdx.x) + k * THREADS, last));
    }
    // The first pass, which brings the row to LDS (any thread meets any element): the
    // largest of what the thread met, and whether any was NaN, and any -inf (or may be).
    __device__ __forceinline__ void largest(const uint4 (&v)[kSlots<THREADS>], float& own, bool& nan, bool& holes) const {
        typedef unsigned short ushort2_t __attribute__((ext_vector_type(2)));
        own = -INFINITY, nan = false, holes = true;
        ushort2_t bits = {0, 0};   // (the largest of bf16 values' bits without the sign)
        auto meet = [&](const Piece<T>& x) {
#pragma unroll
            for (int j = 0; j < VEC; ++j) own = fmaxf(own, x.get(j));
            if constexpr (sizeof(T) == 2) {
                const uint32_t u[4] = {x.v.x, x.v.y, x.v.z, x.v.w};
#pragma unroll
                for (int j = 0; j < 4; ++j) bits = __builtin_elementwise_max(bits, __builtin_bit_cast(ushort2_t, u[j] & 0x7fff7fffu));
            } else {
#pragma unroll
                for (int j = 0; j < VEC; ++j) nan = nan || x.get(j) != x.get(j);
            }
        };
        if constexpr (HELD) {
            const uint32_t inv = ((1u << 18) + slots - 1) / slots;   // (exact for p up to 8192, slots up to 8)
            auto put = [&](const Piece<T>& x, int p) {
                const int t = int(__umul24(uint32_t(p), inv) >> 18), i = p - int(__umul24(uint32_t(t), uint32_t(slots)));
                held_row[held_at(p - i, turn_of(t), i)] = x.v;
                meet(x);
            };
            const int full = V / VEC;
#pragma unroll
            for (int k = 0; k < kSlots<THREADS>; ++k) {
                const int p = int(threadIdx.x) + k * THREADS;
                Piece<T> x;
                x.v = v[k];
                if (k < slots && p < full) put(x, p);
            }
            if (ragged() && int(threadIdx.x) == full % THREADS) put(from_memory(full), full);
        } else {
#pragma unroll 1
            for (int i = 0; i < slots; ++i) {
                int p;
                Piece<T> x;
                if (piece(i, p, x)) meet(x);
            }
        }
        if constexpr (sizeof(T) == 2) nan = max(bits.x, bits.y) > 0x7f80, holes = max(bits.x, bits.y) == 0x7f80;
    }

    // sum over the workgroup of a number a wave has (in all its lanes), and over the waves before
    __device__ __forceinline__ u64 over_waves(u64 v, u64& before) const {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
        __syncthreads();
        if (lane == 0) sh.sum[wave] = v;
        __syncthreads();
        const u64 up = up_to(lane < WAVES ? sh.sum[lane] : 0);
        const u64 own = u64(uint32_t(__builtin_amdgcn_readlane(int(uint32_t(up)), wave))) |
                        u64(uint32_t(__builtin_amdgcn_readlane(int(uint32_t(up >> 32)), wave))) << 32;
        before = own - v;
        return last_lane(up);
    }
    // sum over the threads before; `all`: over all of them
    __device__ __forceinline__ u64 threads_before(u64 v, u64& all) const {
        const u64 up = up_to(v);
        u64 before;
        all = over_waves(last_lane(up), before);
        return before + up - v;
    }
    __device__ __forceinline__ float over_waves_sum(float v) const {
        v = wave_sum(v);
        __syncthreads();
        if ((threadIdx.x & 63) == 0) sh.f[0][threadIdx.x >> 6] = v;
        __syncthreads();
        return wave_sum((threadIdx.x & 63) < WAVES ? sh.f[0][threadIdx.x & 63] : 0.f);
    }

    // The element where the sum of w(x, j), in the order of the index, passes `target`, a sum
    // that is below all of them: done(index, value, weight) on one lane.  `mine`, `before`: the
    // thread's sum and that of the threads before.
    template <typename W, typename D>
    __device__ __forceinline__ void border(u64 mine, u64 before, u64 target, W w, D done) const {
        const int lane = threadIdx.x & 63;
        if constexpr (HELD) {
            if (before <= target && target < before + mine) sh.at = threadIdx.x, sh.before = before;
            __syncthreads();
            if (threadIdx.x >= 64) return;
            const int t = sh.at, start = t * slots, n = min(slots, np - start) * VEC, turned = turn_of(t);
            u64 left = target - sh.before;
            for (int e0 = 0; e0 < n; e0 += 64) {
                const int e = e0 + lane, j = start * VEC + e;
                float x = -INFINITY;
                if (e < n) {
                    const T* at = reinterpret_cast<const T*>(&held_row[held_at(start, turned, e / VEC)]);
                    x = to_f(at[e % VEC]);
                }
                const u64 v = e < n ? w(x, j) : 0, up = up_to(v), sum = last_lane(up);
                if (left < sum) {
                    if (up - v <= left && left < up) done(j, x, v);
                    return;
                }
                left -= sum;
            }
        } else {
            // (a wave's elements are in the order slot, lane, so its lanes' sums say only that they are its)
            const u64 wave_sum_ = last_lane(up_to(mine));
            const u64 wave_before = u64(uint32_t(__builtin_amdgcn_readfirstlane(int(uint32_t(before))))) |
                                    u64(uint32_t(__builtin_amdgcn_readfirstlane(int(uint32_t(before >> 32))))) << 32;
            if (target < wave_before || target >= wave_before + wave_sum_) return;
            u64 left = target - wave_before;
            for (int i = 0; i < slots; ++i) {
                u64 v = 0;
                slot(i, [&](float x, int j) { v += w(x, j); });
                const u64 up = up_to(v), sum = last_lane(up);
                if (left < sum) {
                    if (up - v <= left && left < up) {
                        u64 c = up - v;
                        bool found = false;
                        slot(i, [&](float x, int j) {
                            const u64 one = w(x, j);
                            c += one;
                            if (!found && c > left) found = true, done(j, x, one);
                        });
                    }
                    return;
                }
                left -= sum;
            }
        }
    }

    // Index of the n-th (from 1) live element with this key
    __device__ __forceinline__ int nth(uint32_t key, u64 n) {
        auto is = [&](float x, int) { return u64(x > -INFINITY && key_of(x) == key); };
        uint32_t c = 0;
        each([&](float x, int j) { c += uint32_t(is(x, j)); });
        u64 all;
        const u64 before = threads_before(c, all);
        border(c, before, n - 1, is, [&](int j, float, u64) { sh.bin = uint32_t(j); });
        __syncthreads();
        const int at = int(sh.bin);
        __syncthreads();
        return at;
    }

    // Sorts a number of each of the first n threads, falling (n: a power of two, 64 at least).
    __device__ __forceinline__ u64 sorted(u64 v, int n) const {
        const int tid = threadIdx.x;
        if (n == 64 && tid >= 64) return v;
        for (int size = 2; size <= n; size <<= 1)
            for (int stride = size / 2; stride > 0; stride >>= 1) {
                u64 o;
                if (stride >= 64) {
                    __syncthreads();
                    sh.mass[tid] = v;
                    __syncthreads();
                    o = sh.mass[tid ^ stride];
                } else {
                    o = __shfl_xor(v, stride, 64);
                }
                const bool high = ((tid & stride) == 0) == ((tid & size) == 0);
                v = (v > o) == high ? v : o;
            }
        return v;
    }

    // For every entry of the list (n of them, kPairs at most): how many are ahead of it (in
    // sh.count) and their weight (in sh.mass); BY_INDEX: weight alone, of those with a lower index.
    // A wave takes 64 entries against a part of the others.
    template <bool BY_INDEX>
    __device__ __forceinline__ void pairs(int n) const {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
        const int groups = (n + 63) / 64, parts = WAVES / groups;
        if (wave >= parts * groups) return;
        const int i = wave % groups * 64 + lane, part = wave / groups;
        const int j0 = n * part / parts, j1 = n * (part + 1) / parts;
        const u64 mine = i < n ? sh.list[i].at : 0;
        uint32_t c = 0;
        u64 s = 0;
#pragma unroll 4
        for (int j = j0; j < j1; ++j) {
            const Entry e = sh.list[j];
            const bool ahead = BY_INDEX ? uint32_t(e.at) > uint32_t(mine) : e.at > mine;
            c += ahead;
            s += ahead ? e.w : 0;
        }
        if (i >= n) return;
        if (!BY_INDEX) atomicAdd(&sh.count[i], c);
        atomicAdd(&sh.mass[i], s);
    }

    // Shortens the run to its first `need` elements, or (MASS) to the shortest one with the
    // share p of its weight.  low: the smallest live logit.  total: with weights in
    // bins from gather(), the weight of all (else 0).
    template <bool MASS>
    __device__ __forceinline__ void shorten(Run& run, u64 need, float p, float low, u64 total) {
        constexpr int PER = kBins / THREADS;
        const int tid = threadIdx.x;
        uint32_t lo = 0, hi = 0xffffffffu;   // keys among which the run's end is
        const float scale = MASS ? bin_scale() : m > low ? float(kBins) / (m - low) : 0.f;
        for (int level = 0;; ++level) {
            const int sft = level ? max(0, 32 - __clz(int(hi - lo)) - 10) : 0;
            auto member = [&](float v, uint32_t k, int j) { return v > -INFINITY && k >= lo && k <= hi && run.has(k, j); };
            auto bin = [&](float v, uint32_t k) {
                if (level) return int((hi - k) >> sft);
                const float b = (m - v) * scale;
                return b < float(kBins - 1) ? int(b) : kBins - 1;   // (0 * inf of far values: the last)
            };
            const bool binned = MASS && level == 0 && total;
            if (!binned) {
                __syncthreads();
#pragma unroll
                for (int t = 0; t < PER; ++t) {
                    sh.count[tid + t * THREADS] = 0;
                    if (MASS) sh.mass[tid + t * THREADS] = 0;
                }
                __syncthreads();
                each([&](float v, int j) {
                    const uint32_t k = key_of(v);
                    if (!member(v, k, j)) return;
                    const int b = bin(v, k);
                    atomicAdd(&sh.count[b], 1u);
                    if (MASS) atomicAdd(&sh.mass[b], weight(v));
                });
            }
            __syncthreads();
            // a thread has PER bins; `own` what they hold
            u64 own = 0, all;
#pragma unroll
            for (int t = 0; t < PER; ++t) own += MASS ? sh.mass[tid * PER + t] : u64(sh.count[tid * PER + t]);
            u64 before = threads_before(own, all);
            if (binned) {   // (the last bin's weight is what the others leave)
                if (tid == THREADS - 1) sh.mass[kBins - 1] += total - all;
                all = total;
            }
            if (MASS && level == 0) need = share(p, all);
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
            need -= sh.before;
            auto inside = [&](float v, uint32_t k, int j) { return member(v, k, j) && bin(v, k) == b; };
            __syncthreads();   // (all have read)
            // list the bin's elements, as far as there is room
            uint32_t n = binned ? 0 : sh.count[b];
            if (binned || n <= uint32_t(kPairs)) {
                __syncthreads();   // (sh.count is read before it is cleared)
                if (tid < kPairs) sh.count[tid] = 0, sh.mass[tid] = 0;
                auto put = [&](float v, uint32_t k, int j) {
                    const uint32_t at = atomicAdd(&sh.n, 1u);
                    if (at < uint32_t(kPairs)) sh.list[at] = Entry{place_of(k, j), MASS ? weight(v) : 1};
                };
                if (binned && few()) {
                    u64 marks = 0;
#pragma unroll 1
                    for (int i = 0; i < slots; ++i) {
                        int at;
                        Piece<T> v;
                        if (!piece(i, at, v)) break;
                        marks |= u64(mark(v, [&](float x) { return x > -INFINITY && bin(x, 0) == b; })) << (i * VEC);
                    }
                    for (; marks; marks &= marks - 1) {
                        int j;
                        const float v = marked(__ffsll(marks) - 1, j);
                        put(v, key_of(v), j);
                    }
                } else {
                    each([&](float v, int j) {
                        const uint32_t k = key_of(v);
                        if (inside(v, k, j)) put(v, k, j);
                    });
                }
                __syncthreads();
                n = sh.n;
            }
            if (n <= uint32_t(kPairs)) {
                pairs<false>(int(n));
                __syncthreads();
                if (tid < int(n)) {
                    const u64 ahead = sh.mass[tid];
                    if (ahead < need && need <= ahead + sh.list[tid].w) sh.before = sh.list[tid].at;
                }
                __syncthreads();
                run.key = uint32_t(sh.before >> 32), run.last = int(~uint32_t(sh.before));
                __syncthreads();
                return;
            }
            uint32_t a = 0xffffffffu, z = 0;
            each([&](float v, int j) {
                const uint32_t k = key_of(v);
                if (inside(v, k, j)) a = min(a, k), z = max(z, k);
            });
            atomicMin(&sh.lo, a), atomicMax(&sh.hi, z);
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
    // What the run's weight has to reach: the share p of `all`, at least something
    __device__ __forceinline__ static u64 share(float p, u64 all) {
        bool more;
        const u64 t = fraction(fmaxf(p, 0.f), all, more);
        return max(t + more, u64(1));
    }

    // One pass over the row for what is wanted of it: the sum of exp(x - m); the sum of the
    // weights of all, the number of live ones, and the weights in bins (below); which elements
    // are at least `least` (a bit each, the first 64 of the thread's).
    struct Gathered {
        float e = 0.f;
        u64 mine = 0, marks = 0;
        uint32_t live = 0;
    };
    __device__ __forceinline__ Gathered gather(bool want_e, bool want_w, bool want_live, bool want_bins, float least) const {
        Gathered g;
        const float scale = bin_scale();
#pragma unroll 1
        for (int i = 0; i < slots; ++i) {
            int p;
            Piece<T> v;
            if (!piece(i, p, v)) break;
            if (want_e) {
#pragma unroll
                for (int j = 0; j < VEC; ++j) g.e += __builtin_amdgcn_exp2f((v.get(j) - m) * kLog2e);
            }
            if (want_bins) {
#pragma unroll
                for (int j = 0; j < VEC; ++j) {
                    const u64 w = weight(v.get(j));
                    const float b = (m - v.get(j)) * scale;
                    g.mine += w;
                    if (b < float(kBins - 1)) atomicAdd(&sh.mass[int(b)], w);
                }
            } else if (want_w) {
#pragma unroll
                for (int j = 0; j < VEC; ++j) g.mine += weight.raw(v.get(j));
                g.mine -= VEC * Weight::kOne;
            }
            if (want_live) {
#pragma unroll
                for (int j = 0; j < VEC; ++j) g.live += v.get(j) > -INFINITY;
            }
            if (least > -INFINITY) g.marks |= u64(mark(v, [&](float x) { return x >= least; })) << (i * VEC & 63);
        }
        return g;
    }
    // a bit for each of a piece's elements
    template <typename F>
    __device__ __forceinline__ uint32_t mark(const Piece<T>& v, F f) const {
        uint32_t bits = 0;
#pragma unroll
        for (int j = 0; j < VEC; ++j) bits |= f(v.get(j)) ? 1u << j : 0u;
        return bits;
    }
    // the thread's element of a bit, and its index
    __device__ __forceinline__ float marked(int bit, int& index) const {
        const int i = bit / VEC, j = bit % VEC, p = HELD ? first + i : first + i * 64;
        index = p * VEC + j;
        if constexpr (HELD) return to_f(reinterpret_cast<const T*>(&held_row[held_at(first, turn, i)])[j]);
        else return to_f(row[index]);
    }
    __device__ __forceinline__ bool few() const { return slots * VEC <= 64; }   // (a bit is one element)
    // Bins of weights: 1/32 of a power of two each, the last one all below 2^-32
    __device__ __forceinline__ float bin_scale() const { return 32.f * float(weight.c); }
    // Lists the marked elements (their number in sh.n, which may be more than there is room for)
    __device__ __forceinline__ void list(float least, u64 marks) const {
        const int lane = threadIdx.x & 63;
        uint32_t c = uint32_t(__popcll(marks));
        if (!few()) {   // (a bit may stand for two elements: all are looked at again)
            c = 0;
            if (marks) each([&](float v, int) { c += v >= least; });
        }
        const uint32_t up = up_to(c), sum = last_lane(up);
        if (sum) {
            uint32_t at = 0;
            if (lane == 0) at = atomicAdd(&sh.n, sum);
            at = uint32_t(__builtin_amdgcn_readfirstlane(int(at))) + up - c;
            auto put = [&](float v, int j) {
                if (at < uint32_t(THREADS)) sh.list[at].at = place_of(key_of(v), j);
                ++at;
            };
            if (!few()) {
                if (c)
                    each([&](float v, int j) {
                        if (v >= least) put(v, j);
                    });
            } else {
                for (; marks; marks &= marks - 1) {
                    int j;
                    const float v = marked(__ffsll(marks) - 1, j);
                    put(v, j);
                }
            }
        }
        __syncthreads();
    }
    // A value that at least k logits reach, and few more: the k-th largest of the threads' own
    // maxima, or a little less.  -inf where fewer than k threads have any.  The maxima's range is cut in
    // 64 bins, a lane of every wave has one; where many meet in the k-th's bin, that is cut again.
    __device__ __forceinline__ float reached_by(uint32_t k, float own, float low) const {
        const int lane = threadIdx.x & 63;
        float top = m;
        for (int level = 0;; ++level) {
            const float scale = 63.f / (top - low), b = (top - own) * scale;
            if (threadIdx.x < 65) sh.bins[threadIdx.x] = 0;
            __syncthreads();
            // (0 * inf, inf / inf: the last bin)
            if (own > -INFINITY && own <= top && own >= low) atomicAdd(&sh.bins[b < 63.f ? int(b) : 63], 1u);
            const uint32_t over = uint32_t(__popcll(__ballot(own > top)));
            if (lane == 0 && over) atomicAdd(&sh.bins[64], over);
            __syncthreads();
            const uint32_t c = sh.bins[lane], up = sh.bins[64] + up_to(c);
            __syncthreads();
            const u64 enough = __ballot(up >= k);
            if (!enough) return -INFINITY;
            const int at = __ffsll(enough) - 1;
            const uint32_t there = uint32_t(__builtin_amdgcn_readlane(int(c), at));
            // the bin's ends, moved outwards by what rounding may have put on its other side
            const float width = 1.f / scale, slack = 2e-6f * fmaxf(fabsf(top), fabsf(low));
            const float under = at == 63 ? low : fmaxf(low, top - float(at + 1) * width - slack);
            if (there <= 32 || level == 3 || !(width > 4.f * slack)) return under;
            top = fminf(top, top - float(at) * width + slack), low = under;
        }
    }
};

template <typename T, int THREADS, bool HELD>
__device__ __forceinline__ void sample_row(const SampleArgs& a, Sampler<T, THREADS, HELD>& s, Shared<THREADS>& sh, int r,
                                           bool more) {
    constexpr int WAVES = THREADS / 64;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const float temp = a.T_ ? a.T_[r] : a.T, p = a.p_ ? a.p_[r] : a.p, minp = a.minp_ ? a.minp_[r] : a.minp, u = a.u[r];
    int k = a.k_ ? a.k_[r] : a.k;
    auto answer = [&](int token, float logp, float drawn, int kept) {
        a.tokens[r] = token;
        if (a.logp) a.logp[r] = logp;
        if (a.draw_logp) a.draw_logp[r] = drawn;
        if (a.kept) a.kept[r] = kept;
    };

    // the largest logit of the thread and of the row, the smallest of the threads' largest
    float own;
    bool nan, holes;
    {
        uint4 pieces[kSlots<THREADS>];
        if (HELD) s.fetch(pieces);
        s.largest(pieces, own, nan, holes);
    }
    // The next row comes nearer while this one is worked on: a thread touches one line of 128 bytes
    // (in registers of its own the row took those of the work on this one).
    uint32_t touched = 0;
    if (more) {
        const uintptr_t from = reinterpret_cast<uintptr_t>(static_cast<const T*>(a.logits) + (r + int64_t(gridDim.x)) * a.ld);
        const uintptr_t at = ((from + 127) & ~uintptr_t(127)) + size_t(tid) * 128;
        if (at + 4 <= from + size_t(a.V) * sizeof(T)) touched = *reinterpret_cast<const uint32_t*>(at);
    }
    float m = wave_max(own), low = wave_max(own > -INFINITY ? -own : -INFINITY);
    nan = __ballot(nan) != 0, holes = __ballot(holes) != 0;
    if (lane == 0) sh.f[0][wave] = m, sh.f[1][wave] = low, sh.f[2][wave] = nan ? 2.f : holes ? 1.f : 0.f;
    for (int t = tid; t < kBins; t += THREADS) sh.count[t] = 0, sh.mass[t] = 0;
    if (tid == 0) sh.n = 0, sh.kept = 0, sh.live = 0, sh.total = 0, sh.kept_total = 0;
    const bool greedy = temp == 0.f, some = minp > 0.f && temp < INFINITY && !greedy, part = p < 1.f && !greedy;
    // (a border of log(min_p): long code, one wave's)
    if (some && wave == WAVES - 1) sh.depth = double(temp) * log_of(double(fminf(minp, 1.f)));
    __syncthreads();
    m = wave_max(lane < WAVES ? sh.f[0][lane] : -INFINITY), low = -wave_max(lane < WAVES ? sh.f[1][lane] : -INFINITY);
    const float found = wave_max(lane < WAVES ? sh.f[2][lane] : 0.f);
    nan = found == 2.f, holes = found == 1.f;
    if (nan || m == INFINITY || !(temp >= 0.f) || p != p || minp != minp || u != u) {
        if (tid == 0) answer(-1, NAN, NAN, 0);
        return;
    }
    if (m == -INFINITY) {
        if (tid == 0) answer(-1, -INFINITY, -INFINITY, 0);
        return;
    }
    s.m = m;
    s.weight.set(m, temp, a.bits);
    const float border = some ? __double2float_ru(double(m) + sh.depth) : -INFINITY;
    if (k >= a.V || greedy) k = 0;

    // what is kept is at least `least`
    const float least = greedy ? m : k > 0 ? (k <= THREADS ? s.reached_by(uint32_t(k), own, low) : -INFINITY) : border;
    const bool sum_all = !greedy && k <= 0 && (part || !some);   // the weight of all is wanted
    const bool exps = a.logp && !(sum_all && temp == 1.f);
    const bool bins = sum_all && part && !some;
    const auto g = s.gather(exps, sum_all, sum_all && a.kept && holes, bins, least);
    asm volatile("" ::"v"(touched));
    u64 mine = g.mine;
    uint32_t live = holes ? g.live : uint32_t(a.V);
    auto add_marked = [&](u64 marks) {
        mine = 0, live = uint32_t(__popcll(marks));
        for (; marks; marks &= marks - 1) {
            int j;
            mine += s.weight(s.marked(__ffsll(marks) - 1, j));
        }
    };
    // With min-p alone nothing has to be ranked: the marked weights are added up where they are
    // (2000 rows of 1000 bf16 logits, min_p 0.05: 14.6 us, through a list 32.5; 2000 of 32768: 72 and 150).
    // A mark of two elements would be looked at again: the list is no slower then where it is short.
    // Where the row is in memory a list is faster while it is short (kFewMarked).
    bool marked = least > -INFINITY && some && k <= 0 && !part && s.few();
    if (HELD) {
        if (marked) add_marked(g.marks);
    } else if (marked) {
        const uint32_t c = last_lane(up_to(uint32_t(__popcll(g.marks))));
        if (lane == 0 && c) atomicAdd(&sh.live, c);
        const bool early = c * WAVES > kFewMarked;   // (a wave that has many does not wait to know)
        if (early) add_marked(g.marks);
        __syncthreads();
        marked = sh.live > kFewMarked;
        if (marked && !early) add_marked(g.marks);
    }
    // sums of all, and of the threads before
    u64 all = 0, before = 0;
    if (sum_all) {
        const u64 up = up_to(mine);
        if (a.kept && holes) {
            const uint32_t c = last_lane(up_to(live));
            if (lane == 0 && c) atomicAdd(&sh.live, c);
        }
        all = s.over_waves(last_lane(up), before);
        before += up - mine;
        if (holes) live = sh.live;
    }
    float lse = 0.f;   // the (binary) logarithm of the sum of exp(x - m)
    if (exps) lse = __builtin_amdgcn_logf(s.over_waves_sum(g.e));
    else if (a.logp) lse = __builtin_amdgcn_logf(ldexpf(float(all), -a.bits));
    auto logp_of = [&](float x) { return fmaf(-lse, kLn2, x - m); };
    const float chance = fminf(fmaxf(u, 0.f), 1.f);
    auto target = [&](u64 sum) {   // the last whole number not above u sum, and below sum
        bool cut;
        return min(fraction(chance, sum, cut), sum - 1);
    };

    if (least > -INFINITY && !marked) {
        s.list(least, g.marks);
        const int n = int(sh.n);
        if (greedy && n <= kPairs) {   // the first of the largest
            if (tid >= 64) return;
            uint32_t j = 0;
            for (int i = tid; i < n; i += 64) j = max(j, uint32_t(sh.list[i].at));
            j = wave_scan(j, 0u, [](uint32_t a, uint32_t b) { return max(a, b); });
            if (tid == 63) answer(int(~j), logp_of(m), 0.f, 1);
            return;
        }
        if (n <= kPairs) {
            // (kPairs threads, and no more: the others would take their turns)
            const bool on = tid < kPairs;
            u64 at = 0, w = 0;
            uint32_t key = 0;
            if (on && tid < n) {
                at = sh.list[tid].at, key = uint32_t(at >> 32);
                sh.list[tid].w = w = s.weight(value_of(key));
            }
            __syncthreads();
            s.template pairs<false>(n);
            __syncthreads();
            bool in = tid < n && (k <= 0 || int(sh.count[tid]) < k);
            if (part && k > 0) {   // of the first k
                if (on) {
                    const u64 sum = last_lane(up_to(in ? w : 0));
                    if (lane == 0 && sum) atomicAdd(&sh.total, sum);
                }
                __syncthreads();
                all = sh.total;
            }
            if (on) {
                if (part) in = in && sh.mass[tid] < s.share(p, all);
                in = in && key >= key_of(border);
                if (!in) w = 0;
                const u64 sum = last_lane(up_to(w));
                const uint32_t kept = uint32_t(__popcll(__ballot(in)));
                if (lane == 0 && kept) atomicAdd(&sh.kept_total, sum), atomicAdd(&sh.kept, kept);
                if (tid < n) sh.list[tid].w = w, sh.mass[tid] = 0;
            }
            __syncthreads();
            s.template pairs<true>(n);
            __syncthreads();
            if (!in) return;
            const u64 t = target(sh.kept_total), c = sh.mass[tid];
            if (c <= t && t < c + w)
                answer(int(~uint32_t(at)), logp_of(value_of(key)), float(log_of(double(w) / double(sh.kept_total))), int(sh.kept));
            return;
        }
        if (greedy) {
            const int j = s.nth(key_of(m), 1);
            if (tid == 0) answer(j, logp_of(m), 0.f, 1);
            return;
        }
        if (n <= THREADS) {
            auto pow2 = [](int v) { return v <= 64 ? 64 : 1 << (32 - __clz(v - 1)); };
            u64 e = s.sorted(tid < n ? sh.list[tid].at : 0, pow2(n));
            const uint32_t key = uint32_t(e >> 32), place = uint32_t(e);   // (place: falls with the index)
            bool in = tid < n && (k <= 0 || tid < k);
            u64 w = in ? s.weight(value_of(key)) : 0, sum;
            const u64 ahead = s.threads_before(w, sum);
            in = in && key >= key_of(border) && (!part || ahead < s.share(p, k > 0 ? sum : all));
            u64 skip, W;
            const int kept = int(s.over_waves(u64(__popcll(__ballot(in))), skip));   // (the first ones)
            sh.list[tid] = Entry{u64(key), in ? w : 0};
            // in the order of the index
            e = s.sorted(in ? u64(place) << 32 | uint32_t(tid) : 0, pow2(kept));
            __syncthreads();
            const Entry one = tid < kept ? sh.list[uint32_t(e)] : Entry{0, 0};
            const u64 c = s.threads_before(one.w, W), t = target(W);
            if (c <= t && t < c + one.w)
                answer(int(~uint32_t(e >> 32)), logp_of(value_of(uint32_t(one.at))), float(log_of(double(one.w) / double(W))), kept);
            return;
        }
    }
    Run run;
    if (k > 0) {
        float bottom = -INFINITY;   // (of -x)
        live = 0;
        s.each([&](float x, int) {
            if (x > -INFINITY) ++live, bottom = fmaxf(bottom, -x);
        });
        u64 skip;
        const u64 n = s.over_waves(last_lane(up_to(live)), skip);
        bottom = wave_max(bottom);
        if (lane == 0) sh.f[0][wave] = bottom;
        __syncthreads();
        bottom = -wave_max(lane < WAVES ? sh.f[0][lane] : -INFINITY);
        __syncthreads();
        if (u64(k) < n) s.template shorten<false>(run, u64(k), 0.f, bottom, 0);
    }
    if (part) s.template shorten<true>(run, 0, p, 0.f, bins ? all : 0);
    if (some && key_of(border) > run.key) run.key = key_of(border), run.last = 0x7fffffff;

    auto kept = [&](float x, int j) { return x > -INFINITY && run.has(key_of(x), j); };
    if (!sum_all || part) {   // (else added up already)
        if (!marked && s.few()) {   // a fifth of the row or so: its weights alone
            u64 marks = 0;
#pragma unroll 1
            for (int i = 0; i < s.slots; ++i) {
                int p;
                Piece<T> v;
                if (!s.piece(i, p, v)) break;
                int j = p * Sampler<T, THREADS, HELD>::VEC;
                marks |= u64(s.mark(v, [&](float x) { return kept(x, j++); })) << (i * Sampler<T, THREADS, HELD>::VEC);
            }
            add_marked(marks);
        } else if (!marked) {
            mine = 0, live = 0;
            s.each([&](float x, int j) {
                const u64 w = s.weight(x);
                const bool in = kept(x, j);
                mine += in ? w : 0;
                live += in;
            });
        }
        const u64 up = up_to(mine);
        all = s.over_waves(last_lane(up), before);
        before += up - mine;
        u64 skip;
        live = uint32_t(s.over_waves(last_lane(up_to(live)), skip));
    }
    s.border(mine, before, target(all), [&](float x, int j) { return kept(x, j) ? s.weight(x) : 0; },
             [&](int j, float x, u64 w) { answer(j, logp_of(x), float(log_of(double(w) / double(all))), int(live)); });
}

// A workgroup takes every gridDim.x-th row.
template <typename T, int THREADS, bool HELD>
__global__ __launch_bounds__(THREADS, 4) void sample_kernel(SampleArgs a) {
    __shared__ Shared<THREADS> sh;
    for (int r = blockIdx.x; r < a.rows; r += gridDim.x) {
        Sampler<T, THREADS, HELD> s(static_cast<const T*>(a.logits) + r * a.ld, a.V, sh);
        sample_row(a, s, sh, r, HELD && int64_t(r) + gridDim.x < a.rows);
        __syncthreads();   // (the row in LDS and the lists are done with)
    }
}

bool sample_desc_ok(const janus_sample_desc* d) {
    return d && d->rows > 0 && d->V > 0 && (d->ld == 0 || d->ld >= d->V) && d->temperature >= 0.f &&
           !std::isnan(d->top_p) && !std::isnan(d->min_p);
}

constexpr int kDevices = 64;

// Compute units of the current device, and its number
janus_status device_cus(int& dev, int& cus) {
    static std::mutex lock;
    static int known[kDevices] = {};
    JANUS_HIP(hipGetDevice(&dev));
    if (dev < 0 || dev >= kDevices) return JANUS_ERR_UNSUPPORTED;
    std::lock_guard<std::mutex> guard(lock);
    if (!known[dev]) JANUS_HIP(hipDeviceGetAttribute(&known[dev], hipDeviceAttributeMultiprocessorCount, dev));
    cus = known[dev];
    return JANUS_OK;
}

template <typename T, int THREADS, bool HELD>
janus_status sample_launch(const SampleArgs& a, int64_t np, hipStream_t st) {
    int dev = 0, cus = 0;
    if (janus_status e = device_cus(dev, cus); e != JANUS_OK) return e;
    if (HELD && THREADS > 256) {   // (beyond 64 KB of LDS a kernel has to be told, once on each device)
        static std::mutex lock;
        static bool told[kDevices] = {};
        std::lock_guard<std::mutex> guard(lock);
        if (!told[dev])
            JANUS_HIP(hipFuncSetAttribute(reinterpret_cast<const void*>(sample_kernel<T, THREADS, HELD>),
                                          hipFuncAttributeMaxDynamicSharedMemorySize, int(held_bytes(kHeld))));
        told[dev] = true;
    }
    // 16 waves on a CU: what a workgroup of 1024 threads fills
    const int blocks = std::min(a.rows, cus * (1024 / THREADS));
    hipLaunchKernelGGL((sample_kernel<T, THREADS, HELD>), dim3(blocks), dim3(THREADS), HELD ? held_bytes(np) : 0, st, a);
    JANUS_LAUNCH_CHECK();
    return JANUS_OK;
}
template <typename T>
janus_status sample_dispatch(const SampleArgs& a, hipStream_t st) {
    const int64_t np = (int64_t(a.V) * sizeof(T) + 15) / 16;
    if (np <= kHeldSmall) return sample_launch<T, 256, true>(a, np, st);
    if (np <= kHeldMiddle) return sample_launch<T, 512, true>(a, np, st);
    if (np <= kHeld) return sample_launch<T, 1024, true>(a, np, st);
    return sample_launch<T, 1024, false>(a, np, st);
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
    return d->dtype == JANUS_BF16 ? sample_dispatch<bf16_t>(a, st) : sample_dispatch<float>(a, st);
}
