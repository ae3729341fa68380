// Selective scan over variable-length sequences: forward, backward, and the
// single-token step.
//
//   e = softplus(dt + dt_bias) (or dt + dt_bias),  u = e x
//   h_t[n] = exp(e A[n]) h_{t-1}[n] + u B_t[n]
//   y_t = (sum_n C_t[n] h_t[n] + Dskip x) silu(z)
//
// and backward, with gy = dy silu(z) and G_t[n] = dL/dh_t[n]:
//
//   G_t[n] = w_{t+1}[n] + gy C_t[n],   w_t[n] = G_t[n] exp(e A[n])
//   dC_t[n] = sum_d gy h_t[n],   dB_t[n] = sum_d G_t[n] u
//   s = sum_n G_t[n] B_t[n],  q[n] = w_t[n] h_{t-1}[n],  r = sum_n q[n] A[n]
//   dx = gy Dskip + e s,  de = x s + r,  dA[n] = sum q[n] e
//
// A wave owns 64 channels of one sequence and walks over time.  With few
// sequences the time axis is cut into segments: a first pass forms each
// segment's state from a zero start, a small kernel chains them (the decay over
// a segment is exp(A sum e)), and the second pass starts from the right state.
// States, decays and every sum over states, time or channels are float32.
//
// With 16 states the vector units bound it, not memory: a state takes 4 vector
// operations and an exponential a step forward, 13 and two backward (its state
// formed again, on which the backward of half a chunk spends 1.5 times that).
// Measured a wave: 2.7 cycles for an operation on vector registers where an even
// number of waves shares a SIMD (5.4 with one wave, 3.6 with three), 4.3 with a
// scalar or constant operand or a lane exchange, 8.3 for an exponential or a
// reciprocal.  So B and C come from LDS in vector registers and not from
// scalar ones.  Up to 16 states four waves stand on a SIMD: the forward takes 121
// registers, the backward is held to 128 (with 16 states and a gate it spills 8 of
// them).  Past 16 states there is room for two in the backward, past 32 for one.
// 65536 rows of 2048 bf16 channels, 16 states: forward 0.59 ms (0.27 of these
// operations alone), backward 1.83 ms (0.72), 1.1 and 1.5 TB/s.  25600 rows of
// 1024 channels: 0.14 and 0.39 ms with 16 states, 0.55 and 2.1 with 64.
#include <type_traits>

#include "seq.hpp"

namespace janus {
namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr int kMaxStates = 64;
constexpr int kStage = 32;    // steps whose B and C rows lie in LDS at once

// Steps between two kept states.  Fewer cost more bytes (a kept state is NP
// floats a channel), more cost the backward registers for the states between.
constexpr int chunk_steps(int NP) { return NP <= 32 ? 8 : 4; }
constexpr int kBwdWaves = 4;

struct ScanArgs {
    int32_t D, N, G, Dg, B, T;
    int32_t tiles, blocks;    // 64-channel tiles of a group, workgroups of a group
    int32_t btiles, bblocks;  // the backward's 32-channel tiles, and workgroups
    int32_t seg, nseg;        // steps per segment (a multiple of kStage), segments
    int64_t ldx, ldt, ldb, ldc, ldz, ldy;
    const void *x, *dt, *Bm, *Cm, *z;
    const float *A, *Dskip, *dtb, *h0;
    void* y;
    float* hT;
    float* ck;        // [chunks - 1][B][NP / 4][D][4] states at the chunks' starts, from the second on
    float* seg_h;     // [nseg][B][NP / 4][D][4] states at the segments' ends from a zero start, then at their starts
    float* seg_e;     // [nseg][B][D] sums of e
    // backward
    const void* dy;
    const float* dhT;
    void *dx, *ddt, *dz, *dBm, *dCm;
    float* dh0;
    float* seg_g;     // as seg_h, for G in reverse time
    float* dA_part;   // [nseg * B][D][N]
    float* dv_part;   // [nseg * B][2][D] sums of gy x and of ddt
    float* bc_part;   // [bblocks][T * B][G][2][NP], or NULL with one workgroup a group
    bool softplus;
    bool bc4;         // (step) four states of B and C are one aligned access
};

__device__ __forceinline__ float exp2_(float v) { return __builtin_amdgcn_exp2f(v); }

// log(1 + exp(v)) to a few ulp: with w = exp(-|v|) and s = 1 + w rounded,
// log1p(w) = log(s) w / (s - 1) (Goldberg, What Every Computer Scientist
// Should Know About Floating-Point Arithmetic, theorem 4)
__device__ __forceinline__ float softplus_(float v) {
    const float w = exp2_(-fabsf(v) * kLog2e), s = 1.f + w, m = s - 1.f;
    const float l = m == 0.f ? w : __builtin_amdgcn_logf(s) * kLn2 * w * __builtin_amdgcn_rcpf(m);
    return fmaxf(v, 0.f) + l;
}
__device__ __forceinline__ float step_size(float v, bool softplus) { return softplus ? softplus_(v) : v; }

// The same address in every lane, and known to the compiler as such: a load or
// store then takes it from scalar registers and only the lane's offset (32 bits)
// from a vector register.
template <typename P>
__device__ __forceinline__ P* uniform(P* p) {
    const uint64_t v = reinterpret_cast<uint64_t>(p);
    const uint32_t lo = __builtin_amdgcn_readfirstlane(uint32_t(v));
    const uint32_t hi = __builtin_amdgcn_readfirstlane(uint32_t(v >> 32));
    // (through a global pointer: an integer alone would make it a flat access)
    return (P*)(__attribute__((address_space(1))) P*)(uint64_t(hi) << 32 | lo);
}

// A value that the compiler takes for new where this stands, so that what is
// computed from it (addresses above all) is computed there and not held in
// registers from before the loop on.
__device__ __forceinline__ uint32_t fresh(uint32_t v) {
    asm volatile("" : "+v"(v));
    return v;
}

// [seg or chunk][b][quarter][d][4]
template <int NP>
__device__ __forceinline__ float* state_at(float* p, const ScanArgs& a, int64_t i, int b, int q, int d) {
    return p + (((i * a.B + b) * (NP / 4) + q) * a.D + d) * 4;
}

// Rows [t, t + n) of B and C as float32 in LDS, [step][B, C][NP]; zero past
// the sequence's end and past N.
template <typename T, int NP>
__device__ __forceinline__ void stage_bc(const ScanArgs& a, float* lds, int t, int n, int te, int b, int group) {
    for (int i = threadIdx.x; i < n * 2 * NP; i += blockDim.x) {
        const int st = i / (2 * NP), k = i % (2 * NP), m = k % NP;
        float v = 0.f;
        if (t + st < te && m < a.N) {
            const int64_t r = int64_t(t + st) * a.B + b;
            v = k < NP ? to_f(static_cast<const T*>(a.Bm)[r * a.ldb + int64_t(group) * a.N + m])
                       : to_f(static_cast<const T*>(a.Cm)[r * a.ldc + int64_t(group) * a.N + m]);
        }
        lds[i] = v;
    }
}

// A walk over the rows (t, b) of an operand: the row's address is uniform, and a
// lane adds its channel's byte offset (32 bits).
template <typename T>
struct Walk {
    char* row;
    int64_t step;
    uint32_t off;
    __device__ __forceinline__ Walk(const void* p, int64_t ld, int B, int b, int t, uint32_t d)
        : row(uniform(static_cast<char*>(const_cast<void*>(p)) + (int64_t(t) * B + b) * ld * int64_t(sizeof(T)))),
          step(int64_t(B) * ld * int64_t(sizeof(T))), off(d * uint32_t(sizeof(T))) {}
    __device__ __forceinline__ T get() const { return *reinterpret_cast<const T*>(row + fresh(off)); }
    __device__ __forceinline__ void put(T v) const { *reinterpret_cast<T*>(row + fresh(off)) = v; }
    // to the next row, or (at the end of what there is) not
    __device__ __forceinline__ void on(bool more = true) { row = uniform(row + (more ? step : 0)); }
    __device__ __forceinline__ void back(bool more = true) { row = uniform(row - (more ? step : 0)); }
};

// One lane per channel, its NP states in registers; B and C come from LDS, the
// same address in all lanes.  Eight steps at a time: their rows are loaded while
// the eight before are worked on (842 us before, 701 with; 65536 rows of 2048
// channels).  LOCAL: only the state at the segment's end
// from a zero start, and the sum of e.
template <typename T, int NP, bool LOCAL>
__global__ __launch_bounds__(256, 2) void scan_fwd_kernel(ScanArgs a, SeqSlice s) {
    constexpr int CK = chunk_steps(NP), U = NP >= 64 ? 4 : 8;
    __shared__ float bc[kStage * 2 * NP];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
    const int group = blockIdx.x / a.blocks, tile = (blockIdx.x % a.blocks) * waves + wave;
    const int ch = tile * 64 + lane;
    const bool live = ch < a.Dg;
    const uint32_t d = group * a.Dg + (live ? ch : 0);
    const int len = s.len[blockIdx.y], b = seq_of(s, blockIdx.y), seg = blockIdx.z;
    const int t0 = seg * a.seg, t1 = min(a.T, t0 + a.seg), te = min(t1, len);
    float A2[NP], h[NP];
#pragma unroll
    for (int n = 0; n < NP; ++n) {
        A2[n] = n < a.N ? a.A[d * a.N + n] * kLog2e : 0.f;
        h[n] = 0.f;
    }
    // (with segments the first one's start too is the chain's copy: h0 may be hT, which the last segment writes)
    if (!LOCAL && a.nseg > 1) {
#pragma unroll
        for (int q = 0; q < NP / 4; ++q) {
            const float4 v = *reinterpret_cast<const float4*>(state_at<NP>(a.seg_h, a, seg, b, q, d));
            h[4 * q] = v.x, h[4 * q + 1] = v.y, h[4 * q + 2] = v.z, h[4 * q + 3] = v.w;
        }
    } else if (!LOCAL && a.h0) {
#pragma unroll
        for (int n = 0; n < NP; ++n)
            if (n < a.N) h[n] = a.h0[(int64_t(b) * a.D + d) * a.N + n];
    }
    const float dskip = a.Dskip ? a.Dskip[d] : 0.f, dtb = a.dtb ? a.dtb[d] : 0.f;
    Walk<T> X(a.x, a.ldx, a.B, b, t0, d), DT(a.dt, a.ldt, a.B, b, t0, d), Z(a.z, a.ldz, a.B, b, t0, d),
        Y(a.y, a.ldy, a.B, b, t0, d);
    const bool gate = !LOCAL && a.z;
    float esum = 0.f;
    T nx[U], nt[U], nz[U];   // rows on their way (past the end: the last one again, not used)
    auto fetch = [&](int t) {
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const bool more = t + i + 1 < te;
            nx[i] = X.get();
            X.on(more);
            nt[i] = DT.get();
            DT.on(more);
            if (gate) {
                nz[i] = Z.get();
                Z.on(more);
            }
        }
    };
    if (t0 < te) fetch(t0);
    for (int ts = t0; ts < te; ts += kStage) {
        __syncthreads();
        stage_bc<T, NP>(a, bc, ts, kStage, te, b, group);
        __syncthreads();
        for (int tu = ts; tu < min(te, ts + kStage); tu += U) {
            // past the end e, u and the rows of B and C are 0: the state stays
            float x[U], e[U], z[U];
#pragma unroll
            for (int i = 0; i < U; ++i) {
                const bool on = tu + i < te;
                x[i] = on ? to_f(nx[i]) : 0.f;
                e[i] = on ? step_size(to_f(nt[i]) + dtb, a.softplus) : 0.f;
                if (gate) z[i] = to_f(nz[i]);
            }
            if (tu + U < te) fetch(tu + U);
            float y[U];
#pragma unroll
            for (int i = 0; i < U; ++i) {
                if (!LOCAL && i % CK == 0 && a.ck && tu + i > 0 && (tu + i) % CK == 0 && tu + i < te && live) {
                    float4* ck = reinterpret_cast<float4*>(uniform(state_at<NP>(a.ck, a, (tu + i) / CK - 1, b, 0, 0)));
                    const uint32_t df = fresh(d);
#pragma unroll
                    for (int q = 0; q < NP / 4; ++q)
                        ck[uint32_t(q) * a.D + df] = make_float4(h[4 * q], h[4 * q + 1], h[4 * q + 2], h[4 * q + 3]);
                }
                if (NP >= 64) __builtin_amdgcn_sched_barrier(0);   // (steps side by side would not fit the registers)
                const float u = e[i] * x[i];
                const float* row = bc + (tu + i - ts) * 2 * NP;
                y[i] = dskip * x[i];
#pragma unroll
                for (int n = 0; n < NP; ++n) {
                    h[n] = fmaf(exp2_(e[i] * A2[n]), h[n], u * row[n]);
                    if (!LOCAL) y[i] = fmaf(h[n], row[NP + n], y[i]);
                }
                if (LOCAL) esum += e[i];
            }
            if (!LOCAL) {
                if (gate) {
#pragma unroll
                    for (int i = 0; i < U; ++i) y[i] *= z[i] * sigmoidf_(z[i]);
                }
#pragma unroll
                for (int i = 0; i < U; ++i)
                    if (tu + i < te) {
                        if (live) Y.put(out_f<T>(y[i]));
                        Y.on();
                    }
            }
        }
    }
    if (!live) return;
    const uint32_t df = fresh(d);
    if (LOCAL) {
#pragma unroll
        for (int q = 0; q < NP / 4; ++q)
            *reinterpret_cast<float4*>(state_at<NP>(a.seg_h, a, seg, b, q, df)) =
                make_float4(h[4 * q], h[4 * q + 1], h[4 * q + 2], h[4 * q + 3]);
        a.seg_e[(int64_t(seg) * a.B + b) * a.D + df] = esum;
        return;
    }
    for (int t = max(t0, len); t < t1; ++t, Y.on()) Y.put(out_f<T>(0.f));
    if (a.hT && seg == a.nseg - 1) {
#pragma unroll
        for (int n = 0; n < NP; ++n)
            if (n < a.N) a.hT[(int64_t(b) * a.D + df) * a.N + n] = h[n];
    }
}

// LOCAL in the other direction: what flows from a segment into the one before
// it, from a zero end.
template <typename T, int NP>
__global__ __launch_bounds__(256, 2) void scan_rev_kernel(ScanArgs a, SeqSlice s) {
    constexpr int U = NP >= 64 ? 4 : 8;
    __shared__ float bc[kStage * 2 * NP];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
    const int group = blockIdx.x / a.blocks, tile = (blockIdx.x % a.blocks) * waves + wave;
    const int ch = tile * 64 + lane;
    const bool live = ch < a.Dg;
    const uint32_t d = group * a.Dg + (live ? ch : 0);
    const int len = s.len[blockIdx.y], b = seq_of(s, blockIdx.y), seg = blockIdx.z;
    const int t0 = seg * a.seg, te = min(min(a.T, t0 + a.seg), len);
    float A2[NP], g[NP];
#pragma unroll
    for (int n = 0; n < NP; ++n) {
        A2[n] = n < a.N ? a.A[int64_t(d) * a.N + n] * kLog2e : 0.f;
        g[n] = 0.f;
    }
    const float dtb = a.dtb ? a.dtb[d] : 0.f;
    const int last = max(te - 1, 0);
    Walk<T> DT(a.dt, a.ldt, a.B, b, last, d), Z(a.z, a.ldz, a.B, b, last, d), DY(a.dy, a.ldy, a.B, b, last, d);
    const bool gate = a.z;
    T nt[U], nz[U], ng[U];   // rows t - 1, t - 2, ... on their way (before the start: the first one again, not used)
    auto fetch = [&](int t) {
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const bool more = t - 2 - i >= t0;
            nt[i] = DT.get();
            DT.back(more);
            ng[i] = DY.get();
            DY.back(more);
            if (gate) {
                nz[i] = Z.get();
                Z.back(more);
            }
        }
    };
    if (t0 < te) fetch(te);
    const int n_stage = te > t0 ? (te - t0 + kStage - 1) / kStage : 0;
    for (int k = n_stage - 1; k >= 0; --k) {
        const int ts = t0 + k * kStage, tn = min(te, ts + kStage);
        __syncthreads();
        stage_bc<T, NP>(a, bc, ts, kStage, te, b, group);
        __syncthreads();
        for (int tu = tn; tu > ts; tu -= U) {   // steps tu - 1 down to tu - U
            const int n = min(U, tu - ts);
            float e[U], gy[U];
#pragma unroll
            for (int i = 0; i < U; ++i) {
                e[i] = i < n ? step_size(to_f(nt[i]) + dtb, a.softplus) : 0.f;
                gy[i] = i < n ? to_f(ng[i]) : 0.f;
                if (gate) {
                    const float z = to_f(nz[i]);
                    gy[i] *= z * sigmoidf_(z);
                }
            }
            if (n < U) {   // (a stage of fewer steps: only the last one in time; go on from its first row)
                DT = Walk<T>(a.dt, a.ldt, a.B, b, max(ts - 1, t0), d);
                DY = Walk<T>(a.dy, a.ldy, a.B, b, max(ts - 1, t0), d);
                Z = Walk<T>(a.z, a.ldz, a.B, b, max(ts - 1, t0), d);
            }
            if (tu - n > t0) fetch(tu - n);
#pragma unroll
            for (int i = 0; i < U; ++i) {
                if (i < n) {
                    const float* row = bc + (tu - 1 - i - ts) * 2 * NP + NP;
#pragma unroll
                    for (int m = 0; m < NP; ++m) g[m] = fmaf(gy[i], row[m], g[m]) * exp2_(e[i] * A2[m]);
                }
            }
        }
    }
    if (!live) return;
#pragma unroll
    for (int q = 0; q < NP / 4; ++q)
        *reinterpret_cast<float4*>(state_at<NP>(a.seg_g, a, seg, b, q, d)) =
            make_float4(g[4 * q], g[4 * q + 1], g[4 * q + 2], g[4 * q + 3]);
}

// Chains the segments.  forward: seg_h[i] becomes the state at segment i's
// start; reverse: seg_g[i] becomes what flows into segment i's end.  A lane has
// one state; the loads of 16 segments go out together.
template <int NP, bool REVERSE>
__global__ __launch_bounds__(256) void scan_chain_kernel(ScanArgs a) {
    const int64_t i = int64_t(blockIdx.x) * blockDim.x + threadIdx.x, size = int64_t(a.B) * NP * a.D;   // [B][NP / 4][D][4]
    if (i >= size) return;
    const int d = int(i / 4 % a.D), b = int(i / 4 / a.D / (NP / 4)), n = int(i / 4 / a.D % (NP / 4)) * 4 + int(i % 4);
    const float* first = REVERSE ? a.dhT : a.h0;
    const float A2 = n < a.N ? a.A[int64_t(d) * a.N + n] * kLog2e : 0.f;
    float h = n < a.N && first ? first[(int64_t(b) * a.D + d) * a.N + n] : 0.f;
    float* const p = (REVERSE ? a.seg_g : a.seg_h) + i;
    const float* const ep = a.seg_e + int64_t(b) * a.D + d;
    constexpr int U = 16;
    for (int k0 = 0; k0 < a.nseg; k0 += U) {
        float v[U], e[U];
#pragma unroll
        for (int k = 0; k < U; ++k) {
            const int seg = REVERSE ? max(a.nseg - 1 - k0 - k, 0) : min(k0 + k, a.nseg - 1);
            v[k] = p[seg * size];
            e[k] = ep[int64_t(seg) * a.B * a.D];
        }
#pragma unroll
        for (int k = 0; k < U; ++k)
            if (k0 + k < a.nseg) {
                p[(REVERSE ? a.nseg - 1 - k0 - k : k0 + k) * size] = h;
                h = fmaf(exp2_(e[k] * A2), h, v[k]);   // (past the last segment it is not used)
            }
    }
}

// ------------------------------------------------------------ lane exchange
template <int CTRL>
__device__ __forceinline__ float dpp(float v) {
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, true));
}
// Sums of a in the lanes of even 16-lane rows, of b in the odd ones, each over
// two neighbouring rows
__device__ __forceinline__ float fold16(float a, float b) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(a), __float_as_uint(b), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
// the same for the two halves of the wave
__device__ __forceinline__ float fold32(float a, float b) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(a), __float_as_uint(b), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
// M values summed over the 16 lanes of a row.  Where there are values left to
// share, each step leaves a lane with half of them (which half: a bit of the
// lane's number); then it sums.  Lane l ends with values first(l) + [0, max(1, M / 16)).
template <int M>
struct RowFold {
    static constexpr int left = M > 16 ? M / 16 : 1;
    template <int CTRL, int BIT, int m>
    __device__ __forceinline__ static void step(float* v, int lane) {
        if constexpr (m > 1) {
            const bool up = lane & BIT;
#pragma unroll
            for (int i = 0; i < m / 2; ++i) {
                const float keep = up ? v[i + m / 2] : v[i], give = up ? v[i] : v[i + m / 2];
                v[i] = keep + dpp<CTRL>(give);
            }
        } else {
            v[0] += dpp<CTRL>(v[0]);
        }
    }
    // row_ror:8 meets lane l ^ 8; row_half_mirror l ^ 7, whose bit 4 differs; then l ^ 2 and l ^ 1
    __device__ __forceinline__ static void run(float* v, int lane) {
        step<0x128, 8, M>(v, lane);
        step<0x141, 4, (M > 2 ? M / 2 : 1)>(v, lane);
        step<0x4e, 2, (M > 4 ? M / 4 : 1)>(v, lane);
        step<0xb1, 1, (M > 8 ? M / 8 : 1)>(v, lane);
    }
    __device__ __forceinline__ static int first(int lane) {
        int i = (lane & 8) ? M / 2 : 0;
        if (M > 2 && (lane & 4)) i += M / 4;
        if (M > 4 && (lane & 2)) i += M / 8;
        if (M > 8 && (lane & 1)) i += M / 16;
        return i;
    }
    // of the lanes with equal values, one writes them
    __device__ __forceinline__ static bool writes(int lane) {
        return M >= 16 || (lane & (M == 8 ? 1 : M == 4 ? 3 : 7)) == 0;
    }
};

// What was read from LDS before is read again after: keeps the compiler from
// holding a chunk's decays in registers beside its states.
__device__ __forceinline__ void forget_lds() { asm volatile("" ::: "memory"); }

// Rows (t, b) and (t + 1, b) of an operand: a uniform address, and the 32-bit
// byte offset of the lane's channel in the one or the other.
struct RowPair {
    int64_t step, base;    // bytes from row (t, b) to (t + 1, b), of row (0, b)
    uint32_t first, mine;  // the lane's channel in row t, in its half's row
    __device__ __forceinline__ RowPair(int64_t ld, int B, int b, int es, uint32_t d, int half)
        : step(int64_t(B) * ld * es), base(b * ld * es), first(d * es), mine(d * es + (half ? uint32_t(step) : 0u)) {}
    // both: there is a row t + 1
    template <typename T>
    __device__ __forceinline__ T* at(T* p, int t, bool both = true) const {
        char* row = uniform(reinterpret_cast<char*>(const_cast<std::remove_const_t<T>*>(p)) + base + t * step);
        return reinterpret_cast<T*>(row + fresh(both ? mine : first));
    }
};

// Backward of one segment.  A wave has 32 channels, 2 to a lane (lane l: channels
// 2 (l % 16) + [0, 2)), and the states in four parts over the wave's 16-lane
// rows, so that the sums over states and those over channels (for dB and dC)
// both lie half in-lane and half across lanes.  Two steps' sums over states are
// folded together, which leaves lane l with channel 2 (l % 16) + l / 16 % 2 of
// step l / 32: there it does the work per channel (step size, gate, loads and
// stores).  Values cross between the two layouts in LDS.  Chunks go backwards;
// the states inside one are formed again from its start.
template <typename T, int NP, bool GATE>
__global__ __launch_bounds__(64 * kBwdWaves, NP <= 16 ? 4 : NP == 32 ? 2 : 1) void scan_bwd_kernel(ScanArgs a, SeqSlice s) {
    constexpr int CK = chunk_steps(NP), NL = NP / 4, P = CK / 2, HK = CK / 2;
    __shared__ float bc[CK * 2 * NP];
    __shared__ float red[kBwdWaves][CK][2 * NP];
    __shared__ float sh[kBwdWaves][GATE ? 6 : 5][CK][32];   // e, u, gy, x, de/dv, and with a gate dy silu'(z)
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
    const int c16 = lane & 15, ng = lane >> 4;
    const int group = blockIdx.x / a.bblocks, blk = blockIdx.x % a.bblocks, ch0 = (blk * waves + wave) * 32;
    const int own = 2 * c16 + (ng & 1), half = ng >> 1;
    const bool live = ch0 + own < a.Dg;
    const uint32_t d = group * a.Dg + (live ? ch0 + own : 0);
    const int len = s.len[blockIdx.y], b = seq_of(s, blockIdx.y), seg = blockIdx.z;
    const int t0 = seg * a.seg, t1 = min(a.T, t0 + a.seg), lim = min(len, t1);
    float A2[2][NL], g[2][NL], dA[2][NL];
    // the lane's channels in the state layout: d2 + r for r < n2
    const uint32_t d2 = group * a.Dg + min(ch0 + 2 * c16, a.Dg - 1);
    const int n2 = a.Dg - (ch0 + 2 * c16);
    // its states in the rows [quarter][d][4] from p
    auto load_states = [&](const float* p, float (&v)[2][NL]) {
        const uint32_t df = fresh(d2);
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            const uint32_t dr = min(df + r, uint32_t(a.D - 1));
            if constexpr (NL >= 4) {
#pragma unroll
                for (int q = 0; q < NL / 4; ++q) {
                    const float4 f = reinterpret_cast<const float4*>(p)[uint32_t(ng * (NL / 4) + q) * a.D + dr];
                    v[r][4 * q] = f.x, v[r][4 * q + 1] = f.y, v[r][4 * q + 2] = f.z, v[r][4 * q + 3] = f.w;
                }
            } else {
#pragma unroll
                for (int i = 0; i < NL; ++i) {
                    const int n = ng * NL + i;
                    v[r][i] = p[(uint32_t(n / 4) * a.D + dr) * 4 + n % 4];
                }
            }
#pragma unroll
            for (int i = 0; i < NL; ++i) v[r][i] = r < n2 ? v[r][i] : 0.f;
        }
    };
    // the same from a dense [D, N], 0 where it is NULL
    auto load_dense = [&](const float* p, float (&v)[2][NL]) {
        const uint32_t df = fresh(d2);
#pragma unroll
        for (int r = 0; r < 2; ++r)
#pragma unroll
            for (int i = 0; i < NL; ++i)
                v[r][i] = p && r < n2 && ng * NL + i < a.N ? p[(df + r) * a.N + ng * NL + i] : 0.f;
    };
    load_dense(a.A, A2);
#pragma unroll
    for (int r = 0; r < 2; ++r)
#pragma unroll
        for (int i = 0; i < NL; ++i) A2[r][i] *= kLog2e, dA[r][i] = 0.f;
    const int64_t bstate = int64_t(b) * a.D * a.N;
    if (a.nseg > 1) load_states(uniform(state_at<NP>(a.seg_g, a, seg, b, 0, 0)), g);
    else load_dense(a.dhT ? a.dhT + bstate : nullptr, g);
    const float dskip = a.Dskip ? a.Dskip[d] : 0.f, dtb = a.dtb ? a.dtb[d] : 0.f;
    const T *X = static_cast<const T*>(a.x), *DT = static_cast<const T*>(a.dt), *Z = static_cast<const T*>(a.z),
            *DY = static_cast<const T*>(a.dy);
    T *DX = static_cast<T*>(a.dx), *DDT = static_cast<T*>(a.ddt), *DZ = static_cast<T*>(a.dz);
    const RowPair rx(a.ldx, a.B, b, sizeof(T), d, half), rt(a.ldt, a.B, b, sizeof(T), d, half),
        rz(a.ldz, a.B, b, sizeof(T), d, half), ry(a.ldy, a.B, b, sizeof(T), d, half);
    float dD = 0.f, dtbs = 0.f;
    for (int tc = t0 + (t1 - 1 - t0) / CK * CK; tc >= t0; tc -= CK) {
        const int tn = min(CK, t1 - tc);
        if (tc < len) {
            T vx[P], vt[P], vg[P], vz[P];   // (past the end: the last row's values, not used)
#pragma unroll
            for (int i = 0; i < P; ++i) {
                const int t = min(tc + 2 * i, lim - 1);
                const bool both = tc + 2 * i + 1 < lim;
                vx[i] = *rx.at(X, t, both);
                vt[i] = *rt.at(DT, t, both);
                vg[i] = *ry.at(DY, t, both);
                if (GATE) vz[i] = *rz.at(Z, t, both);
            }
#pragma unroll
            for (int i = 0; i < P; ++i) {
                const int k = 2 * i + half;
                const bool on = tc + k < lim && live;
                const float x = on ? to_f(vx[i]) : 0.f, v = to_f(vt[i]) + dtb;
                const float e = on ? step_size(v, a.softplus) : 0.f;
                float gy = on ? to_f(vg[i]) : 0.f;
                sh[wave][3][k][own] = x;
                sh[wave][4][k][own] = !on ? 0.f : a.softplus ? sigmoidf_(v) : 1.f;
                if (GATE) {
                    const float z = on ? to_f(vz[i]) : 0.f, q = sigmoidf_(z);
                    sh[wave][GATE ? 5 : 0][k][own] = gy * q * (1.f + z * (1.f - q));
                    gy *= z * q;
                }
                sh[wave][0][k][own] = e;
                sh[wave][1][k][own] = e * x;
                sh[wave][2][k][own] = gy;
            }
            stage_bc<T, NP>(a, bc, tc, CK, lim, b, group);
        }
        __syncthreads();
        if (tc < len) {
            // Half a chunk at a time, the later one first: h[i] is the state before the half's step i.  (The
            // earlier half's steps run twice; holding a whole chunk's states would leave two waves a SIMD.)
            float h[HK + 1][2][NL];
            auto load_start = [&] {
                if (tc > 0) load_states(uniform(state_at<NP>(a.ck, a, tc / CK - 1, b, 0, 0)), h[0]);
                else load_dense(a.h0 ? a.h0 + bstate : nullptr, h[0]);
            };
            load_start();
            auto advance = [&](int k, const float (&from)[2][NL], float (&to)[2][NL]) {
                __builtin_amdgcn_sched_barrier(0);
                const float2 e2 = *reinterpret_cast<const float2*>(&sh[wave][0][k][2 * c16]);
                const float2 u2 = *reinterpret_cast<const float2*>(&sh[wave][1][k][2 * c16]);
                const float e[2] = {e2.x, e2.y}, u[2] = {u2.x, u2.y};
#pragma unroll
                for (int i = 0; i < NL; ++i) {
                    const float bn = bc[k * 2 * NP + ng * NL + i];
#pragma unroll
                    for (int r = 0; r < 2; ++r) to[r][i] = fmaf(exp2_(e[r] * A2[r][i]), from[r][i], u[r] * bn);
                }
            };
#pragma unroll
            for (int k = 0; k < CK - HK; ++k) advance(k, h[0], h[0]);
            float odd[3];   // the odd step's sums over states, folded once
#pragma unroll
            for (int k0 = CK - HK; k0 >= 0; k0 -= HK) {
            if (k0 == 0) load_start();
            forget_lds();
#pragma unroll
            for (int k = 0; k < HK; ++k) advance(k0 + k, h[k], h[k + 1]);
            forget_lds();
#pragma unroll
            for (int k = k0 + HK - 1; k >= k0; --k) {
                __builtin_amdgcn_sched_barrier(0);
                // Past the end G stays; the sums would be 0 times what may be infinite.  (Said to be unlikely: otherwise
                // the compiler's order of the code costs the backward 2 %.)
                if (__builtin_expect(tc + k >= lim, 0)) {
                    odd[0] = odd[1] = odd[2] = 0.f;
                    continue;
                }
                const float2 e2 = *reinterpret_cast<const float2*>(&sh[wave][0][k][2 * c16]);
                const float2 u2 = *reinterpret_cast<const float2*>(&sh[wave][1][k][2 * c16]);
                const float2 g2 = *reinterpret_cast<const float2*>(&sh[wave][2][k][2 * c16]);
                const float e[2] = {e2.x, e2.y}, u[2] = {u2.x, u2.y}, gy[2] = {g2.x, g2.y};
                float bcs[2 * NL], sb[2] = {}, sa[2] = {}, yr[2] = {};
#pragma unroll
                for (int i = 0; i < 2 * NL; ++i) bcs[i] = 0.f;
#pragma unroll
                for (int i = 0; i < NL; ++i) {
                    const float bn = bc[k * 2 * NP + ng * NL + i], cn = bc[k * 2 * NP + NP + ng * NL + i];
#pragma unroll
                    for (int r = 0; r < 2; ++r) {
                        const float gn = fmaf(gy[r], cn, g[r][i]);
                        bcs[NL + i] = fmaf(gy[r], h[k - k0 + 1][r][i], bcs[NL + i]);
                        bcs[i] = fmaf(gn, u[r], bcs[i]);
                        sb[r] = fmaf(gn, bn, sb[r]);
                        if (GATE) yr[r] = fmaf(h[k - k0 + 1][r][i], cn, yr[r]);
                        const float w = gn * exp2_(e[r] * A2[r][i]), q = w * h[k - k0][r][i];
                        sa[r] = fmaf(q, A2[r][i], sa[r]);
                        dA[r][i] = fmaf(q, e[r], dA[r][i]);
                        g[r][i] = w;
                    }
                }
                // (left alone, the compiler puts dA off to the chunk's end and keeps every step's terms)
#pragma unroll
                for (int r = 0; r < 2; ++r)
#pragma unroll
                    for (int i = 0; i < NL; ++i) asm volatile("" : "+v"(dA[r][i]));
                RowFold<2 * NL>::run(bcs, lane);
                if (RowFold<2 * NL>::writes(lane)) {
                    const int f = RowFold<2 * NL>::first(c16);
#pragma unroll
                    for (int j = 0; j < RowFold<2 * NL>::left; ++j) {
                        const int m = f + j;   // states NL of dB, then of dC
                        red[wave][k][(m < NL ? 0 : NP - NL) + ng * NL + m] = bcs[j];
                    }
                }
                const float fs = fold16(sb[0], sb[1]), fa = fold16(sa[0], sa[1]), fy = GATE ? fold16(yr[0], yr[1]) : 0.f;
                if (k & 1) {
                    odd[0] = fs, odd[1] = fa, odd[2] = fy;
                } else {
                    const float S = fold32(fs, odd[0]), R = fold32(fa, odd[1]) * kLn2;
                    const float oe = sh[wave][0][k + half][own], ogy = sh[wave][2][k + half][own];
                    const float x = sh[wave][3][k + half][own], ddt = (x * S + R) * sh[wave][4][k + half][own];
                    dD += ogy * x;
                    dtbs += ddt;
                    float dz = 0.f;
                    if (GATE) dz = sh[wave][GATE ? 5 : 0][k + half][own] * fmaf(dskip, x, fold32(fy, odd[2]));
                    if (tc + k + half < lim && live) {
                        *rx.at(DX, tc + k) = out_f<T>(fmaf(ogy, dskip, oe * S));
                        *rt.at(DDT, tc + k) = out_f<T>(ddt);
                        if (GATE) *rz.at(DZ, tc + k) = out_f<T>(dz);
                    }
                }
            }
            }
        }
        const bool ends = lim < tc + tn;
        if (__builtin_expect(ends, 0) && live) {   // 0 in the rows past the sequence's end
            for (int k = max(lim - tc, 0) & ~1; k < tn; k += 2) {
                if (tc + k + half < lim || k + half >= tn) continue;
                *rx.at(DX, tc + k) = out_f<T>(0.f);
                *rt.at(DDT, tc + k) = out_f<T>(0.f);
                if (GATE) *rz.at(DZ, tc + k) = out_f<T>(0.f);
            }
        }
        __syncthreads();
        for (int i = fresh(threadIdx.x); i < tn * 2 * NP; i += blockDim.x) {
            const int k = i / (2 * NP), m = i % (2 * NP), n = m % NP;
            float v = 0.f;
            if (tc + k < len)
                for (int w = 0; w < waves; ++w) v += red[w][k][m];
            const int64_t r = int64_t(tc + k) * a.B + b;
            if (a.bc_part) {
                a.bc_part[((int64_t(blk) * a.T * a.B + r) * a.G + group) * 2 * NP + m] = v;
            } else if (n < a.N) {
                if (m < NP) static_cast<T*>(a.dBm)[r * a.ldb + int64_t(group) * a.N + n] = out_f<T>(v);
                else static_cast<T*>(a.dCm)[r * a.ldc + int64_t(group) * a.N + n] = out_f<T>(v);
            }
        }
    }
    const int64_t part = int64_t(seg) * a.B + b;
    const uint32_t df = fresh(d2);
#pragma unroll
    for (int r = 0; r < 2; ++r)
#pragma unroll
        for (int i = 0; i < NL; ++i) {
            const int n = ng * NL + i;
            if (r >= n2 || n >= a.N) continue;
            a.dA_part[(part * a.D + df + r) * a.N + n] = dA[r][i];
            if (a.dh0 && seg == 0) a.dh0[bstate + int64_t(df + r) * a.N + n] = g[r][i];
        }
    dD += __shfl_xor(dD, 32, 64);
    dtbs += __shfl_xor(dtbs, 32, 64);
    if (live && half == 0) {
        a.dv_part[part * 2 * a.D + d] = dD;
        a.dv_part[(part * 2 + 1) * a.D + d] = dtbs;
    }
}

// dA, dDskip, ddt_bias: 64 values at a time a workgroup, each wave sums every
// 16th part, then the waves' sums in their order.
__global__ __launch_bounds__(1024) void scan_param_kernel(const float* dA_part, const float* dv_part, int parts, int D,
                                                          int N, float* dA, float* dD, float* ddtb) {
    __shared__ float red[16][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t na = int64_t(D) * N, all = na + 2 * int64_t(D);
    for (int64_t i0 = int64_t(blockIdx.x) * 64; i0 < all; i0 += int64_t(gridDim.x) * 64) {
        const int64_t i = i0 + lane;
        const bool on = i < all;
        const float* p = i < na ? dA_part + i : dv_part + (i - na);
        const int64_t step = i < na ? na : 2 * int64_t(D);
        float v = 0.f;
        if (on)
            for (int k = wave; k < parts; k += 16) v += p[k * step];
        red[wave][lane] = v;
        __syncthreads();
        if (wave == 0 && on) {
            for (int w = 1; w < 16; ++w) v += red[w][lane];
            if (i < na) dA[i] = v;
            else if (i < na + D) {
                if (dD) dD[i - na] = v;
            } else if (ddtb) {
                ddtb[i - na - D] = v;
            }
        }
        __syncthreads();
    }
}

// dB and dC: the workgroups' parts of each row
template <typename T, int NP>
__global__ __launch_bounds__(256) void scan_bc_kernel(ScanArgs a) {
    const int64_t rows = int64_t(a.T) * a.B, all = rows * a.G * 2 * NP;
    for (int64_t i = int64_t(blockIdx.x) * blockDim.x + threadIdx.x; i < all; i += int64_t(gridDim.x) * blockDim.x) {
        const int m = int(i % (2 * NP)), n = m % NP, group = int(i / (2 * NP) % a.G);
        const int64_t row = i / (2 * NP) / a.G;
        if (n >= a.N) continue;
        float v = 0.f;
        for (int k = 0; k < a.bblocks; ++k) v += a.bc_part[k * all + i];
        if (m < NP) static_cast<T*>(a.dBm)[row * a.ldb + int64_t(group) * a.N + n] = out_f<T>(v);
        else static_cast<T*>(a.dCm)[row * a.ldc + int64_t(group) * a.N + n] = out_f<T>(v);
    }
}

// One token: QL lanes per channel with 4 states each.  Bound by the states' bytes:
// 256 rows of 4096 channels, 16 states, 29 us (143 MB: 4.9 TB/s).
template <typename T, int QL, bool VEC4>
__global__ __launch_bounds__(256) void scan_step_kernel(ScanArgs a, const int32_t* slots, int32_t n_slots,
                                                        float* state) {
    const int i = blockIdx.x * blockDim.x + threadIdx.x, q = i % QL, d0 = i / QL, b = blockIdx.y;
    const bool live = d0 < a.D;
    const int d = live ? d0 : 0;
    const int slot = slots ? slots[b] : b;
    T* yp = static_cast<T*>(a.y) + b * a.ldy + d;
    if (slot < 0 || slot >= n_slots) {
        if (live && q == 0) *yp = out_f<T>(0.f);
        return;
    }
    const int n0 = 4 * q, group = d / a.Dg;
    float* sp = state + (int64_t(slot) * a.D + d) * a.N + n0;
    float h[4] = {}, A[4] = {}, bn[4] = {}, cn[4] = {};
    const float* ap = a.A + int64_t(d) * a.N + n0;
    const T* bp = static_cast<const T*>(a.Bm) + b * a.ldb + int64_t(group) * a.N + n0;
    const T* cp = static_cast<const T*>(a.Cm) + b * a.ldc + int64_t(group) * a.N + n0;
    if (VEC4) {
        if (n0 < a.N) {
            const float4 v = *reinterpret_cast<const float4*>(sp), w = *reinterpret_cast<const float4*>(ap);
            h[0] = v.x, h[1] = v.y, h[2] = v.z, h[3] = v.w;
            A[0] = w.x, A[1] = w.y, A[2] = w.z, A[3] = w.w;
        }
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (n0 + j < a.N) h[j] = sp[j], A[j] = ap[j];
    }
    if (VEC4 && a.bc4) {
        if (n0 < a.N) {
            Chan<T, 4> rb, rc;
            rb.load(bp);
            rc.load(cp);
            rb.get(bn);
            rc.get(cn);
        }
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (n0 + j < a.N) bn[j] = to_f(bp[j]), cn[j] = to_f(cp[j]);
    }
    const float x = to_f(static_cast<const T*>(a.x)[b * a.ldx + d]);
    const float e = step_size(to_f(static_cast<const T*>(a.dt)[b * a.ldt + d]) + (a.dtb ? a.dtb[d] : 0.f), a.softplus);
    float y = 0.f;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        h[j] = fmaf(exp2_(e * A[j] * kLog2e), h[j], e * x * bn[j]);
        y = fmaf(h[j], cn[j], y);
    }
    if (live) {
        if (VEC4) {
            if (n0 < a.N) *reinterpret_cast<float4*>(sp) = make_float4(h[0], h[1], h[2], h[3]);
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (n0 + j < a.N) sp[j] = h[j];
        }
    }
#pragma unroll
    for (int o = QL / 2; o > 0; o >>= 1) y += __shfl_xor(y, o, 64);
    if (live && q == 0) {
        y = fmaf(a.Dskip ? a.Dskip[d] : 0.f, x, y);
        if (a.z) {
            const float z = to_f(static_cast<const T*>(a.z)[b * a.ldz + d]);
            y *= z * sigmoidf_(z);
        }
        *yp = out_f<T>(y);
    }
}

// -------------------------------------------------------------------- host
bool scan_desc_ok(const janus_scan_desc* d) {
    if (!d || d->D <= 0 || d->N <= 0 || d->G <= 0 || d->B <= 0 || d->T < 0 || d->D % d->G != 0) return false;
    for (int64_t ld : {d->ldx, d->ldt, d->ldz, d->ldy})
        if (ld != 0 && ld < d->D) return false;
    for (int64_t ld : {d->ldb, d->ldc})
        if (ld != 0 && ld < int64_t(d->G) * d->N) return false;
    return true;
}
bool scan_supported(const janus_scan_desc* d) {
    return dtype_ok(d->dtype) && d->N <= kMaxStates && (d->flags & ~(JANUS_SCAN_SOFTPLUS | JANUS_SCAN_KEEP)) == 0 &&
           d->T <= (1 << 30) && d->D <= (1 << 22) && d->B <= (1 << 24) &&
           std::max({d->ldx, d->ldt, d->ldz, d->ldy, int64_t(d->D)}) <= (int64_t(1) << 29) / d->B;
}
// states rounded up to what the kernels are built for
int padded_states(int N) { return N <= 4 ? 4 : N <= 8 ? 8 : N <= 16 ? 16 : N <= 32 ? 32 : 64; }

constexpr int kScanWaves = 4;

// The geometry of a descriptor: a function of it alone, so that the forward,
// the backward and the workspace agree.
ScanArgs scan_geometry(const janus_scan_desc* d) {
    ScanArgs a{};
    a.D = d->D, a.N = d->N, a.G = d->G, a.Dg = d->D / d->G, a.B = d->B, a.T = d->T;
    a.ldx = d->ldx ? d->ldx : d->D, a.ldt = d->ldt ? d->ldt : d->D, a.ldz = d->ldz ? d->ldz : d->D;
    a.ldy = d->ldy ? d->ldy : d->D;
    a.ldb = d->ldb ? d->ldb : int64_t(d->G) * d->N, a.ldc = d->ldc ? d->ldc : int64_t(d->G) * d->N;
    a.softplus = d->flags & JANUS_SCAN_SOFTPLUS;
    a.tiles = (a.Dg + 63) / 64;
    a.blocks = (a.tiles + kScanWaves - 1) / kScanWaves;
    a.btiles = (a.Dg + 31) / 32;
    a.bblocks = (a.btiles + kBwdWaves - 1) / kBwdWaves;
    // With fewer waves than the chip's 1024 SIMDs the time axis is cut, into segments of 64 steps
    // and more, for four waves a SIMD.  The cut costs a second pass over the inputs: one prompt of
    // 8192 steps and 2048 channels takes 32 waves 4.1 ms in one piece, 0.17 ms in 128.
    const int64_t waves = int64_t(a.B) * a.G * a.tiles;
    int64_t want = 1;
    if (waves < 1024) want = std::max<int64_t>(1, std::min<int64_t>((4096 + waves - 1) / waves, a.T / 64));
    a.seg = int(std::max<int64_t>(kStage, round_up((a.T + want - 1) / want, kStage)));
    a.nseg = std::max(1, (a.T + a.seg - 1) / a.seg);
    return a;
}
// workspace regions (sizes only with ws NULL)
size_t scan_carve(ScanArgs& a, bool keep, void* ws) {
    const int NP = padded_states(a.N), CK = chunk_steps(NP);
    const size_t state = size_t(a.B) * NP * a.D;
    Carver c(ws);
    if (a.nseg > 1) {
        a.seg_h = c.take<float>(a.nseg * state);
        a.seg_e = c.take<float>(size_t(a.nseg) * a.B * a.D);
    }
    if (keep) {
        const size_t chunks = size_t((a.T + CK - 1) / CK), parts = size_t(a.nseg) * a.B;
        a.ck = c.take<float>((chunks ? chunks - 1 : 0) * state);
        if (a.nseg > 1) a.seg_g = c.take<float>(a.nseg * state);
        a.dA_part = c.take<float>(parts * a.D * a.N);
        a.dv_part = c.take<float>(parts * 2 * a.D);
        if (a.bblocks > 1) a.bc_part = c.take<float>(size_t(a.bblocks) * a.T * a.B * a.G * 2 * NP);
    }
    return c.off;
}
janus_status scan_check(const janus_scan_desc* d, const void* x, const void* dt, const float* A, const void* Bm,
                        const void* Cm, const float* Dskip, const void* z, const float* dt_bias, const void* y,
                        bool rows) {
    if (!scan_desc_ok(d) || !A || (rows && (!x || !dt || !Bm || !Cm || !y))) return JANUS_ERR_INVALID_ARG;
    if (!scan_supported(d)) return JANUS_ERR_UNSUPPORTED;
    const size_t es = dtype_size(d->dtype);
    for (const void* p : {x, dt, Bm, Cm, z, y})
        if (!aligned(p, es)) return JANUS_ERR_INVALID_ARG;
    for (const float* p : {A, Dskip, dt_bias})
        if (!aligned(p, 4)) return JANUS_ERR_INVALID_ARG;
    if (y && (y == x || y == dt || y == z || y == Bm || y == Cm)) return JANUS_ERR_INVALID_ARG;
    return JANUS_OK;
}
void scan_inputs(ScanArgs& a, const void* x, const void* dt, const float* A, const void* Bm, const void* Cm,
                 const float* Dskip, const void* z, const float* dt_bias) {
    a.x = x, a.dt = dt, a.A = A, a.Bm = Bm, a.Cm = Cm, a.Dskip = Dskip, a.z = z, a.dtb = dt_bias;
}

// A launch holds fewer than 2^32 threads; kernels of more loop.
dim3 launch_blocks(int64_t blocks, int threads) { return dim3(std::min<int64_t>(blocks, (int64_t(1) << 31) / threads)); }

dim3 scan_block(const ScanArgs& a) { return dim3(64 * std::min(kScanWaves, a.tiles)); }

template <typename T, int NP>
janus_status scan_fwd_run(const ScanArgs& a, const int32_t* lengths, hipStream_t st) {
    const double el = double(a.T) * a.B * a.D;
    if (a.nseg > 1) {
        for (int32_t b0 = 0; b0 < a.B; b0 += kSlice) {
            SeqSlice s;
            const int n = fill_slice(s, b0, a.B, a.T, lengths);
            TraceScope trace("scan_fwd_local", el / a.B * n * 5 * a.N, el / a.B * n * 2 * sizeof(T), st);
            hipLaunchKernelGGL((scan_fwd_kernel<T, NP, true>), dim3(a.blocks * a.G, n, a.nseg), scan_block(a), 0, st, a,
                               s);
            JANUS_LAUNCH_CHECK();
        }
        const int64_t all = int64_t(a.B) * NP * a.D;
        TraceScope trace("scan_chain", 2.0 * all * a.nseg, 9.0 * all * a.nseg, st);
        hipLaunchKernelGGL((scan_chain_kernel<NP, false>), dim3((all + 255) / 256), dim3(256), 0, st, a);
        JANUS_LAUNCH_CHECK();
    }
    for (int32_t b0 = 0; b0 < a.B; b0 += kSlice) {
        SeqSlice s;
        const int n = fill_slice(s, b0, a.B, a.T, lengths);
        TraceScope trace("scan_fwd", el / a.B * n * 7 * a.N, el / a.B * n * (a.z ? 4 : 3) * sizeof(T), st);
        hipLaunchKernelGGL((scan_fwd_kernel<T, NP, false>), dim3(a.blocks * a.G, n, a.nseg), scan_block(a), 0, st, a, s);
        JANUS_LAUNCH_CHECK();
    }
    return JANUS_OK;
}

template <typename T, int NP>
janus_status scan_bwd_run(const ScanArgs& a, const int32_t* lengths, float* dA, float* dDskip, float* ddt_bias,
                          hipStream_t st) {
    const double el = double(a.T) * a.B * a.D;
    if (a.nseg > 1) {
        for (int32_t b0 = 0; b0 < a.B; b0 += kSlice) {
            SeqSlice s;
            const int n = fill_slice(s, b0, a.B, a.T, lengths);
            TraceScope trace("scan_bwd_local", el / a.B * n * 5 * a.N, el / a.B * n * 3 * sizeof(T), st);
            hipLaunchKernelGGL((scan_rev_kernel<T, NP>), dim3(a.blocks * a.G, n, a.nseg), scan_block(a), 0, st, a, s);
            JANUS_LAUNCH_CHECK();
        }
        const int64_t all = int64_t(a.B) * NP * a.D;
        TraceScope trace("scan_chain", 2.0 * all * a.nseg, 9.0 * all * a.nseg, st);
        hipLaunchKernelGGL((scan_chain_kernel<NP, true>), dim3((all + 255) / 256), dim3(256), 0, st, a);
        JANUS_LAUNCH_CHECK();
    }
    for (int32_t b0 = 0; b0 < a.B; b0 += kSlice) {
        SeqSlice s;
        const int n = fill_slice(s, b0, a.B, a.T, lengths);
        TraceScope trace("scan_bwd", el / a.B * n * 24 * a.N, el / a.B * n * (a.z ? 7 : 5) * sizeof(T), st);
        const dim3 grid(a.bblocks * a.G, n, a.nseg), block(64 * std::min(kBwdWaves, a.btiles));
        if (a.z) hipLaunchKernelGGL((scan_bwd_kernel<T, NP, true>), grid, block, 0, st, a, s);
        else hipLaunchKernelGGL((scan_bwd_kernel<T, NP, false>), grid, block, 0, st, a, s);
        JANUS_LAUNCH_CHECK();
    }
    const int64_t np = int64_t(a.D) * a.N + 2 * a.D;
    {
        const int parts = a.nseg * a.B;
        TraceScope trace("scan_param", double(np) * parts, 4.0 * np * parts, st);
        hipLaunchKernelGGL(scan_param_kernel, launch_blocks((np + 63) / 64, 1024), dim3(1024), 0, st, a.dA_part,
                           a.dv_part, parts, a.D, a.N, dA, dDskip, ddt_bias);
        JANUS_LAUNCH_CHECK();
    }
    if (a.bc_part && a.T > 0) {
        const int64_t all = int64_t(a.T) * a.B * a.G * 2 * NP;
        TraceScope trace("scan_bc", double(all) * a.bblocks, 4.0 * all * a.bblocks, st);
        hipLaunchKernelGGL((scan_bc_kernel<T, NP>), launch_blocks((all + 255) / 256, 256), dim3(256), 0, st, a);
        JANUS_LAUNCH_CHECK();
    }
    return JANUS_OK;
}

template <template <typename, int> class F, typename T, class... P>
janus_status with_states(int N, P&&... p) {
    switch (padded_states(N)) {
        case 4: return F<T, 4>::run(p...);
        case 8: return F<T, 8>::run(p...);
        case 16: return F<T, 16>::run(p...);
        case 32: return F<T, 32>::run(p...);
        default: return F<T, 64>::run(p...);
    }
}
template <typename T, int NP> struct FwdRun {
    static janus_status run(const ScanArgs& a, const int32_t* lengths, hipStream_t st) {
        return scan_fwd_run<T, NP>(a, lengths, st);
    }
};
template <typename T, int NP> struct BwdRun {
    static janus_status run(const ScanArgs& a, const int32_t* lengths, float* dA, float* dD, float* dtb, hipStream_t st) {
        return scan_bwd_run<T, NP>(a, lengths, dA, dD, dtb, st);
    }
};
template <typename T, int NP> struct StepRun {
    static janus_status run(const ScanArgs& a, const int32_t* slots, int32_t n_slots, float* state, hipStream_t st) {
        constexpr int QL = NP / 4;
        const dim3 grid((int64_t(a.D) * QL + 255) / 256, a.B);
        if (a.N % 4 == 0 && aligned(state, 16) && aligned(a.A, 16))
            hipLaunchKernelGGL((scan_step_kernel<T, QL, true>), grid, dim3(256), 0, st, a, slots, n_slots, state);
        else
            hipLaunchKernelGGL((scan_step_kernel<T, QL, false>), grid, dim3(256), 0, st, a, slots, n_slots, state);
        JANUS_LAUNCH_CHECK();
        return JANUS_OK;
    }
};

}  // namespace
}  // namespace janus

using namespace janus;

extern "C" size_t janus_selective_scan_workspace_bytes(const janus_scan_desc* d) {
    if (!scan_desc_ok(d) || !scan_supported(d)) return 0;
    ScanArgs a = scan_geometry(d);
    return scan_carve(a, d->flags & JANUS_SCAN_KEEP, nullptr);
}

extern "C" janus_status janus_selective_scan_fwd(const janus_scan_desc* d, const void* x, const void* dt,
                                                 const float* A, const void* Bm, const void* Cm, const float* Dskip,
                                                 const void* z, const float* dt_bias, const int32_t* lengths,
                                                 const float* h0, void* y, float* hT, void* ws, size_t ws_bytes,
                                                 void* stream) {
    janus_status e = scan_check(d, x, dt, A, Bm, Cm, Dskip, z, dt_bias, y, d && d->T > 0);
    if (e != JANUS_OK) return e;
    const bool keep = d->flags & JANUS_SCAN_KEEP;
    if (!aligned(h0, 4) || !aligned(hT, 4) || (keep && hT && hT == h0)) return JANUS_ERR_INVALID_ARG;
    if ((e = check_lengths(d->B, d->T, lengths)) != JANUS_OK) return e;
    ScanArgs a = scan_geometry(d);
    const size_t need = scan_carve(a, keep, ws);
    if (need > 0 && (!ws || ws_bytes < need || !aligned(ws, 256))) return JANUS_ERR_WORKSPACE;
    scan_inputs(a, x, dt, A, Bm, Cm, Dskip, z, dt_bias);
    a.h0 = h0, a.y = y, a.hT = hT;
    hipStream_t st = static_cast<hipStream_t>(stream);
    return d->dtype == JANUS_BF16 ? with_states<FwdRun, bf16_t>(a.N, a, lengths, st)
                                  : with_states<FwdRun, float>(a.N, a, lengths, st);
}

extern "C" janus_status janus_selective_scan_bwd(const janus_scan_desc* d, const void* x, const void* dt,
                                                 const float* A, const void* Bm, const void* Cm, const float* Dskip,
                                                 const void* z, const float* dt_bias, const int32_t* lengths,
                                                 const float* h0, const void* dy, const float* dhT, void* dx,
                                                 void* ddt, float* dA, void* dBm, void* dCm, float* dDskip, void* dz,
                                                 float* ddt_bias, float* dh0, void* ws, size_t ws_bytes,
                                                 void* stream) {
    const bool rows = d && d->T > 0;
    janus_status e = scan_check(d, x, dt, A, Bm, Cm, Dskip, z, dt_bias, dy, rows);
    if (e != JANUS_OK) return e;
    if (!(d->flags & JANUS_SCAN_KEEP) || !dA || (rows && (!dx || !ddt || !dBm || !dCm || (z && !dz))))
        return JANUS_ERR_INVALID_ARG;
    const size_t es = dtype_size(d->dtype);
    for (const void* p : {static_cast<const void*>(dx), static_cast<const void*>(ddt), static_cast<const void*>(dBm),
                          static_cast<const void*>(dCm), static_cast<const void*>(dz)}) {
        if (!aligned(p, es)) return JANUS_ERR_INVALID_ARG;
        for (const void* q : {x, dt, Bm, Cm, z, dy})
            if (p && p == q) return JANUS_ERR_INVALID_ARG;
    }
    for (const float* p : {h0, dhT, static_cast<const float*>(dA), static_cast<const float*>(dDskip),
                           static_cast<const float*>(ddt_bias), static_cast<const float*>(dh0)})
        if (!aligned(p, 4)) return JANUS_ERR_INVALID_ARG;
    if ((e = check_lengths(d->B, d->T, lengths)) != JANUS_OK) return e;
    ScanArgs a = scan_geometry(d);
    const size_t need = scan_carve(a, true, ws);
    if (!ws || ws_bytes < need || !aligned(ws, 256)) return JANUS_ERR_WORKSPACE;
    scan_inputs(a, x, dt, A, Bm, Cm, Dskip, z, dt_bias);
    a.h0 = h0, a.dy = dy, a.dhT = dhT, a.dx = dx, a.ddt = ddt, a.dz = dz, a.dBm = dBm, a.dCm = dCm, a.dh0 = dh0;
    hipStream_t st = static_cast<hipStream_t>(stream);
    return d->dtype == JANUS_BF16 ? with_states<BwdRun, bf16_t>(a.N, a, lengths, dA, dDskip, ddt_bias, st)
                                  : with_states<BwdRun, float>(a.N, a, lengths, dA, dDskip, ddt_bias, st);
}

extern "C" janus_status janus_selective_scan_step(const janus_scan_desc* d, const void* x, const void* dt,
                                                  const float* A, const void* Bm, const void* Cm, const float* Dskip,
                                                  const void* z, const float* dt_bias, const int32_t* slots,
                                                  int32_t n_slots, float* state, void* y, void* stream) {
    janus_status e = scan_check(d, x, dt, A, Bm, Cm, Dskip, z, dt_bias, y, true);
    if (e != JANUS_OK) return e;
    if (!state || n_slots < 1 || (!slots && n_slots < d->B) || !aligned(slots, 4) || !aligned(state, 4))
        return JANUS_ERR_INVALID_ARG;
    if (d->B > 65535) return JANUS_ERR_UNSUPPORTED;
    ScanArgs a = scan_geometry(d);
    scan_inputs(a, x, dt, A, Bm, Cm, Dskip, z, dt_bias);
    a.y = y;
    const size_t four = 4 * dtype_size(d->dtype);
    a.bc4 = a.ldb % 4 == 0 && a.ldc % 4 == 0 && aligned(Bm, four) && aligned(Cm, four);
    hipStream_t st = static_cast<hipStream_t>(stream);
    TraceScope trace("scan_step", 7.0 * a.B * a.D * a.N, 8.0 * a.B * a.D * a.N, st);
    return d->dtype == JANUS_BF16 ? with_states<StepRun, bf16_t>(a.N, a, slots, n_slots, state, st)
                                  : with_states<StepRun, float>(a.N, a, slots, n_slots, state, st);
}
