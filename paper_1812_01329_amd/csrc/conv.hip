// Short causal convolution over variable-length sequences (depthwise, up to 8
// taps): forward, backward, and the single-token step.
//
//   p_t = b + sum_k w[k] x_{t-K+1+k},   y = p or p s(p)
//   g_t = dy_t f'(p_t),  dx_t = sum_j w[K-1-j] g_{t+j},
//   dw[k] = sum_t g_t x_{t-K+1+k},  db = sum_t g_t
//
// A lane owns VEC channels (16 bytes where the operands allow it) and walks
// over the time steps of its segment with the last K inputs in registers, so
// every row is read once but for K - 1 rows at a segment's edge.  K is a
// template parameter: a tap padded with a zero weight would turn an infinite
// input into NaN.
//
// Bound by memory.  25600 rows of 1024 bf16 channels, 4 taps, half of the rows
// past their sequences' ends: forward 18 us (78 MB: 4.3 TB/s), backward 38 us
// (105 MB: 2.8 TB/s; the rows at segments' edges are read twice, and two waves
// stand on a SIMD: 163 registers a lane would leave room for a third, but not
// for a second workgroup of eight waves on a CU).  All rows within the sequences:
// bf16 21 and 51 us, float32 34 and 69 us, float32 with 8 taps 37 and 195 us (7
// and 8 taps of four float32 channels spill 16 and 83 registers in the backward).
// One token of 20 rows of 1300: 3.4 us, a launch.
#include "seq.hpp"

namespace janus {
namespace {

constexpr int kMaxTaps = 8;
constexpr int kMaxChannels = 1 << 24, kMaxSteps = 1 << 30;   // (32-bit indexes)

struct ConvArgs {
    int32_t D, B, T, seg, nseg;    // seg time steps per segment
    int64_t ldx, ldy;
    const void* x;
    const void* w;
    const void* bias;
    const void* s0;
    void* y;            // forward, step
    void* sT;           // forward
    const void* dy;     // backward
    const float* dsT;
    void* dx;
    float* ds0;
    float* part;        // [parts, K + 1, D] sums of dw and dbias, or NULL
    bool silu, w16;     // w16: w is 16-byte aligned
};

// The taps and biases of a lane's channels; in 16-byte loads where the lanes'
// parts of w [D, K] are whole ones of those (each tap alone is K loads a channel).
template <typename T, int K, int VEC>
__device__ __forceinline__ void load_taps(const ConvArgs& a, int d, float (&w)[K][VEC], float (&bias)[VEC]) {
    constexpr int N = K * VEC, PER = 16 / sizeof(T);
    const T* wp = static_cast<const T*>(a.w) + int64_t(d) * K;
    const T* bp = static_cast<const T*>(a.bias);
    T raw[N];
    if (N % PER == 0 && a.w16) {
#pragma unroll
        for (int i = 0; i < N / PER; ++i) {
            const uint4 v = reinterpret_cast<const uint4*>(wp)[i];
            __builtin_memcpy(raw + i * PER, &v, 16);
        }
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) raw[i] = wp[i];
    }
#pragma unroll
    for (int v = 0; v < VEC; ++v) {
        bias[v] = bp ? to_f(bp[d + v]) : 0.f;
#pragma unroll
        for (int k = 0; k < K; ++k) w[k][v] = to_f(raw[v * K + k]);
    }
}

// input of time t (negative: the carried state), 0 where there is none
template <typename T, int K, int VEC>
__device__ __forceinline__ void load_input(const ConvArgs& a, int b, int t, int d, float (&f)[VEC]) {
    if (t >= 0) {
        Chan<T, VEC> r;
        r.load(static_cast<const T*>(a.x) + (int64_t(t) * a.B + b) * a.ldx + d);
        r.get(f);
    } else if (a.s0) {
        Chan<T, VEC> r;
        r.load(static_cast<const T*>(a.s0) + (int64_t(b) * (K - 1) + (K - 1 + t)) * a.D + d);
        r.get(f);
    } else {
#pragma unroll
        for (int v = 0; v < VEC; ++v) f[v] = 0.f;
    }
}

template <typename T, int K, int VEC>
__global__ __launch_bounds__(256) void conv_fwd_kernel(ConvArgs a, SeqSlice s) {
    const int d = (blockIdx.x * blockDim.x + threadIdx.x) * VEC;
    if (d >= a.D) return;
    const int len = s.len[blockIdx.y], b = seq_of(s, blockIdx.y);
    const int t0 = blockIdx.z * a.seg, t1 = min(a.T, t0 + a.seg), te = min(t1, len);
    float w[K][VEC], bias[VEC], win[K][VEC];   // win[k]: input of time t - K + 1 + k
    load_taps<T, K, VEC>(a, d, w, bias);
    T* yp = static_cast<T*>(a.y) + b * a.ldy + d;
    const T* xp = static_cast<const T*>(a.x) + b * a.ldx + d;
    const int64_t sx = a.B * a.ldx, sy = a.B * a.ldy;
    if (t0 < te) {
#pragma unroll
        for (int k = 0; k < K - 1; ++k) load_input<T, K, VEC>(a, b, t0 - K + 1 + k, d, win[k]);
    }
    constexpr int U = 8;
    int t = t0;
    for (; t < te; t += U) {
        Chan<T, VEC> r[U];
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (t + u < te) r[u].load(xp + (t + u) * sx);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (t + u < te) {
                r[u].get(win[K - 1]);
                float y[VEC];
#pragma unroll
                for (int v = 0; v < VEC; ++v) {
                    float p = bias[v];
#pragma unroll
                    for (int k = 0; k < K; ++k) p = fmaf(w[k][v], win[k][v], p);
                    y[v] = a.silu ? p * sigmoidf_(p) : p;
                }
                Chan<T, VEC>::store(yp + (t + u) * sy, y);
#pragma unroll
                for (int k = 0; k + 1 < K; ++k)
#pragma unroll
                    for (int v = 0; v < VEC; ++v) win[k][v] = win[k + 1][v];
            }
        }
    }
    float zero[VEC] = {};
    for (t = max(t0, len); t < t1; ++t) Chan<T, VEC>::store(yp + t * sy, zero);
    if (a.sT && blockIdx.z == 0) {
        T* sp = static_cast<T*>(a.sT) + int64_t(b) * (K - 1) * a.D + d;
        for (int i = 0; i < K - 1; ++i) {
            float f[VEC];
            load_input<T, K, VEC>(a, b, len - (K - 1) + i, d, f);
            Chan<T, VEC>::store(sp + int64_t(i) * a.D, f);
        }
    }
}

// What a lane keeps between the time steps of an item
template <int K, int VEC>
struct ConvWin {
    float x[K][VEC], g[K][VEC];   // [j]: of time u - K + 1 + j
    __device__ __forceinline__ void shift() {
#pragma unroll
        for (int k = 0; k + 1 < K; ++k)
#pragma unroll
            for (int v = 0; v < VEC; ++v) x[k][v] = x[k + 1][v], g[k][v] = g[k + 1][v];
    }
};

// A lane walks over items (sequence, segment) of the slice and keeps the sums of
// dw and dbias in registers.  At time u it has g_u and so dx_{u-K+1}; an item
// reads K - 1 rows past its end for the last ones, and the first item of a
// sequence starts K - 1 steps early in dx: the gradient of the carried state.
// A workgroup is `groups` rows of lanes, each with its own items; their sums
// are added in LDS, which leaves a part a workgroup to write.
template <typename T, int K, int VEC>
__global__ __launch_bounds__(512) void conv_bwd_kernel(ConvArgs a, SeqSlice s, int items, int part0, int lanes,
                                                       int groups) {
    extern __shared__ float red[];   // [groups - 1][lanes * VEC]
    const int lane = threadIdx.x % lanes, group = threadIdx.x / lanes;
    const int d = (blockIdx.x * lanes + lane) * VEC;
    const bool on = d < a.D && group < groups;
    float w[K][VEC], bias[VEC], dw[K + 1][VEC];   // dw[K]: dbias
#pragma unroll
    for (int v = 0; v < VEC; ++v)
#pragma unroll
        for (int k = 0; k <= K; ++k) dw[k][v] = 0.f;
    if (on) load_taps<T, K, VEC>(a, d, w, bias);
    const int64_t sx = a.B * a.ldx, sy = a.B * a.ldy;
    for (int item = blockIdx.y * groups + group; on && item < items; item += gridDim.y * groups) {
        const int bs = item / a.nseg, seg = item - bs * a.nseg;
        const int len = s.len[bs], b = s.b0 + s.at[bs];
        const int t0 = seg * a.seg, t1 = min(a.T, t0 + a.seg);
        const T* xp = static_cast<const T*>(a.x) + b * a.ldx + d;
        const T* gp = static_cast<const T*>(a.dy) + b * a.ldy + d;
        T* dxp = a.dx ? static_cast<T*>(a.dx) + b * a.ldx + d : nullptr;
        ConvWin<K, VEC> win;
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int v = 0; v < VEC; ++v) win.x[k][v] = win.g[k][v] = 0.f;
        if (t0 < len) {
#pragma unroll
            for (int k = 0; k < K - 1; ++k) load_input<T, K, VEC>(a, b, t0 - K + 1 + k, d, win.x[k]);
        }
        // g_u from row u, and its part of the sums (the rows past the segment are the next item's)
        auto take = [&](const Chan<T, VEC>& rx, const Chan<T, VEC>& rg, bool sum) {
            rx.get(win.x[K - 1]);
            rg.get(win.g[K - 1]);
            if (a.silu) {
#pragma unroll
                for (int v = 0; v < VEC; ++v) {
                    float p = bias[v];
#pragma unroll
                    for (int k = 0; k < K; ++k) p = fmaf(w[k][v], win.x[k][v], p);
                    const float q = sigmoidf_(p);
                    win.g[K - 1][v] *= q * (1.f + p * (1.f - q));
                }
            }
            if (sum) {
#pragma unroll
                for (int v = 0; v < VEC; ++v) {
                    dw[K][v] += win.g[K - 1][v];
#pragma unroll
                    for (int k = 0; k < K; ++k) dw[k][v] = fmaf(win.g[K - 1][v], win.x[k][v], dw[k][v]);
                }
            }
        };
        auto input_grad = [&](float (&dx)[VEC]) {
#pragma unroll
            for (int v = 0; v < VEC; ++v) {
                dx[v] = 0.f;
#pragma unroll
                for (int j = 0; j < K; ++j) dx[v] = fmaf(w[K - 1 - j][v], win.g[j][v], dx[v]);
            }
        };
        // one step at the edges of a segment or a sequence
        auto edge = [&](const Chan<T, VEC>& rx, const Chan<T, VEC>& rg, int u) {
            if (u < len) {
                take(rx, rg, u < t1);
            } else {
#pragma unroll
                for (int v = 0; v < VEC; ++v) win.g[K - 1][v] = 0.f;
            }
            const int t = u - (K - 1);
            if (t >= t0 || seg == 0) {
                float dx[VEC] = {};
                if (t < len) {
                    input_grad(dx);
                    const int i = t - (len - (K - 1));   // row of the final state
                    if (a.dsT && i >= 0) {
#pragma unroll
                        for (int v = 0; v < VEC; ++v) dx[v] += a.dsT[(int64_t(b) * (K - 1) + i) * a.D + d + v];
                    }
                }
                if (t >= 0) {
                    if (dxp) Chan<T, VEC>::store(dxp + t * sx, dx);
                } else if (a.ds0) {
#pragma unroll
                    for (int v = 0; v < VEC; ++v)
                        a.ds0[(int64_t(b) * (K - 1) + (K - 1 + t)) * a.D + d + v] = dx[v];
                }
            }
            win.shift();
        };
        constexpr int U = 4;
        const int ue = t1 + K - 1, ul = min(ue, len);
        Chan<T, VEC> rx[U], rg[U], nx[U], ng[U];   // rows [u, u + U) and the U after them, on their way
#pragma unroll
        for (int i = 0; i < U; ++i)
            if (t0 + i < ul) nx[i].load(xp + (t0 + i) * sx), ng[i].load(gp + (t0 + i) * sy);
        for (int u = t0; u < ue; u += U) {
#pragma unroll
            for (int i = 0; i < U; ++i) rx[i] = nx[i], rg[i] = ng[i];
#pragma unroll
            for (int i = 0; i < U; ++i)
                if (u + U + i < ul) nx[i].load(xp + (u + U + i) * sx), ng[i].load(gp + (u + U + i) * sy);
            if (u >= t0 + K - 1 && u + U <= min(t1, len)) {   // their dx is this item's and no part of the final state
#pragma unroll
                for (int i = 0; i < U; ++i) {
                    take(rx[i], rg[i], true);
                    float dx[VEC];
                    input_grad(dx);
                    if (dxp) Chan<T, VEC>::store(dxp + (u + i - (K - 1)) * sx, dx);
                    win.shift();
                }
            } else {
#pragma unroll
                for (int i = 0; i < U; ++i)
                    if (u + i < ue) edge(rx[i], rg[i], u + i);
            }
        }
    }
    if (!a.part) return;
    float* p = a.part + int64_t(part0 + blockIdx.y) * (K + 1) * a.D;
#pragma unroll
    for (int k = 0; k <= K; ++k) {
        if (group > 0 && group < groups) {
#pragma unroll
            for (int v = 0; v < VEC; ++v) red[(group - 1) * lanes * VEC + v * lanes + lane] = dw[k][v];
        }
        __syncthreads();
        if (group == 0 && on) {
#pragma unroll
            for (int v = 0; v < VEC; ++v) {
                float f = dw[k][v];
                for (int g = 0; g < groups - 1; ++g) f += red[g * lanes * VEC + v * lanes + lane];
                p[int64_t(k) * a.D + d + v] = f;
            }
        }
        __syncthreads();
    }
}

// dw [D, K] and dbias [D] from the parts: 64 values a workgroup, each wave sums
// every 16th part, then the waves' sums in their order.
__global__ __launch_bounds__(1024) void conv_param_kernel(const float* part, int parts, int D, int K, float* dw,
                                                          float* dbias) {
    __shared__ float red[16][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n = (K + 1) * D;
    const int i = blockIdx.x * 64 + lane;   // k * D + d
    float s = 0.f;
    if (i < n)
        for (int p = wave; p < parts; p += 16) s += part[int64_t(p) * n + i];
    red[wave][lane] = s;
    __syncthreads();
    if (wave != 0 || i >= n) return;
    for (int w = 1; w < 16; ++w) s += red[w][lane];
    const int k = i / D, d = i - k * D;
    if (k < K) {
        if (dw) dw[int64_t(d) * K + k] = s;
    } else if (dbias) {
        dbias[d] = s;
    }
}

template <typename T, int K, int VEC>
__global__ __launch_bounds__(64) void conv_step_kernel(ConvArgs a, const int32_t* slots, int32_t n_slots) {
    const int d = (blockIdx.x * blockDim.x + threadIdx.x) * VEC, b = blockIdx.y;
    if (d >= a.D) return;
    const int slot = slots ? slots[b] : b;
    T* yp = static_cast<T*>(a.y) + b * a.ldy + d;
    if (slot < 0 || slot >= n_slots) {
        float zero[VEC] = {};
        Chan<T, VEC>::store(yp, zero);
        return;
    }
    float w[K][VEC], bias[VEC];
    Chan<T, VEC> in[K];   // as stored: the state moves on bit for bit
    T* sp = static_cast<T*>(a.sT) + int64_t(slot) * (K - 1) * a.D + d;
#pragma unroll
    for (int k = 0; k < K - 1; ++k) in[k].load(sp + int64_t(k) * a.D);
    in[K - 1].load(static_cast<const T*>(a.x) + b * a.ldx + d);
    load_taps<T, K, VEC>(a, d, w, bias);
    float p[VEC];
#pragma unroll
    for (int v = 0; v < VEC; ++v) p[v] = bias[v];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        float f[VEC];
        in[k].get(f);
#pragma unroll
        for (int v = 0; v < VEC; ++v) p[v] = fmaf(w[k][v], f[v], p[v]);
    }
    if (a.silu) {
#pragma unroll
        for (int v = 0; v < VEC; ++v) p[v] *= sigmoidf_(p[v]);
    }
    Chan<T, VEC>::store(yp, p);
#pragma unroll
    for (int k = 0; k + 1 < K; ++k) *reinterpret_cast<decltype(in[0].v)*>(sp + int64_t(k) * a.D) = in[k + 1].v;
}

// -------------------------------------------------------------------- host
bool conv_desc_ok(const janus_conv_desc* d) {
    return d && d->D > 0 && d->K > 0 && d->B > 0 && d->T >= 0 && (d->ldx == 0 || d->ldx >= d->D) &&
           (d->ldy == 0 || d->ldy >= d->D);
}
janus_status conv_check(const janus_conv_desc* d, const void* x, const void* w, const void* bias, const void* s0,
                        const void* y, const void* sT, bool rows) {
    if (!conv_desc_ok(d) || !w || (rows && (!x || !y))) return JANUS_ERR_INVALID_ARG;
    if (!dtype_ok(d->dtype) || d->K > kMaxTaps || d->D > kMaxChannels || d->T > kMaxSteps || (d->act != JANUS_CONV_LINEAR && d->act != JANUS_CONV_SILU))
        return JANUS_ERR_UNSUPPORTED;
    const size_t es = dtype_size(d->dtype);
    for (const void* p : {x, w, bias, s0, y, sT})
        if (!aligned(p, es)) return JANUS_ERR_INVALID_ARG;
    return JANUS_OK;
}

ConvArgs conv_args(const janus_conv_desc* d, const void* x, const void* w, const void* bias, const void* s0) {
    ConvArgs a{};
    a.D = d->D, a.B = d->B, a.T = d->T;
    a.ldx = d->ldx ? d->ldx : d->D;
    a.ldy = d->ldy ? d->ldy : d->D;
    a.x = x, a.w = w, a.bias = bias, a.s0 = s0;
    a.silu = d->act == JANUS_CONV_SILU;
    a.w16 = aligned(w, 16);
    return a;
}

// Channels per lane: 4, or 2 for bf16, or 1: as many as every row of every
// operand is aligned to and as leave a wave's lanes filled.  (8 bf16 channels
// a lane take so many registers that fewer waves hide the loads' latency:
// 25600 rows of 1024 channels, half of them past their ends, forward 28.8 us
// with 8, 21.8 with 4, 23.2 with 2.)
int conv_vec(const janus_conv_desc* d, const ConvArgs& a, std::initializer_list<const void*> ptrs) {
    const size_t es = dtype_size(d->dtype);
    for (int v : {4, 2}) {
        if (v == 2 && es == 4) continue;
        const size_t bytes = v * es;
        bool ok = a.D % v == 0 && a.D / v >= 64 && a.ldx % v == 0 && a.ldy % v == 0;
        for (const void* p : ptrs) ok = ok && aligned(p, bytes);
        if (ok) return v;
    }
    return 1;
}

template <typename T, int VEC, class F>
void with_taps(int K, F f) {
    switch (K) {
        case 1: f.template go<T, 1, VEC>(); break;
        case 2: f.template go<T, 2, VEC>(); break;
        case 3: f.template go<T, 3, VEC>(); break;
        case 4: f.template go<T, 4, VEC>(); break;
        case 5: f.template go<T, 5, VEC>(); break;
        case 6: f.template go<T, 6, VEC>(); break;
        case 7: f.template go<T, 7, VEC>(); break;
        default: f.template go<T, 8, VEC>(); break;
    }
}
template <class F>
void conv_dispatch(janus_dtype dt, int K, int vec, F f) {
    if (dt == JANUS_F32) {
        if (vec == 4) with_taps<float, 4>(K, f);
        else with_taps<float, 1>(K, f);
    } else {
        if (vec == 4) with_taps<bf16_t, 4>(K, f);
        else if (vec == 2) with_taps<bf16_t, 2>(K, f);
        else with_taps<bf16_t, 1>(K, f);
    }
}

struct FwdLaunch {
    const ConvArgs& a;
    const SeqSlice& s;
    dim3 grid, block;
    hipStream_t st;
    template <typename T, int K, int VEC> void go() {
        hipLaunchKernelGGL((conv_fwd_kernel<T, K, VEC>), grid, block, 0, st, a, s);
    }
};
struct BwdLaunch {
    const ConvArgs& a;
    const SeqSlice& s;
    int items, part0, lanes, groups;
    dim3 grid;
    hipStream_t st;
    template <typename T, int K, int VEC> void go() {
        hipLaunchKernelGGL((conv_bwd_kernel<T, K, VEC>), grid, dim3(lanes * groups),
                           size_t(groups - 1) * lanes * VEC * sizeof(float), st, a, s, items, part0, lanes, groups);
    }
};
struct StepLaunch {
    const ConvArgs& a;
    const int32_t* slots;
    int32_t n_slots;
    dim3 grid, block;
    hipStream_t st;
    template <typename T, int K, int VEC> void go() {
        hipLaunchKernelGGL((conv_step_kernel<T, K, VEC>), grid, block, 0, st, a, slots, n_slots);
    }
};

// Threads of a block of the channels, blocks along them, and how the time axis
// is cut: segments of at least 16 steps, as many as it takes for 4096 waves.
struct ConvShape {
    int threads, blocks;
};
ConvShape conv_shape(ConvArgs& a, int vec) {
    const int lanes = (a.D + vec - 1) / vec;
    ConvShape c;
    c.threads = std::min(256, int(round_up(lanes, 64)));
    c.blocks = (lanes + c.threads - 1) / c.threads;
    const int64_t waves = int64_t(a.B) * ((lanes + 63) / 64);
    const int64_t want = std::max<int64_t>(1, std::min<int64_t>(a.T / 16, 4096 / waves));
    a.seg = std::max(1, int((a.T + want - 1) / want));
    a.nseg = std::max(1, (a.T + a.seg - 1) / a.seg);
    return c;
}

// Parts of the sums of dw and dbias in one slice, at most: workgroups of 8 waves
// along the items, for two waves a SIMD of 4 channels a lane and D up to 4096.
int conv_parts(int32_t D) { return std::max(16, 256 / ((D + 4095) / 4096)); }
int conv_slices(int32_t B) { return (B + kSlice - 1) / kSlice; }
size_t conv_ws_bytes(const janus_conv_desc* d) {
    Carver c(nullptr);
    c.take<float>(size_t(conv_slices(d->B)) * conv_parts(d->D) * (d->K + 1) * d->D);
    return c.off;
}

}  // namespace
}  // namespace janus

using namespace janus;

extern "C" size_t janus_causal_conv_workspace_bytes(const janus_conv_desc* d) {
    if (!conv_desc_ok(d) || d->K > kMaxTaps || d->D > kMaxChannels || !dtype_ok(d->dtype)) return 0;
    return conv_ws_bytes(d);
}

extern "C" janus_status janus_causal_conv_fwd(const janus_conv_desc* d, const void* x, const int32_t* lengths,
                                              const void* w, const void* bias, const void* s0, void* y, void* sT,
                                              void* stream) {
    janus_status e = conv_check(d, x, w, bias, s0, y, sT, d && d->T > 0);
    if (e != JANUS_OK) return e;
    if ((y && y == x) || (sT && sT == s0)) return JANUS_ERR_INVALID_ARG;
    if ((e = check_lengths(d->B, d->T, lengths)) != JANUS_OK) return e;
    hipStream_t st = static_cast<hipStream_t>(stream);
    ConvArgs a = conv_args(d, x, w, bias, s0);
    a.y = y, a.sT = d->K > 1 ? sT : nullptr;
    if (d->T == 0 && !a.sT) return JANUS_OK;
    const int vec = conv_vec(d, a, {x, y, s0, sT});
    const ConvShape c = conv_shape(a, vec);
    const double el = double(d->T) * d->B * d->D;
    for (int32_t b0 = 0; b0 < d->B; b0 += kSlice) {
        SeqSlice s;
        const int n = fill_slice(s, b0, d->B, d->T, lengths);
        TraceScope trace("conv_fwd", el / d->B * n * 2 * d->K, el / d->B * n * 2 * dtype_size(d->dtype), st);
        conv_dispatch(d->dtype, d->K, vec, FwdLaunch{a, s, dim3(c.blocks, n, a.nseg), dim3(c.threads), st});
        JANUS_LAUNCH_CHECK();
    }
    return JANUS_OK;
}

extern "C" janus_status janus_causal_conv_bwd(const janus_conv_desc* d, const void* x, const int32_t* lengths,
                                              const void* w, const void* bias, const void* s0, const void* dy,
                                              const float* dsT, void* dx, float* dw, float* dbias, float* ds0,
                                              void* ws, size_t ws_bytes, void* stream) {
    janus_status e = conv_check(d, x, w, bias, s0, dy, dx, d && d->T > 0);
    if (e != JANUS_OK) return e;
    if ((dx && (dx == x || dx == dy)) || (ds0 && ds0 == dsT)) return JANUS_ERR_INVALID_ARG;
    for (const float* p : {dsT, static_cast<const float*>(dw), static_cast<const float*>(dbias),
                           static_cast<const float*>(ds0)})
        if (!aligned(p, 4)) return JANUS_ERR_INVALID_ARG;
    if ((e = check_lengths(d->B, d->T, lengths)) != JANUS_OK) return e;
    if (!ws || ws_bytes < conv_ws_bytes(d) || !aligned(ws, 256)) return JANUS_ERR_WORKSPACE;
    hipStream_t st = static_cast<hipStream_t>(stream);
    ConvArgs a = conv_args(d, x, w, bias, s0);
    a.dy = dy, a.dsT = dsT, a.dx = dx, a.ds0 = ds0;
    a.part = dw || dbias ? static_cast<float*>(ws) : nullptr;
    const int vec = conv_vec(d, a, {x, dy, dx, s0});
    const ConvShape c = conv_shape(a, vec);
    const double el = double(d->T) * d->B * d->D;
    int parts = 0;
    for (int32_t b0 = 0; b0 < d->B; b0 += kSlice) {
        SeqSlice s;
        const int n = fill_slice(s, b0, d->B, d->T, lengths);
        const int items = n * a.nseg, groups = std::min(512 / c.threads, items);
        const int rows = std::min((items + groups - 1) / groups, conv_parts(d->D));
        TraceScope trace("conv_bwd", el / d->B * n * 6 * d->K, el / d->B * n * 3 * dtype_size(d->dtype), st);
        conv_dispatch(d->dtype, d->K, vec, BwdLaunch{a, s, items, parts, c.threads, groups, dim3(c.blocks, rows), st});
        JANUS_LAUNCH_CHECK();
        parts += rows;
    }
    if (a.part) {
        const int n = (d->K + 1) * d->D;
        TraceScope trace("conv_param", double(n) * parts, 4.0 * n * parts, st);
        hipLaunchKernelGGL(conv_param_kernel, dim3((n + 63) / 64), dim3(1024), 0, st, a.part, parts, d->D, d->K, dw,
                           dbias);
        JANUS_LAUNCH_CHECK();
    }
    return JANUS_OK;
}

extern "C" janus_status janus_causal_conv_step(const janus_conv_desc* d, const void* x, const void* w,
                                               const void* bias, const int32_t* slots, int32_t n_slots, void* state,
                                               void* y, void* stream) {
    janus_status e = conv_check(d, x, w, bias, state, y, nullptr, true);
    if (e != JANUS_OK) return e;
    if ((d->K > 1 && !state) || n_slots < 1 || (!slots && n_slots < d->B) || !aligned(slots, 4) || y == x)
        return JANUS_ERR_INVALID_ARG;
    if (d->B > 65535) return JANUS_ERR_UNSUPPORTED;
    hipStream_t st = static_cast<hipStream_t>(stream);
    ConvArgs a = conv_args(d, x, w, bias, nullptr);
    a.y = y, a.sT = state;
    const int vec = conv_vec(d, a, {x, y, state});
    const int lanes = (d->D + vec - 1) / vec;
    TraceScope trace("conv_step", 2.0 * d->B * d->D * d->K, 2.0 * d->B * d->D * d->K * dtype_size(d->dtype), st);
    conv_dispatch(d->dtype, d->K, vec, StepLaunch{a, slots, n_slots, dim3((lanes + 63) / 64, d->B), dim3(64), st});
    JANUS_LAUNCH_CHECK();
    return JANUS_OK;
}
