// The router's balance loss with per-expert counts and gradients (gfx950).
//
// stat_kernel sums the probabilities (fp64) and counts the selections of every
// expert, a share of the tokens per workgroup; the last workgroup to finish
// adds the shares in order and forms the loss and q = dloss / dP.  dz_kernel
// makes the scores' gradient dz = p (q - <q, p>) / n row by row, dx_kernel
// its product with the router weights, dw_kernel with x (fp32 matrix
// instructions), over slices of the tokens that dw_join_kernel adds in order.
#include <math.h>

#include <algorithm>

#include "eat_device.h"
#include "eat_internal.h"

namespace eat {
namespace {

constexpr int kStatWaves = 16;
constexpr int kStatThreads = kStatWaves * kWave;
constexpr int kStatBlocks = 64;           // most shares of the tokens

struct StatArgs {
    const float* prob;
    const uint64_t* mask;
    const uint8_t* valid;
    int T, E;
    float coef, entropy_coef;
    int32_t* head;             // {workgroups done}
    float* q;                  // [E] dloss / dP_e / max(n, 1)
    double* sum;               // [blocks][E]
    int32_t* cnt;              // [blocks][E + 1]: selections, then valid tokens
    float* loss;
    int64_t* count;
    float* mean_prob;
};

// Lane l holds experts l % EP + 64 j of token l / EP of a group of 64 / EP
// tokens (EP: E rounded up to a power of two, 64 at most).
template <int J>
__global__ __launch_bounds__(kStatThreads) void stat_kernel(StatArgs a) {
    __shared__ double red[kStatWaves][kWave];
    __shared__ int redc[kStatWaves][kWave];
    __shared__ double fin[4][kMaxExperts];
    __shared__ int finc[4][kMaxExperts];
    __shared__ int redn[kStatWaves];
    __shared__ int last;
    const int lane = lane_id(), wave = threadIdx.x / kWave;
    const int E = a.E;
    int ep = 1;
    while (ep < min(E, 64)) ep *= 2;
    const int sub = lane / ep, e0 = lane % ep, tpw = kWave / ep;
    const int per = (a.T + gridDim.x - 1) / gridDim.x;
    const int tbeg = min(a.T, static_cast<int>(blockIdx.x) * per), tend = min(a.T, tbeg + per);
    double s[J];
    int c[J], n = 0;
#pragma unroll
    for (int j = 0; j < J; ++j) { s[j] = 0.0; c[j] = 0; }
    for (int t0 = tbeg + wave * tpw; t0 < tend; t0 += kStatWaves * tpw) {
        const int t = t0 + sub;
        if (t < tend && (!a.valid || a.valid[t])) {
            n += e0 == 0;
#pragma unroll
            for (int j = 0; j < J; ++j)
                if (64 * j + e0 < E) {
                    s[j] += static_cast<double>(a.prob[static_cast<size_t>(t) * E + 64 * j + e0]);
                    c[j] += static_cast<int>((a.mask[static_cast<size_t>(t) * J + j] >> e0) & 1);
                }
        }
    }
    n = wave_sum(n);
    if (lane == 0) redn[wave] = n;
#pragma unroll
    for (int j = 0; j < J; ++j) {
        red[wave][lane] = s[j];
        redc[wave][lane] = c[j];
        __syncthreads();
        const int e = 64 * j + threadIdx.x;
        if (static_cast<int>(threadIdx.x) < ep && e < E) {
            double t = 0.0;
            int k = 0;
            for (int w = 0; w < kStatWaves; ++w)
                for (int u = 0; u < tpw; ++u) {
                    t += red[w][u * ep + threadIdx.x];
                    k += redc[w][u * ep + threadIdx.x];
                }
            a.sum[static_cast<size_t>(blockIdx.x) * E + e] = t;
            a.cnt[static_cast<size_t>(blockIdx.x) * (E + 1) + e] = k;
        }
        __syncthreads();
    }
    if (threadIdx.x == 0) {
        int k = 0;
        for (int w = 0; w < kStatWaves; ++w) k += redn[w];
        a.cnt[static_cast<size_t>(blockIdx.x) * (E + 1) + E] = k;
    }
    __threadfence();
    __syncthreads();
    if (threadIdx.x == 0)
        last = __hip_atomic_fetch_add(a.head, 1, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) ==
               static_cast<int>(gridDim.x) - 1;
    __syncthreads();
    if (!last) return;
    __threadfence();
    // the shares in order: quarter g of them per thread and expert, then the quarters
    const int blocks = gridDim.x;
    const int g = threadIdx.x >> 8, e = threadIdx.x & 255;
    double t = 0.0;
    int k = 0, nn = 0;
    if (e < E)
        for (int b = blocks * g / 4; b < blocks * (g + 1) / 4; ++b) {
            t += __hip_atomic_load(a.sum + static_cast<size_t>(b) * E + e, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            k += __hip_atomic_load(a.cnt + static_cast<size_t>(b) * (E + 1) + e, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
    fin[g][e] = t;
    finc[g][e] = k;
    if (wave == 0) {
        for (int b = lane; b < blocks; b += kWave)
            nn += __hip_atomic_load(a.cnt + static_cast<size_t>(b) * (E + 1) + E, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        nn = wave_sum(nn);
        if (lane == 0) redn[0] = nn;
    }
    __syncthreads();
    // one thread per expert from here on (waves 0 to 3)
    const double inv = 1.0 / max(redn[0], 1);
    double p = 0.0;
    if (wave < 4) {
        k = finc[0][e] + finc[1][e] + finc[2][e] + finc[3][e];
        p = (fin[0][e] + fin[1][e] + fin[2][e] + fin[3][e]) * inv;
        // (a call's selections are below 2^31: max_tokens times the most experts of a token is)
        const int sel = wave_sum(e < E ? k : 0);
        if (lane == 0) redc[0][wave] = sel;
    }
    __syncthreads();
    if (wave < 4) {
        const int total = redc[0][0] + redc[0][1] + redc[0][2] + redc[0][3];
        const double f = static_cast<double>(k) / max(total, 1);
        const double lg = p > 0.0 ? log(p) : p == 0.0 ? 0.0 : p;      // (NaN stays)
        const double l = wave_sum(e < E ? a.coef * E * f * p + a.entropy_coef * p * lg : 0.0);
        if (lane == 0) red[0][wave] = l;
        if (e < E) {
            a.q[e] = static_cast<float>((a.coef * E * f + a.entropy_coef * (lg + 1.0)) * inv);
            if (a.count) a.count[e] = k;
            if (a.mean_prob) a.mean_prob[e] = static_cast<float>(p);
        }
    }
    __syncthreads();
    if (threadIdx.x == 0) *a.loss = static_cast<float>((red[0][0] + red[0][1]) + (red[0][2] + red[0][3]));
}

__global__ void clear_kernel(int32_t* head) { *head = 0; }

constexpr int kDzWaves = 4;
template <int J>
__global__ __launch_bounds__(kDzWaves * kWave) void dz_kernel(const float* prob, const uint8_t* __restrict__ valid,
                                                              int T, int E, const float* __restrict__ q, float* dz) {
    const int lane = lane_id();
    int ep = 1;
    while (ep < min(E, 64)) ep *= 2;
    const int sub = lane / ep, e0 = lane % ep, tpw = kWave / ep;
    const int t = (blockIdx.x * kDzWaves + threadIdx.x / kWave) * tpw + sub;
    const bool live = t < T && (!valid || valid[t < T ? t : 0]);
    float p[J], qe[J];
    double s = 0.0;
#pragma unroll
    for (int j = 0; j < J; ++j) {
        const int e = 64 * j + e0;
        p[j] = live && e < E ? prob[static_cast<size_t>(t) * E + e] : 0.f;
        qe[j] = e < E ? q[e] : 0.f;
        s += static_cast<double>(qe[j]) * p[j];
    }
    for (int o = ep / 2; o >= 1; o /= 2) s += __shfl_xor(s, o, kWave);
#pragma unroll
    for (int j = 0; j < J; ++j) {
        const int e = 64 * j + e0;
        if (t < T && e < E)
            dz[static_cast<size_t>(t) * E + e] = live ? p[j] * static_cast<float>(qe[j] - s) : 0.f;
    }
}

__device__ __forceinline__ float load_f32(const float* p) { return *p; }
__device__ __forceinline__ float load_f32(const uint16_t* p) { return bf16_to_f32(*p); }
__device__ __forceinline__ void store_f32(float* p, float v) { *p = v; }
__device__ __forceinline__ void store_f32(uint16_t* p, float v) { *p = f32_to_bf16(v); }

// 64 tokens x 64 columns per workgroup, 16 tokens per wave.
template <typename XT>
__global__ __launch_bounds__(256) void dx_kernel(const float* __restrict__ dz, const float* __restrict__ w, int T, int E,
                                                 int d, float scale, XT* dx) {
    const int lane = lane_id(), wave = threadIdx.x / kWave;
    const int t0 = blockIdx.x * 64 + 16 * wave, c0 = blockIdx.y * 64;
    const int l16 = lane & 15, lk = lane >> 4;
    f32x4 acc[4] = {};
    const int t = min(t0 + l16, T - 1);
    for (int e = 0; e < E; e += 4) {
        const int k = min(e + lk, E - 1);
        const float z = dz[static_cast<size_t>(t) * E + k];
        const float a = e + lk < E ? z : 0.f;
#pragma unroll
        for (int f = 0; f < 4; ++f) {
            const float wv = w[static_cast<size_t>(k) * d + c0 + 16 * f + l16];
            acc[f] = __builtin_amdgcn_mfma_f32_16x16x4f32(a, e + lk < E ? wv : 0.f, acc[f], 0, 0, 0);
        }
    }
#pragma unroll
    for (int f = 0; f < 4; ++f)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int row = t0 + 4 * lk + i;
            if (row < T) store_f32(dx + static_cast<size_t>(row) * d + c0 + 16 * f + l16, acc[f][i] * scale);
        }
}

// 64 experts x 64 columns per workgroup, 16 experts per wave, over slice
// blockIdx.z of the tokens; tokens that are not valid read as zeros.
template <typename XT>
__global__ __launch_bounds__(256) void dw_kernel(const float* __restrict__ dz, const XT* __restrict__ x,
                                                 const uint8_t* __restrict__ valid, int T, int E, int d, float* out) {
    const int lane = lane_id(), wave = threadIdx.x / kWave;
    const int e0 = blockIdx.x * 64 + 16 * wave, c0 = blockIdx.y * 64;
    const int l16 = lane & 15, lk = lane >> 4;
    const int per = ((T + static_cast<int>(gridDim.z) - 1) / static_cast<int>(gridDim.z) + 3) / 4 * 4;
    const int tbeg = min(T, static_cast<int>(blockIdx.z) * per), tend = min(T, tbeg + per);
    f32x4 acc[4] = {};
    const int e = min(e0 + l16, E - 1);
    for (int t0 = tbeg; t0 < tend; t0 += 4) {
        const int t = min(t0 + lk, tend - 1);
        const bool live = t0 + lk < tend && (!valid || valid[t]);
        const float z = dz[static_cast<size_t>(t) * E + e];
        const float a = live ? z : 0.f;
#pragma unroll
        for (int f = 0; f < 4; ++f) {
            const float xv = load_f32(x + static_cast<size_t>(t) * d + c0 + 16 * f + l16);
            acc[f] = __builtin_amdgcn_mfma_f32_16x16x4f32(a, live ? xv : 0.f, acc[f], 0, 0, 0);
        }
    }
    float* const o = out + static_cast<size_t>(blockIdx.z) * E * d;
#pragma unroll
    for (int f = 0; f < 4; ++f)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int row = e0 + 4 * lk + i;
            if (row < E) o[static_cast<size_t>(row) * d + c0 + 16 * f + l16] = acc[f][i];
        }
}

__global__ __launch_bounds__(256) void dw_join_kernel(const float* __restrict__ part, int splits, int64_t n, float scale,
                                                      float* dw) {
    const int64_t i = 4 * (blockIdx.x * int64_t(256) + threadIdx.x);
    if (i >= n) return;
    f32x4 s = *reinterpret_cast<const f32x4*>(part + i);
    for (int k = 1; k < splits; ++k) s += *reinterpret_cast<const f32x4*>(part + k * n + i);
    *reinterpret_cast<f32x4*>(dw + i) = s * scale;
}

template <int J>
hipError_t launch_rows(const eat_params_t& p, const BalancePlan& b, const BalanceCall& c, const StatArgs& a, float* dz,
                       bool grads, hipStream_t s) {
    stat_kernel<J><<<b.blocks, kStatThreads, 0, s>>>(a);
    if (grads && c.T > 0) {
        int ep = 1;
        while (ep < std::min(p.E, 64)) ep *= 2;
        const int per = kDzWaves * (kWave / ep);
        dz_kernel<J><<<(c.T + per - 1) / per, kDzWaves * kWave, 0, s>>>(c.prob, c.valid, c.T, p.E, a.q, dz);
    }
    return hipGetLastError();
}

template <typename XT>
hipError_t launch_products(const eat_params_t& p, const BalancePlan& b, const BalanceCall& c, const float* dz, float* dwp,
                           hipStream_t s) {
    const int E = p.E, d = p.d_model;
    if (c.dw) {
        dw_kernel<XT><<<dim3((E + 63) / 64, d / 64, b.splits), 256, 0, s>>>(dz, static_cast<const XT*>(c.x), c.valid, c.T, E,
                                                                           d, dwp);
        const int64_t n = static_cast<int64_t>(E) * d;
        dw_join_kernel<<<static_cast<int>((n / 4 + 255) / 256), 256, 0, s>>>(dwp, b.splits, n, p.inv_temperature, c.dw);
    }
    if (c.dx && c.T > 0)
        dx_kernel<XT><<<dim3((c.T + 63) / 64, d / 64), 256, 0, s>>>(dz, c.w_router, c.T, E, d, p.inv_temperature,
                                                                     static_cast<XT*>(c.dx));
    return hipGetLastError();
}

}  // namespace

BalancePlan plan_balance(const eat_params_t& p, int32_t T) {
    BalancePlan b{};
    size_t off = 0;
    auto take = [&](size_t bytes) { const size_t at = off; off += (bytes + 255) & ~size_t(255); return at; };
    b.blocks = std::max(1, std::min(kStatBlocks, (T + 63) / 64));
    const int64_t items = static_cast<int64_t>((p.E + 63) / 64) * (p.d_model / 64);
    b.splits = 1;
    while (items * b.splits * 2 <= 1024 && T / (b.splits * 2) >= 64) b.splits *= 2;
    b.head = take(4);
    b.q = take(static_cast<size_t>(p.E) * 4);
    b.sum = take(static_cast<size_t>(b.blocks) * p.E * 8);
    b.cnt = take(static_cast<size_t>(b.blocks) * (p.E + 1) * 4);
    b.dz = take(static_cast<size_t>(T) * p.E * 4);
    b.dwp = take(static_cast<size_t>(b.splits) * p.E * p.d_model * 4);
    b.total = off;
    return b;
}

hipError_t launch_balance(const eat_params_t& p, const BalancePlan& b, const BalanceCall& c, char* ws, hipStream_t s) {
    const StatArgs a{c.prob, c.mask, c.valid, c.T, p.E, c.coef, c.entropy_coef, reinterpret_cast<int32_t*>(ws + b.head),
                     reinterpret_cast<float*>(ws + b.q), reinterpret_cast<double*>(ws + b.sum),
                     reinterpret_cast<int32_t*>(ws + b.cnt), c.loss, c.count, c.mean_prob};
    float* const dz = c.dlogits ? c.dlogits : reinterpret_cast<float*>(ws + b.dz);
    const bool grads = c.dlogits || c.dx || c.dw;
    clear_kernel<<<1, 1, 0, s>>>(a.head);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    switch ((p.E + 63) / 64) {
        case 1: e = launch_rows<1>(p, b, c, a, dz, grads, s); break;
        case 2: e = launch_rows<2>(p, b, c, a, dz, grads, s); break;
        case 3: e = launch_rows<3>(p, b, c, a, dz, grads, s); break;
        default: e = launch_rows<4>(p, b, c, a, dz, grads, s); break;
    }
    if (e != hipSuccess || (!c.dx && !c.dw)) return e;
    float* const dwp = reinterpret_cast<float*>(ws + b.dwp);
    return p.act_dtype == EAT_BF16 ? launch_products<uint16_t>(p, b, c, dz, dwp, s)
                                   : launch_products<float>(p, b, c, dz, dwp, s);
}

}  // namespace eat
