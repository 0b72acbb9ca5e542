// The router's balance loss with per-expert counts and gradients (gfx950).
//
// stat_kernel sums the probabilities (fp64) and counts the selections of every
// expert, a share of the tokens per workgroup (and lists the tokens that count,
// in a workgroup beside them); total_kernel adds the shares in order (adding them in
// every workgroup of prep_kernel took 10 us longer, in the last of stat_kernel's to
// finish 4 us); prep_kernel makes the scores' gradient dz = p (q - <q, p>) / n
// row by row, q = dloss / dP.
//
// The products of dz with the router weights (dx) and with x (dW_r), small
// calls: product_kernel on fp32 matrix instructions, straight from memory, both
// products in one launch.  Larger ones: the bf16 instructions, which are 16 times
// as fast, on
// fp32 numbers written as sums of bf16 parts (each part the rounding of what the
// ones before leave, so three hold 24 bits or more, two 16): dz in three parts, x
// as it is (bf16) or in three, the router weights in two (dx in bf16) or three.
// dW_r takes every product of parts, dx those above its precision (loss_gemm's
// GROUPS).  Tokens that do not count are left out of the reduction (loss_gemm's
// GATHER), so nothing of theirs is read.
//
// Bounds, measured: small calls by their launches (two to four that wait for each
// other: 256 tokens, 64 experts, d 2048, dW_r only: 25 us, its bytes are 0.4); large
// ones by the matrix instructions on the parts (16384 tokens, 256 experts, d 4096:
// 242 - 254 us, of which dx 105 and dW_r 97, at 0.98 and 1.06 PFLOP/s of bf16
// products); in between by both (8000 tokens, 60 experts, d 2048: 56 us, 63 MB).
#include <math.h>

#include <algorithm>

#include "loss_gemm.h"

namespace eat {
namespace {

constexpr int kStatWaves = 16;
constexpr int kStatThreads = kStatWaves * kWave;
constexpr int kStatBlocks = 64;           // most shares of the tokens

// dz of a row whose lanes (EP of them, E rounded up to a power of two up to 64)
// hold experts e0 + 64 j: p (q - <q, p>), <q, p> in fp64.  Not `live` (or no
// expert): 0, whatever q holds (a token that counts may have made it NaN).
template <int J>
__device__ __forceinline__ void score_grad(const float (&p)[J], const float (&q)[J], int ep, bool live, int e0, int E,
                                           float (&dz)[J]) {
    double s = 0.0;
#pragma unroll
    for (int j = 0; j < J; ++j) s += static_cast<double>(q[j]) * p[j];
    if (J > 1 || ep == kWave) s = wave_sum(s);
    else
        for (int o = ep / 2; o >= 1; o /= 2) s += __shfl_xor(s, o, kWave);
#pragma unroll
    for (int j = 0; j < J; ++j) dz[j] = live && 64 * j + e0 < E ? p[j] * static_cast<float>(q[j] - s) : 0.f;
}

struct StatArgs {
    const float* prob;
    const uint64_t* mask;
    const uint8_t* valid;
    int T, E, blocks;          // blocks: shares of the tokens
    float coef, entropy_coef;
    float* q;                  // [E] dloss / dP_e / max(n, 1) (of one workgroup)
    double* sum;               // [blocks][E] (of several)
    int32_t* cnt;              // [blocks][E + 1]: selections, then valid tokens
    float* loss;
    int64_t* count;
    float* mean_prob;
    float* dz;                 // one workgroup: [T][E], made here too (or null)
    int32_t* rows;             // the valid tokens' list, made by a workgroup more (or null)
    int32_t* head;             // {n, n in whole chunks, .} of it
};

// From the totals (a thread per expert: the sum of its probabilities, its
// selections; `tokens`, thread 0's, those that count) q into qs (LDS) and the
// call's results out.  Every thread of the workgroup calls it; a thread's q is
// its own until a barrier.
struct Totals {
    double loss[4];
    int sel[4], tokens;
};
__device__ __forceinline__ void finish(const StatArgs& a, double sum, int sel, int tokens, float* qs, Totals& s) {
    const int tid = threadIdx.x, wave = tid / kWave, E = a.E;
    // (a call's selections are below 2^31: max_tokens times the most experts of a token is)
    const int part = wave_sum(tid < E ? sel : 0);
    if (lane_id() == 0 && wave < 4) s.sel[wave] = part;
    if (tid == 0) s.tokens = tokens;
    __syncthreads();
    const double inv = 1.0 / max(s.tokens, 1), p = sum * inv;
    const double f = static_cast<double>(sel) / max(s.sel[0] + s.sel[1] + s.sel[2] + s.sel[3], 1);
    const double lg = p > 0.0 ? log(p) : p == 0.0 ? 0.0 : p;      // (NaN stays)
    if (tid < E) {
        qs[tid] = static_cast<float>((a.coef * E * f + a.entropy_coef * (lg + 1.0)) * inv);
        if (a.count) a.count[tid] = sel;
        if (a.mean_prob) a.mean_prob[tid] = static_cast<float>(p);
    }
    const double l = wave_sum(tid < E ? a.coef * E * f * p + a.entropy_coef * p * lg : 0.0);
    if (lane_id() == 0 && wave < 4) s.loss[wave] = l;
    __syncthreads();
    if (tid == 0) *a.loss = static_cast<float>((s.loss[0] + s.loss[1]) + (s.loss[2] + s.loss[3]));
}

// Lane l holds experts l % EP + 64 j of token l / EP of a group of 64 / EP
// tokens (EP: E rounded up to a power of two, 64 at most); a wave has kStatRows
// groups' loads in flight.
template <int J>
__global__ __launch_bounds__(kStatThreads) void stat_kernel(StatArgs a) {
    constexpr int kStatRows = J <= 2 ? 8 : 4;
    __shared__ double red[kStatWaves][kWave * J];
    __shared__ int redc[kStatWaves][kWave * J];
    __shared__ int redn[kStatWaves];
    __shared__ Totals totals;
    if (static_cast<int>(blockIdx.x) == a.blocks) {
        list_rows<uint8_t>(a.valid, a.T, 0, a.rows, a.head);
        return;
    }
    const int lane = lane_id(), wave = threadIdx.x / kWave, tid = threadIdx.x;
    const int E = a.E;
    int ep = 1;
    while (ep < min(E, 64)) ep *= 2;
    const int sub = lane / ep, e0 = lane % ep, tpw = kWave / ep;
    const int per = (a.T + a.blocks - 1) / a.blocks;
    const int tbeg = min(a.T, static_cast<int>(blockIdx.x) * per), tend = min(a.T, tbeg + per);
    double s[J];
    int c[J], n = 0;
#pragma unroll
    for (int j = 0; j < J; ++j) { s[j] = 0.0; c[j] = 0; }
    for (int t0 = tbeg + wave * tpw * kStatRows; t0 < tend; t0 += kStatWaves * tpw * kStatRows) {
        float p[kStatRows][J];
        uint64_t m[kStatRows][J];
        bool live[kStatRows];
        // (every load is unconditional, of a token and an expert that exist)
#pragma unroll
        for (int u = 0; u < kStatRows; ++u) {
            const int t = t0 + u * tpw + sub, ts = min(t, tend - 1);
            live[u] = t < tend && (!a.valid || a.valid[ts]);
#pragma unroll
            for (int j = 0; j < J; ++j) {
                p[u][j] = a.prob[static_cast<size_t>(ts) * E + min(64 * j + e0, E - 1)];
                m[u][j] = a.mask[static_cast<size_t>(ts) * J + j];
            }
        }
#pragma unroll
        for (int u = 0; u < kStatRows; ++u) {
            n += live[u] && e0 == 0;
#pragma unroll
            for (int j = 0; j < J; ++j) {
                const bool on = live[u] && 64 * j + e0 < E;
                s[j] += on ? static_cast<double>(p[u][j]) : 0.0;
                c[j] += on ? static_cast<int>((m[u][j] >> e0) & 1) : 0;
            }
        }
    }
    for (int o = ep; o < kWave; o *= 2)
#pragma unroll
        for (int j = 0; j < J; ++j) {
            s[j] += __shfl_xor(s[j], o, kWave);
            c[j] += __shfl_xor(c[j], o, kWave);
        }
    n = wave_sum(n);
    if (lane == 0) redn[wave] = n;
#pragma unroll
    for (int j = 0; j < J; ++j) {
        red[wave][64 * j + lane] = s[j];
        redc[wave][64 * j + lane] = c[j];
    }
    __syncthreads();
    // an expert per thread: the waves' sums in order
    double t = 0.0;
    int k = 0, nn = 0;
    if (tid < E) {
#pragma unroll
        for (int w = 0; w < kStatWaves; ++w) {
            t += red[w][tid];
            k += redc[w][tid];
        }
    }
    if (wave == 0) nn = wave_sum(lane < kStatWaves ? redn[lane] : 0);
    if (a.blocks > 1) {                       // (added up by total_kernel)
        if (tid < E) {
            a.sum[static_cast<size_t>(blockIdx.x) * E + tid] = t;
            a.cnt[static_cast<size_t>(blockIdx.x) * (E + 1) + tid] = k;
        }
        if (tid == 0) a.cnt[static_cast<size_t>(blockIdx.x) * (E + 1) + E] = nn;
        return;
    }
    __syncthreads();
    float* const qs = reinterpret_cast<float*>(red);
    finish(a, t, k, nn, qs, totals);
    __syncthreads();
    if (tid < E) a.q[tid] = qs[tid];
    if (!a.dz) return;
    // small calls: the scores' gradient without a launch of its own
    float q[J];
#pragma unroll
    for (int j = 0; j < J; ++j) q[j] = 64 * j + e0 < E ? qs[64 * j + e0] : 0.f;
    for (int t0 = wave * tpw * kStatRows; t0 < a.T; t0 += kStatWaves * tpw * kStatRows) {
        float p[kStatRows][J];
        bool live[kStatRows];
#pragma unroll
        for (int u = 0; u < kStatRows; ++u) {
            const int t = t0 + u * tpw + sub, ts = min(t, a.T - 1);
            live[u] = t < a.T && (!a.valid || a.valid[ts]);
#pragma unroll
            for (int j = 0; j < J; ++j) {
                const float v = a.prob[static_cast<size_t>(ts) * E + min(64 * j + e0, E - 1)];
                p[u][j] = live[u] && 64 * j + e0 < E ? v : 0.f;
            }
        }
#pragma unroll
        for (int u = 0; u < kStatRows; ++u) {
            const int t = t0 + u * tpw + sub;
            float dz[J];
            score_grad<J>(p[u], q, ep, live[u], e0, E, dz);
#pragma unroll
            for (int j = 0; j < J; ++j)
                if (t < a.T && 64 * j + e0 < E) a.dz[static_cast<size_t>(t) * E + 64 * j + e0] = dz[j];
        }
    }
}

// The shares of several workgroups: a wave adds those of its residue, a lane per
// expert, a thread per expert the waves' in order.
template <int J>
__global__ __launch_bounds__(kStatThreads) void total_kernel(StatArgs a) {
    __shared__ double red[kStatWaves][kWave * J];
    __shared__ int redc[kStatWaves][kWave * J];
    __shared__ float qs[kMaxExperts];
    __shared__ Totals totals;
    const int lane = lane_id(), wave = threadIdx.x / kWave, tid = threadIdx.x;
    const int E = a.E;
    constexpr int N = kStatBlocks / kStatWaves;
    double v[N][J];
    int c[N][J];
    const int tokens = wave_sum(lane < a.blocks ? a.cnt[static_cast<size_t>(min(lane, a.blocks - 1)) * (E + 1) + E] : 0);
    static_assert(kStatBlocks <= kWave, "a lane per share");
#pragma unroll
    for (int u = 0; u < N; ++u)
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const int b = min(wave + u * kStatWaves, a.blocks - 1), e = min(64 * j + lane, E - 1);
            v[u][j] = a.sum[static_cast<size_t>(b) * E + e];
            c[u][j] = a.cnt[static_cast<size_t>(b) * (E + 1) + e];
        }
#pragma unroll
    for (int j = 0; j < J; ++j) {
        double s = 0.0;
        int k = 0;
#pragma unroll
        for (int u = 0; u < N; ++u)
            if (wave + u * kStatWaves < a.blocks) {
                s += v[u][j];
                k += c[u][j];
            }
        red[wave][64 * j + lane] = s;
        redc[wave][64 * j + lane] = k;
    }
    __syncthreads();
    double t = 0.0;
    int k = 0;
    if (tid < E) {
#pragma unroll
        for (int w = 0; w < kStatWaves; ++w) {
            t += red[w][tid];
            k += redc[w][tid];
        }
    }
    finish(a, t, k, tokens, qs, totals);
    if (tid < E) a.q[tid] = qs[tid];
}

// v as a sum of three bf16 numbers, largest first
__device__ __forceinline__ void split3(float v, uint16_t (&part)[3]) {
#pragma unroll
    for (int i = 0; i < 3; ++i) {
        part[i] = f32_to_bf16(v);
        v -= bf16_to_f32(part[i]);
    }
}

struct PrepArgs {
    StatArgs stat;
    const int32_t* rows;       // tokens that count, or null: all (valid null, or dz in token order alone)
    int d;
    float* dz;                 // [T][E], or null
    uint16_t* dzs;             // [list row][group][4][64] parts, or null
    void* dx;                  // rows to clear where the token does not count, or null
    int row_bytes;             // of dx
    const float* w;            // [E][d]
    uint16_t* ws;              // dx's stack of w's parts ([group][segs][64][d]), or null
    int segs, map;             // part of w in each
    const float* x;            // fp32 x to split
    uint16_t* xs;              // [list row][3][d], or null
    int blocks_z, blocks_w, blocks_x;      // workgroups of each kind of work
};
// A grid has fewer than 2^32 threads: 256 of them in each of this many
// workgroups at most, which go on to the next piece of work beyond.
constexpr int kMostBlocks = 1 << 22;

constexpr int kPrepWaves = 4;
constexpr int kPrepThreads = kPrepWaves * kWave;
template <int J>
__global__ __launch_bounds__(kPrepThreads) void prep_kernel(PrepArgs a) {
    const int lane = lane_id(), wave = threadIdx.x / kWave;
    const int E = a.stat.E, T = a.stat.T;
    const int block = blockIdx.x;
    const int n = a.rows ? a.stat.head[0] : T, padded = (n + kBK - 1) / kBK * kBK;
    if (block >= a.blocks_z + a.blocks_w) {               // x: a list row per workgroup
        for (int i = block - a.blocks_z - a.blocks_w; i < padded; i += a.blocks_x) {
            const bool live = i < n;
            const int t = live && a.rows ? a.rows[i] : i;
            for (int c = 4 * threadIdx.x; c < a.d; c += 4 * kPrepThreads) {
                f32x4 v{};
                if (live) v = *reinterpret_cast<const f32x4*>(a.x + static_cast<size_t>(t) * a.d + c);
                uint16_t p[4][3];
#pragma unroll
                for (int e = 0; e < 4; ++e) split3(v[e], p[e]);
#pragma unroll
                for (int k = 0; k < 3; ++k)
                    *reinterpret_cast<uint2*>(a.xs + (static_cast<size_t>(i) * 3 + k) * a.d + c) =
                        uint2{p[0][k] | static_cast<uint32_t>(p[1][k]) << 16, p[2][k] | static_cast<uint32_t>(p[3][k]) << 16};
            }
        }
        return;
    }
    if (block >= a.blocks_z) {                            // w: an expert (or a row of zeros) per workgroup
        const int e = block - a.blocks_z, grp = e / 64;
        for (int c = 4 * threadIdx.x; c < a.d; c += 4 * kPrepThreads) {
            f32x4 v{};
            if (e < E) v = *reinterpret_cast<const f32x4*>(a.w + static_cast<size_t>(e) * a.d + c);
            uint16_t p[4][3];
#pragma unroll
            for (int k = 0; k < 4; ++k) split3(v[k], p[k]);
            for (int sg = 0; sg < a.segs; ++sg) {
                const int k = (a.map >> (4 * sg)) & 15;
                auto pick = [&](int u) { return k == 0 ? p[u][0] : k == 1 ? p[u][1] : p[u][2]; };
                *reinterpret_cast<uint2*>(a.ws + ((static_cast<size_t>(grp) * a.segs + sg) * 64 + e % 64) * a.d + c) =
                    uint2{pick(0) | static_cast<uint32_t>(pick(1)) << 16, pick(2) | static_cast<uint32_t>(pick(3)) << 16};
            }
        }
        return;
    }
    // lane l: experts l % EP + 64 j of row l / EP of a group
    int ep = 1;
    while (ep < min(E, 64)) ep *= 2;
    const int sub = lane / ep, e0 = lane % ep, tpw = kWave / ep;
    float q[J];
#pragma unroll
    for (int j = 0; j < J; ++j) q[j] = 64 * j + e0 < E ? a.stat.q[64 * j + e0] : 0.f;
    // the row of the list at this place (without a list: the token)
    const int i = (block * kPrepWaves + wave) * tpw + sub;
    const bool live = i < n && (a.rows || !a.stat.valid || a.stat.valid[min(i, T - 1)]);
    const int t = n == 0 ? 0 : a.rows ? a.rows[min(i, n - 1)] : min(i, T - 1);
    float p[J], dz[J];
#pragma unroll
    for (int j = 0; j < J; ++j) {
        const float v = a.stat.prob[static_cast<size_t>(t) * E + min(64 * j + e0, E - 1)];
        p[j] = live && 64 * j + e0 < E ? v : 0.f;
    }
    score_grad<J>(p, q, ep, live, e0, E, dz);
#pragma unroll
    for (int j = 0; j < J; ++j) {
        const int e = 64 * j + e0;
        if (a.dz && live && e < E) a.dz[static_cast<size_t>(t) * E + e] = dz[j];
        if (a.dzs && i < padded) {
            uint16_t part[3];
            split3(dz[j], part);
            uint16_t* const o = a.dzs + (static_cast<size_t>(i) * J + j) * 256;
#pragma unroll
            for (int k = 0; k < 3; ++k) {
                o[64 * k + e0] = part[k];
                for (int z = e0 + ep; z < 64; z += ep) o[64 * k + z] = 0;
            }
        }
    }
    // the token at this place: cleared where it does not count
    if (i < T && a.stat.valid && !a.stat.valid[i]) {
        if (a.dz)
            for (int e = e0; e < E; e += ep) a.dz[static_cast<size_t>(i) * E + e] = 0.f;
        if (a.dx)
            for (int c = 16 * e0; c < a.row_bytes; c += 16 * ep)
                *reinterpret_cast<uint4*>(static_cast<char*>(a.dx) + static_cast<size_t>(i) * a.row_bytes + c) = uint4{};
    }
}

__device__ __forceinline__ float load_f32(const float* p) { return *p; }
__device__ __forceinline__ float load_f32(const uint16_t* p) { return bf16_to_f32(*p); }
__device__ __forceinline__ void store_f32(float* p, float v) { *p = v; }
__device__ __forceinline__ void store_f32(uint16_t* p, float v) { *p = f32_to_bf16(v); }

// The products of small calls, fp32 matrix instructions on operands straight
// from memory, kSteps of 4 reduction elements' loads in flight: 64 columns and
// 16 rows per wave, 64 rows per workgroup.  Workgroups below blocks_w make
// dW_r (rows: experts; reduction: a slice of the tokens, those that are not
// valid read as zeros), the others dx (rows: tokens; reduction: experts).
constexpr int kSteps = 8;
struct ProductArgs {
    const float* dz;
    const void* x;
    const float* w;
    const uint8_t* valid;
    int T, E, d, splits;
    int64_t blocks_w, blocks_x;
    float scale;
    float* dw;                 // dW_r where splits is 1
    float* dwp;                // else its slices [splits][E][d], unscaled
    void* dx;
};
// out[r][c] = scale sum_k dz[r rs + k ks] v[k][c] over k in [kbeg, kend), those
// whose valid[k] is 0 left out, for rows r0 .. r0 + 63 and columns c0 .. c0 + 63;
// 0 in rows whose live[r] is 0 (v may hold infinities).  valid, live: null, all.
template <typename VT, typename OT>
__device__ __forceinline__ void product_tile(const float* dz, int rs, int ks, const VT* v, const uint8_t* valid, int kbeg,
                                             int kend, int rows, int r0, const uint8_t* live, int d, int c0, float scale,
                                             OT* out) {
    const int lane = lane_id(), wave = threadIdx.x / kWave;
    const int l16 = lane & 15, lk = lane >> 4;
    r0 += 16 * wave;
    const float* const zr = dz + static_cast<size_t>(min(r0 + l16, rows - 1)) * rs;
    f32x4 acc[4] = {};
    for (int k0 = kbeg; k0 < kend; k0 += 4 * kSteps) {
        float z[kSteps], x[kSteps][4];
        uint8_t ok[kSteps];
#pragma unroll
        for (int s = 0; s < kSteps; ++s) ok[s] = 1;
        if (valid) {
#pragma unroll
            for (int s = 0; s < kSteps; ++s) ok[s] = valid[min(k0 + 4 * s + lk, kend - 1)];
        }
        // (every load is unconditional, of a reduction element that exists)
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
            const int k = min(k0 + 4 * s + lk, kend - 1);
            z[s] = zr[static_cast<size_t>(k) * ks];
#pragma unroll
            for (int f = 0; f < 4; ++f) x[s][f] = load_f32(v + static_cast<size_t>(k) * d + c0 + 16 * f + l16);
        }
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
            const bool on = k0 + 4 * s + lk < kend && ok[s];
#pragma unroll
            for (int f = 0; f < 4; ++f)
                acc[f] = __builtin_amdgcn_mfma_f32_16x16x4f32(on ? z[s] : 0.f, on ? x[s][f] : 0.f, acc[f], 0, 0, 0);
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int r = r0 + 4 * lk + i;
        const bool on = !live || live[min(r, rows - 1)];
#pragma unroll
        for (int f = 0; f < 4; ++f)
            if (r < rows) store_f32(out + static_cast<size_t>(r) * d + c0 + 16 * f + l16, on ? acc[f][i] * scale : 0.f);
    }
}

template <typename XT>
__global__ __launch_bounds__(256) void product_kernel(ProductArgs a) {
    const int cols = a.d / 64;
    for (int64_t at = blockIdx.x; at < a.blocks_w + a.blocks_x; at += gridDim.x) {
        const bool dw = at < a.blocks_w;
        const int block = static_cast<int>(dw ? at : at - a.blocks_w);
        const int c0 = block % cols * 64, b = block / cols;
        if (dw) {
            const int tiles = (a.E + 63) / 64, sp = b / tiles;
            const int per = ((a.T + a.splits - 1) / a.splits + 3) / 4 * 4;
            const int kbeg = min(a.T, sp * per), kend = min(a.T, kbeg + per);
            float* const out = a.splits == 1 ? a.dw : a.dwp + static_cast<size_t>(sp) * a.E * a.d;
            product_tile(a.dz, 1, a.E, static_cast<const XT*>(a.x), a.valid, kbeg, kend, a.E, b % tiles * 64, nullptr, a.d, c0,
                         a.splits == 1 ? a.scale : 1.f, out);
        } else {
            product_tile(a.dz, a.E, 1, a.w, nullptr, 0, a.E, a.T, b * 64, a.valid, a.d, c0, a.scale, static_cast<XT*>(a.dx));
        }
    }
}

// dW_r: the slices' rows of `parts` blocks of d added in order, times scale.
__global__ __launch_bounds__(256) void dw_join_kernel(const float* __restrict__ part, int splits, int parts, int E, int d,
                                                      float scale, float* dw) {
    const int64_t i = 4 * (blockIdx.x * int64_t(256) + threadIdx.x), n = static_cast<int64_t>(E) * d;
    if (i >= n) return;
    const int64_t e = i / d, c = i % d;
    f32x4 s{};
    for (int k = 0; k < splits; ++k)
        for (int u = 0; u < parts; ++u)
            s += *reinterpret_cast<const f32x4*>(part + (k * static_cast<int64_t>(E) + e) * parts * d + u * static_cast<int64_t>(d) + c);
    *reinterpret_cast<f32x4*>(dw + i) = s * scale;
}


// Most probabilities that one workgroup sums up, of 1024 tokens at most: two
// launches less (whole calls, one workgroup | many: 256 x 64: 25 | 31 us;
// 1024 x 8: 25 | 32; 1024 x 32: 42 | 32; 2048 x 8: 36 | 32).
constexpr int kOneBlock = 16384;

// Whether the products run on bf16 parts (more launches, faster products) or on
// fp32 instructions, by measured times of whole calls (fp32 instructions |
// parts, us).  bf16 tokens, three products of parts each for dx and dW_r:
//   T 16384, E 8, d 64: 55 | 47;  E 64, d 512: 73 | 56;  E 256, d 128: 78 | 77
//   T 8192, E 8, d 512: 39 | 42;  E 256, d 512: 93 | 67
//   T 4096, E 64, d 512: 36 | 40;  d 2048: 59 | 44;  E 256, d 512: 61 | 60
//   T 2048, E 64, d 2048: 38 | 40;  T 3000: 49 | 45
//   T 1024, E 64, d 4096: 35 | 41;  T 512, E 256, d 4096: 50 | 59, d 8192: 89 | 65
// fp32 tokens are three parts, so six products for dx and nine for dW_r:
//   T 2048, E 256, d 2048: 85 | 90;  d 4096: 152 | 120;  T 16384: 1056 | 741
//   T 16384, E 64, d 4096: 310 | 350;  T 65536, E 8: 850 | 1263
// (A row of x's parts is addressed with 24 bits.)
bool split_products(const eat_params_t& p, int32_t T) {
    if (p.d_model > 1 << 20) return false;
    const int64_t work = static_cast<int64_t>(T) * p.d_model;
    if (p.act_dtype != EAT_BF16) return p.E > 64 && work * p.E >= int64_t{1} << 31;
    return T >= 16384 || work * ((p.E + 63) / 64 * 64) >= int64_t{1} << (T >= 2048 ? 29 : 30);
}

template <int J>
hipError_t launch_rows(const eat_params_t& p, const BalancePlan& b, const StatArgs& a, const PrepArgs* prep, int blocks,
                       hipStream_t s) {
    stat_kernel<J><<<b.blocks + (a.rows ? 1 : 0), kStatThreads, 0, s>>>(a);
    if (b.blocks > 1) total_kernel<J><<<1, kStatThreads, 0, s>>>(a);
    if (prep && blocks) prep_kernel<J><<<blocks, kPrepThreads, 0, s>>>(*prep);
    return hipGetLastError();
}

template <typename XT>
hipError_t launch_products(const eat_params_t& p, const BalancePlan& b, const BalanceCall& c, const float* dz, float* dwp,
                           hipStream_t s) {
    const int E = p.E, d = p.d_model;
    const int64_t bw = c.dw ? int64_t{(E + 63) / 64} * (d / 64) * b.splits : 0;
    const int64_t bx = c.dx ? int64_t{(c.T + 63) / 64} * (d / 64) : 0;
    if (bw > INT32_MAX || bx > INT32_MAX) return hipErrorInvalidConfiguration;
    const ProductArgs a{dz, c.x, c.w_router, c.valid, c.T, E, d, b.splits, bw, bx, p.inv_temperature, c.dw, dwp, c.dx};
    if (bw + bx > 0) product_kernel<XT><<<static_cast<int>(std::min<int64_t>(bw + bx, kMostBlocks)), 256, 0, s>>>(a);
    if (c.dw && b.splits > 1)
        dw_join_kernel<<<static_cast<int>((static_cast<int64_t>(E) * d / 4 + 255) / 256), 256, 0, s>>>(
            dwp, b.splits, 1, E, d, p.inv_temperature, c.dw);
    return hipGetLastError();
}

// Parts of dz (low nibble first) and of the router weights that meet in dx:
// bf16 rows keep 2^-8, so the products of parts down to 2^-16 of the largest do;
// fp32 rows take those down to 2^-24.
constexpr int kSegs16 = 3, kDz16 = 0x010, kW16 = 0x100;
constexpr int kSegs32 = 6, kDz32 = 0x211000, kW32 = 0x010210;

hipError_t launch_split(const eat_params_t& p, const BalancePlan& b, const BalanceCall& c, const int32_t* rows,
                        const int32_t* head, char* ws, hipStream_t s) {
    const int E = p.E, d = p.d_model, groups = (E + 63) / 64;
    const bool bf16 = p.act_dtype == EAT_BF16;
    const uint16_t* const dzs = reinterpret_cast<const uint16_t*>(ws + b.dzs);
    hipError_t e = hipSuccess;
    if (c.dw) {
        float* const dwp = reinterpret_cast<float*>(ws + b.dwp);
        const int parts = bf16 ? 1 : 3;
        GemmArgs g{};
        g.a = bf16 ? static_cast<const uint16_t*>(c.x) : reinterpret_cast<const uint16_t*>(ws + b.xs);
        g.lda = g.na = parts * d;
        g.a_rows = bf16 ? c.T : 1 << 30;
        g.k_rows = rows;
        g.b = dzs; g.ldb = 256 * groups; g.nb = E;
        g.K = (c.T + kBK - 1) / kBK * kBK; g.k_dev = rows ? head + 1 : nullptr; g.k_times = 1;
        g.splits = b.splits;
        g.out = dwp; g.ldo = parts * d; g.split_stride = static_cast<int64_t>(E) * parts * d;
        e = bf16 && rows ? launch_gemm<Big, true, true, PART, GROUPS, true>(g, s)
                         : launch_gemm<Big, true, true, PART, GROUPS, false>(g, s);
        if (e == hipSuccess) {
            dw_join_kernel<<<static_cast<int>((static_cast<int64_t>(E) * d / 4 + 255) / 256), 256, 0, s>>>(
                dwp, b.splits, parts, E, d, p.inv_temperature, c.dw);
            e = hipGetLastError();
        }
    }
    if (c.dx && e == hipSuccess) {
        GemmArgs g{};
        g.segs = bf16 ? kSegs16 : kSegs32;
        g.map = bf16 ? kDz16 : kDz32;
        g.K = g.a_rows = groups * g.segs * 64;
        g.a = reinterpret_cast<const uint16_t*>(ws + b.ws); g.lda = g.na = d;
        g.b = dzs; g.ldb = 256 * groups; g.nb = c.T; g.nb_dev = rows ? head : nullptr;
        g.splits = 1;
        g.out = c.dx; g.ldo = d; g.rows = rows; g.factor = p.inv_temperature;
        e = bf16 ? launch_gemm<Big, true, false, ROWS, GROUPS>(g, s) : launch_gemm<Big, true, false, ROWS32, GROUPS>(g, s);
    }
    return e;
}

}  // namespace

BalancePlan plan_balance(const eat_params_t& p, int32_t T) {
    BalancePlan b{};
    size_t off = 0;
    auto take = [&](size_t bytes) { const size_t at = off; off += (bytes + 255) & ~size_t(255); return at; };
    // (one workgroup needs no meeting of several, and makes dz of a small call as well)
    b.blocks = T <= 1024 && static_cast<int64_t>(T) * p.E <= kOneBlock ? 1 : std::min(kStatBlocks, (T + 63) / 64);
    b.split = split_products(p, T);
    const size_t groups = (p.E + 63) / 64, d = p.d_model, pad = (static_cast<size_t>(T) + 255) / 256 * 256;
    const int parts = b.split && p.act_dtype != EAT_BF16 ? 3 : 1;
    // dw_router: slices of the tokens, joined by a launch.  On parts about 512 tokens
    // each, 64 at most, while the CUs have no two items (T 16384, E 8, d 1024: 512
    // tokens 53 us, 384 56, 256 61, 1024 56; T 65536, E 64, d 512: 64 slices 107, 32
    // 112, 128 122).  On fp32 instructions, of smaller tiles, until there are four
    // items per CU, none under 512 tokens, or 128 while CUs would idle (T
    // 16384, E 64, d 256: 64 slices of 256 tokens 59 us, 128 of 128 76, 32 of 512 63).
    const int64_t items = b.split ? groups * ((parts * d + Big::NA - 1) / Big::NA) : groups * (d / 64);
    b.splits = 1;
    if (b.split)
        b.splits = static_cast<int>(std::max<int64_t>(1, std::min<int64_t>({64, 256 / items, (T + 511) / 512})));
    else
        for (int n = 2; items * n <= 1024 && n <= 256; n *= 2)
            if (T / n >= (items * n > 256 ? 512 : 128)) b.splits = n;
    b.head = take(12);
    b.rows = take(b.split ? pad * 4 : 0);
    b.q = take(static_cast<size_t>(p.E) * 4);
    b.sum = take(static_cast<size_t>(b.blocks) * p.E * 8);
    b.cnt = take(static_cast<size_t>(b.blocks) * (p.E + 1) * 4);
    b.dz = take(b.split ? 0 : static_cast<size_t>(T) * p.E * 4);
    b.dzs = take(b.split ? pad * groups * 256 * 2 : 0);
    b.ws = take(b.split ? groups * (p.act_dtype == EAT_BF16 ? kSegs16 : kSegs32) * 64 * d * 2 : 0);
    b.xs = take(parts == 3 ? pad * 3 * d * 2 : 0);
    b.dwp = take(static_cast<size_t>(b.splits) * parts * p.E * d * 4);
    b.total = off;
    return b;
}

hipError_t launch_balance(const eat_params_t& p, const BalancePlan& b, const BalanceCall& c, char* ws, hipStream_t s) {
    int32_t* const head = reinterpret_cast<int32_t*>(ws + b.head);
    float* const q = reinterpret_cast<float*>(ws + b.q);
    const bool products = c.dx || c.dw, split = b.split && products;
    const bool bf16 = p.act_dtype == EAT_BF16;
    int32_t* const list = split && c.valid ? reinterpret_cast<int32_t*>(ws + b.rows) : nullptr;
    float* const dz = c.dlogits ? c.dlogits : products && !split ? reinterpret_cast<float*>(ws + b.dz) : nullptr;
    const bool fused = b.blocks == 1 && !split;            // dz by the sums' workgroup
    const StatArgs a{c.prob, c.mask, c.valid, c.T, p.E, b.blocks, c.coef, c.entropy_coef, q,
                     reinterpret_cast<double*>(ws + b.sum), reinterpret_cast<int32_t*>(ws + b.cnt), c.loss, c.count,
                     c.mean_prob, fused ? dz : nullptr, list, head};
    PrepArgs r{};
    r.stat = a;
    r.rows = list;
    r.d = p.d_model;
    r.dz = dz;
    int ep = 1;
    while (ep < std::min(p.E, 64)) ep *= 2;
    const int per = kPrepWaves * (kWave / ep);
    const int places = split ? (c.T + kBK - 1) / kBK * kBK : c.T;      // rows of dz there are
    r.blocks_z = dz || split ? (places + per - 1) / per : 0;
    int blocks = r.blocks_z;
    if (split) {
        r.dzs = reinterpret_cast<uint16_t*>(ws + b.dzs);
        if (c.dx) {
            r.dx = c.dx; r.row_bytes = p.d_model * (bf16 ? 2 : 4);
            r.w = c.w_router;
            r.ws = reinterpret_cast<uint16_t*>(ws + b.ws);
            r.segs = bf16 ? kSegs16 : kSegs32;
            r.map = bf16 ? kW16 : kW32;
            r.blocks_w = (p.E + 63) / 64 * 64;
            blocks += r.blocks_w;
        }
        if (c.dw && !bf16) {
            r.x = static_cast<const float*>(c.x);
            r.xs = reinterpret_cast<uint16_t*>(ws + b.xs);
            r.blocks_x = std::min(places, kMostBlocks);
            blocks += r.blocks_x;
        }
    }
    const PrepArgs* const rp = (dz && !fused) || split ? &r : nullptr;
    hipError_t e;
    switch ((p.E + 63) / 64) {
        case 1: e = launch_rows<1>(p, b, a, rp, blocks, s); break;
        case 2: e = launch_rows<2>(p, b, a, rp, blocks, s); break;
        case 3: e = launch_rows<3>(p, b, a, rp, blocks, s); break;
        default: e = launch_rows<4>(p, b, a, rp, blocks, s); break;
    }
    if (e != hipSuccess || !products) return e;
    if (split) return launch_split(p, b, c, list, head, ws, s);
    float* const dwp = reinterpret_cast<float*>(ws + b.dwp);
    return bf16 ? launch_products<uint16_t>(p, b, c, dz, dwp, s) : launch_products<float>(p, b, c, dz, dwp, s);
}

}  // namespace eat
