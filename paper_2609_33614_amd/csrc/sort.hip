// Tokens sorted by expert and back, with their gradients (gfx950).
//
//   sort             rows[place(t, e)] = x[t] for every selected (t, e), expert-major, tokens in
//                    order inside an expert's segment; its backward dx[t] = sum_e drows[place(t, e)]
//   combine          y[t] = sum_e gate[t][e] rows[place(t, e)]
//   combine backward drows[place(t, e)] = gate[t][e] dy[t],  dg_te = <dy[t], rows[place(t, e)]>,
//                    dz_te = [e in S_t] g_te (dg_te - G) - p_te G eps / (P + eps)
//                    with G = sum_S g dg, P = sum_S p: what g = p / (P + eps) and the softmax give
//
// Everything moves rows of d elements once: bound by memory.  The places come
// from the selection masks alone: a bit transpose turns 64 tokens' masks into
// each expert's tokens as bits (eat_device.h), whose popcounts are ranks.
#include <algorithm>

#include "eat_device.h"
#include "eat_internal.h"

namespace eat {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / kWave;
// Tokens per workgroup of the index kernels: 64 keep the loop over a chunk's tokens short
// (4097 tokens, 128 experts: 12.2 us for the launches against 13.7, 300 and 256: 10.1 and 14.5), 256
// the counts of earlier chunks few (16384 tokens, 64 experts: 13.6 against 16.3; 8192: equal).
constexpr int kChunk = 256, kSmallChunk = 64, kSmallTokens = 8192;
// Up to so many 64-token words of masks every workgroup counts them all by itself (1000
// tokens, 64 experts: 9.1 us against 10.5 with a launch of counts; 130 words: 16.2 and 13.5).
constexpr int kCountPairs = 64;
constexpr int kSumChunks = 64;            // more chunks of 256 tokens' counts are added up in a launch of their own
constexpr int kBatch = 8;                 // rows of a token in flight together

// 16 bytes of a row as fp32 numbers and back.
template <typename T>
struct Vec;
template <>
struct Vec<uint16_t> {
    static constexpr int N = 8;
    static __device__ __forceinline__ void get(const uint4& q, float (&v)[8]) {
        const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[2 * i] = __uint_as_float(w[i] << 16);
            v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        }
    }
    static __device__ __forceinline__ uint4 put(const float (&v)[8]) {
        return uint4{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])};
    }
};
template <>
struct Vec<float> {
    static constexpr int N = 4;
    static __device__ __forceinline__ void get(const uint4& q, float (&v)[4]) {
        v[0] = __uint_as_float(q.x); v[1] = __uint_as_float(q.y); v[2] = __uint_as_float(q.z); v[3] = __uint_as_float(q.w);
    }
    static __device__ __forceinline__ uint4 put(const float (&v)[4]) {
        return uint4{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
    }
};

// (rows are read or written once, in bulk: past the caches)
__device__ __forceinline__ uint4 load_row(const uint4* p) {
    const u32x4 v = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p));
    return uint4{v[0], v[1], v[2], v[3]};
}
__device__ __forceinline__ void store_row(uint4* p, const uint4& q) {
    __builtin_nontemporal_store(u32x4{q.x, q.y, q.z, q.w}, reinterpret_cast<u32x4*>(p));
}

// ---- index -----------------------------------------------------------------

// Selections per expert of each chunk of tokens: cnt[chunk][E].
template <int CHUNK>
__global__ __launch_bounds__(CHUNK) void count_kernel(const uint64_t* __restrict__ mask, int T, int E, int W,
                                                      int32_t* __restrict__ cnt) {
    __shared__ int part[CHUNK / kWave][kMaxExperts];
    const int lane = lane_id(), wave = threadIdx.x / kWave;
    const int t = blockIdx.x * CHUNK + wave * kWave + lane;
    for (int w = 0; w < W; ++w)
        part[wave][kWave * w + lane] = __popcll(bit_transpose(t < T ? mask[static_cast<size_t>(t) * W + w] : 0ull));
    __syncthreads();
    for (int e = threadIdx.x; e < E; e += CHUNK) {
        int n = 0;
#pragma unroll
        for (int q = 0; q < CHUNK / kWave; ++q) n += part[q][e];
        cnt[static_cast<size_t>(blockIdx.x) * E + e] = n;
    }
}

// Per expert (a workgroup each): cnt becomes the selections in earlier chunks,
// total[e] those of all.
__global__ __launch_bounds__(kThreads) void scan_kernel(int32_t* __restrict__ cnt, int chunks, int E, int32_t* __restrict__ total) {
    __shared__ int part[kWaves];
    const int e = blockIdx.x, lane = lane_id(), wave = threadIdx.x / kWave;
    int carry = 0;
    for (int c0 = 0; c0 < chunks; c0 += kThreads) {
        const int c = c0 + static_cast<int>(threadIdx.x);
        const int n = c < chunks ? cnt[static_cast<size_t>(c) * E + e] : 0;
        const int s = wave_scan(n);
        if (lane == kWave - 1) part[wave] = s;
        __syncthreads();
        int before = carry, all = 0;
#pragma unroll
        for (int q = 0; q < kWaves; ++q) {
            before += q < wave ? part[q] : 0;
            all += part[q];
        }
        if (c < chunks) cnt[static_cast<size_t>(c) * E + e] = before + s - n;
        carry += all;
        __syncthreads();
    }
    if (threadIdx.x == 0) total[e] = carry;
}

struct IndexArgs {
    const uint64_t* mask;      // [T][W]
    int T, E, W, cap;
    const int32_t* cnt;        // [chunks][E] selections of each chunk, or in earlier chunks where total is set (null: counted here)
    int chunks;
    const int32_t* total;      // [E] or null
    int32_t* offsets;          // [E+1]
    int32_t* token;            // [cap]
    int32_t* place;            // [T][E]
};

// offsets, token and place of one chunk of tokens per workgroup.  A bit transpose
// costs 100 instructions per 64 tokens: where every workgroup counted all tokens
// itself, 16384 tokens of 64 experts took 15 us, and the two launches take 10.
constexpr int kIndexWaves = 16;
template <int CHUNK>
__global__ __launch_bounds__(kIndexWaves* kWave) void index_kernel(IndexArgs a) {
    constexpr int NW = kIndexWaves, kGroups = CHUNK / kWave;
    // (pairs are counted in unsigned numbers: 2^24 tokens of 256 experts have up to 2^32)
    __shared__ int tot[kMaxExperts], before[kMaxExperts];
    __shared__ uint32_t base[kMaxExperts];
    const uint32_t cap = a.cap;
    __shared__ int own[kGroups][kMaxExperts];
    __shared__ uint64_t cols[kGroups][kMaxExperts];
    const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) / kWave);
    const int t0 = blockIdx.x * CHUNK, blk = blockIdx.x;
    // the chunk's own masks: (group, word) pairs, one per wave
    static_assert(kGroups * kMaxExperts / kWave <= NW, "a pair per wave");
    const int og = wave % kGroups, ow = wave / kGroups, ot = t0 + og * kWave + lane;
    const uint64_t mine = ow < a.W && ot < a.T ? a.mask[static_cast<size_t>(ot) * a.W + ow] : 0ull;
    const int e0 = threadIdx.x % kMaxExperts, part = threadIdx.x / kMaxExperts;
    if (part == 0) {
        const bool given = a.total && e0 < a.E;
        tot[e0] = given ? a.total[e0] : 0;
        before[e0] = given ? a.cnt[static_cast<size_t>(blk) * a.E + e0] : 0;
    }
    __syncthreads();
    if (!a.cnt) {
        constexpr int kPre = 4;
        const int pairs = (a.T + kWave - 1) / kWave * a.W;
        for (int p0 = wave; p0 < pairs; p0 += NW * kPre) {
            uint64_t m[kPre];
#pragma unroll
            for (int i = 0; i < kPre; ++i) {
                const int p = p0 + NW * i, t = p / a.W * kWave + lane;
                m[i] = p < pairs && t < a.T ? a.mask[static_cast<size_t>(t) * a.W + p % a.W] : 0ull;
            }
#pragma unroll
            for (int i = 0; i < kPre; ++i) {
                const int p = p0 + NW * i, e = p % a.W * kWave + lane;
                if (p >= pairs) break;
                const int n = __popcll(bit_transpose(m[i]));
                atomicAdd(&tot[e], n);                     // (whole numbers: any order gives the same sum)
                if (p / a.W * kWave < t0) atomicAdd(&before[e], n);
            }
        }
    } else if (!a.total && e0 < a.E) {
        constexpr int kStep = NW * kWave / kMaxExperts, kPre = 8;
        int all = 0, pre = 0;
        for (int c0 = part; c0 < a.chunks; c0 += kStep * kPre) {
            int n[kPre];
#pragma unroll
            for (int i = 0; i < kPre; ++i) n[i] = c0 + kStep * i < a.chunks ? a.cnt[static_cast<size_t>(c0 + kStep * i) * a.E + e0] : 0;
#pragma unroll
            for (int i = 0; i < kPre; ++i) {
                all += n[i];
                pre += c0 + kStep * i < blk ? n[i] : 0;
            }
        }
        atomicAdd(&tot[e0], all);
        atomicAdd(&before[e0], pre);
    }
    if (ow < a.W) {
        const uint64_t m = bit_transpose(mine);
        cols[og][kWave * ow + lane] = m;
        own[og][kWave * ow + lane] = __popcll(m);
    }
    __syncthreads();
    if (wave == 0) {
        uint32_t carry = 0;
        for (int e1 = 0; e1 < a.E; e1 += kWave) {
            const int e = e1 + lane;
            const int n = e < a.E ? tot[e] : 0;
            const int s = wave_scan(n);                    // (at most 2^30)
            if (e < a.E) {
                base[e] = carry + static_cast<uint32_t>(s - n);
                if (blk == 0) {
                    a.offsets[e] = static_cast<int32_t>(min(base[e], cap));
                    if (e == a.E - 1) a.offsets[a.E] = static_cast<int32_t>(base[e] >= cap ? cap : min(base[e] + static_cast<uint32_t>(n), cap));
                }
            }
            carry += static_cast<uint32_t>(__builtin_amdgcn_readlane(s, kWave - 1));
        }
    }
    __syncthreads();
    // places: the chunk's (group, word) pairs again, in parts of 64 / parts tokens so
    // that every wave has some
    const int share = max(1, NW / (kGroups * a.W)), parts = 1 << (31 - __builtin_clz(share)), len = kWave / parts;
    for (int p = wave; p < kGroups * a.W * parts; p += NW) {
        const int g = p % kGroups, w = p / kGroups % a.W, k0 = p / (kGroups * a.W) * len, e = kWave * w + lane;
        if (e >= a.E) continue;
        uint64_t m = cols[g][e];
        uint32_t row = base[e] + before[e] + __popcll(m & ((1ull << k0) - 1));
        for (int q = 0; q < g; ++q) row += own[q][e];
        m >>= k0;
        const int first = t0 + g * kWave + k0, n = min(len, a.T - first);
        int32_t* to = a.place + static_cast<size_t>(first) * a.E + e;
        for (int k = 0; k < n; ++k, m >>= 1, to += a.E) {
            const bool on = m & 1ull;
            *to = on && row < cap ? static_cast<int32_t>(row) : -1;
            if (on) {
                if (row < cap) a.token[row] = first + k;
                ++row;
            }
        }
    }
}

// Calls of up to kFusedTokens tokens, indices and rows in one launch: a workgroup
// per token works out all segments (build_segments), then its token's places and
// copies (two launches: 18 us for 64 tokens of 4096 elements).
__global__ __launch_bounds__(kThreads) void small_sort_kernel(IndexArgs a, const uint4* __restrict__ x, uint4* __restrict__ rows, int vecs) {
    constexpr int NC = kFusedTokens / kWave;
    __shared__ uint64_t cols[kMaxExperts * NC];
    __shared__ int soff[kMaxExperts + 1];
    __shared__ int list[kMaxExperts], found;
    const int t = blockIdx.x, e = threadIdx.x;
    // (the token's first vectors arrive meanwhile)
    uint4 q{0, 0, 0, 0};
    if (rows && t < a.T && e < vecs) q = x[static_cast<size_t>(t) * vecs + e];
    if (e == 0) found = 0;
    build_segments<kWaves, NC>(a.mask, a.T, a.E, a.W, cols, soff);
    if (t == 0)
        for (int i = e; i <= a.E; i += kThreads) a.offsets[i] = min(soff[i], a.cap);
    if (t >= a.T) return;                                 // (no tokens: one workgroup for the offsets)
    if (e < a.E) {
        const uint64_t* const c = cols + e * NC;
        int row = -1;
        if ((c[t / kWave] >> (t % kWave)) & 1ull) {
            row = soff[e] + __popcll(c[t / kWave] & ((1ull << (t % kWave)) - 1));
            for (int i = 0; i < t / kWave; ++i) row += __popcll(c[i]);
            if (row < a.cap) {
                a.token[row] = t;
                list[atomicAdd(&found, 1)] = row;          // (the order of copies does not matter)
            } else {
                row = -1;
            }
        }
        a.place[static_cast<size_t>(t) * a.E + e] = row;
    }
    if (!rows) return;
    __syncthreads();
    const int n = found;
    for (int v = e; v < vecs; v += kThreads) {
        if (v != e) q = x[static_cast<size_t>(t) * vecs + v];
        for (int i = 0; i < n; ++i) rows[static_cast<size_t>(list[i]) * vecs + v] = q;
    }
}

// ---- rows ------------------------------------------------------------------

struct RowArgs {
    const uint64_t* mask;      // [T][W]
    const int32_t* place;      // [T][E]
    const float* gate;         // [T][E] or null: 1
    int T, E, W, cap;
    int vecs;                  // 16-byte vectors of a row
    int tpb;                   // tokens per workgroup at a time
    const uint4* src;
    uint4* dst;
};

// A token's next up to kBatch selected experts, from word w with bits `rest`
// left: their places (-1: none, or outside the rows) and gates; returns how many
// bits were taken.
struct Cursor {
    int w;
    uint64_t rest;
};
template <bool GATES, bool WHOLE>
__device__ __forceinline__ int next_rows(const RowArgs& a, int t, Cursor& c, int (&rows)[kBatch], float (&gates)[kBatch],
                                         int (&es)[kBatch]) {
    const uint64_t* const m = a.mask + static_cast<size_t>(t) * a.W;
    int n = 0;
#pragma unroll
    for (int b = 0; b < kBatch; ++b) {
        while (c.rest == 0 && c.w + 1 < a.W) {
            c.rest = m[++c.w];
            if (c.w + 1 == a.W && a.E % kWave) c.rest &= ~0ull >> (kWave - a.E % kWave);
        }
        es[b] = 0;
        if (c.rest != 0) {
            es[b] = kWave * c.w + __builtin_ctzll(c.rest);
            c.rest &= c.rest - 1;
            n = b + 1;
        }
    }
    // (without branches, so that these loads are under way together: 16384 tokens x 2048, 8 rows
    // each, sort and its gradient 252 -> 220 us, combine and its gradients 358 -> 336)
    const size_t at = static_cast<size_t>(t) * a.E;
#pragma unroll
    for (int b = 0; b < kBatch; ++b) {
        rows[b] = a.place[at + es[b]];
        gates[b] = GATES ? a.gate[at + es[b]] : 1.f;
    }
#pragma unroll
    for (int b = 0; b < kBatch; ++b)
        if (b >= n || static_cast<unsigned>(rows[b]) >= static_cast<unsigned>(a.cap)) rows[b] = -1;
    if constexpr (WHOLE) {                    // the wave has one token, so its rows are scalars (registers
                                              // of combine_grad_kernel 148 -> 100, 336 -> 330 us; 8192 x 1024, 4 rows: 88 -> 79)
        n = __builtin_amdgcn_readfirstlane(n);
#pragma unroll
        for (int b = 0; b < kBatch; ++b) {
            rows[b] = __builtin_amdgcn_readfirstlane(rows[b]);
            es[b] = __builtin_amdgcn_readfirstlane(es[b]);
            gates[b] = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(gates[b])));
        }
    }
    return n;
}
__device__ __forceinline__ Cursor first_rows(const RowArgs& a, int t) {
    uint64_t m = a.mask[static_cast<size_t>(t) * a.W];
    if (a.W == 1 && a.E % kWave) m &= ~0ull >> (kWave - a.E % kWave);
    return Cursor{0, m};
}

// rows[place] = x[t]: each token's row is read once.  16384 tokens x 2048 to 8 rows each: 604 MB
// in 114 us, 5.3 TB/s.
__global__ __launch_bounds__(kThreads) void spread_kernel(RowArgs a) {
    const int v0 = a.tpb > 1 ? threadIdx.x % a.vecs : threadIdx.x, sub = a.tpb > 1 ? threadIdx.x / a.vecs : 0;
    if (sub >= a.tpb) return;
    for (int64_t t = static_cast<int64_t>(blockIdx.x) * a.tpb + sub; t < a.T; t += static_cast<int64_t>(gridDim.x) * a.tpb) {
        Cursor c = first_rows(a, t);
        for (;;) {
            int rows[kBatch], es[kBatch];
            float gates[kBatch];
            const int n = next_rows<false, false>(a, t, c, rows, gates, es);
            if (n == 0) break;
            for (int v = v0; v < a.vecs; v += kThreads) {
                const uint4 q = a.src[t * a.vecs + v];
#pragma unroll
                for (int b = 0; b < kBatch; ++b)
                    if (rows[b] >= 0) store_row(a.dst + static_cast<int64_t>(rows[b]) * a.vecs + v, q);
            }
            if (n < kBatch) break;
        }
    }
}

// y[t] = sum gate rows[place] (gate null: 1), in fp32 in the experts' order; 8 rows at a
// time in flight per thread.  16384 tokens x 2048 from 8 rows each: 604 MB in 110 us, 5.5 TB/s.
template <typename T, bool GATES>
__global__ __launch_bounds__(kThreads) void gather_kernel(RowArgs a) {
    using V = Vec<T>;
    const int v0 = a.tpb > 1 ? threadIdx.x % a.vecs : threadIdx.x, sub = a.tpb > 1 ? threadIdx.x / a.vecs : 0;
    if (sub >= a.tpb) return;
    for (int64_t t = static_cast<int64_t>(blockIdx.x) * a.tpb + sub; t < a.T; t += static_cast<int64_t>(gridDim.x) * a.tpb) {
        for (int v = v0; v < a.vecs; v += kThreads) {
            float acc[V::N];
#pragma unroll
            for (int i = 0; i < V::N; ++i) acc[i] = 0.f;
            Cursor c = first_rows(a, t);
            for (;;) {
                int rows[kBatch], es[kBatch];
                float gates[kBatch];
                const int n = next_rows<GATES, false>(a, t, c, rows, gates, es);
                if (n == 0) break;
                uint4 q[kBatch];
#pragma unroll
                for (int b = 0; b < kBatch; ++b)
                    if (rows[b] >= 0) q[b] = load_row(a.src + static_cast<int64_t>(rows[b]) * a.vecs + v);
#pragma unroll
                for (int b = 0; b < kBatch; ++b) {
                    if (rows[b] < 0) continue;
                    float f[V::N];
                    V::get(q[b], f);
#pragma unroll
                    for (int i = 0; i < V::N; ++i) acc[i] = GATES ? fmaf(gates[b], f[i], acc[i]) : acc[i] + f[i];
                }
                if (n < kBatch) break;
            }
            a.dst[t * a.vecs + v] = V::put(acc);
        }
    }
}

struct GradArgs {
    RowArgs r;                 // src: dy [T][d], dst: drows (or null)
    const uint4* rows;         // [cap][d] (read where dots)
    bool dots;                 // dg is asked for
    const float* prob;         // [T][E] (dlogits only)
    float eps;
    float* dgate;              // [T][E] or null
    float* dlogits;            // [T][E] or null
};

// One token per NT threads (a wave or the workgroup): its rows in batches, dy
// read again per batch (from L1), the batch's dot products reduced together.
// 16384 tokens x 2048 of 8 rows each: 1.14 GB in 229 us, 5.0 TB/s.
template <typename T, int NT>
__global__ __launch_bounds__(kThreads) void combine_grad_kernel(GradArgs g) {
    using V = Vec<T>;
    constexpr int kSub = kThreads / NT;
    __shared__ float dgs[kSub][kMaxExperts];
    __shared__ float gs[kSub][kMaxExperts];
    __shared__ float red[kBatch][kWaves];
    const RowArgs& a = g.r;
    const int sub = threadIdx.x / NT, id = threadIdx.x % NT, lane = lane_id(), wave = threadIdx.x / kWave;
    auto sync = [&]() __attribute__((always_inline)) {
        if constexpr (NT == kWave) wave_lds_sync();
        else __syncthreads();
    };
    for (int64_t t0 = static_cast<int64_t>(blockIdx.x) * kSub; t0 < a.T; t0 += static_cast<int64_t>(gridDim.x) * kSub) {
        const int64_t t = t0 + sub;
        if (NT == kWave && t >= a.T) break;               // (the wave's own tokens are over)
        for (int e = id; e < a.E; e += NT) { dgs[sub][e] = 0.f; gs[sub][e] = 0.f; }
        sync();
        Cursor c = first_rows(a, t);
        float P = 0.f;
        bool any = false;                                 // the token selected an expert
        for (;;) {
            int rows[kBatch], es[kBatch];
            float gates[kBatch], dot[kBatch];
            const int n = next_rows<true, true>(a, t, c, rows, gates, es);
            if (n == 0) break;
            any = true;
            if (g.dlogits) {
#pragma unroll
                for (int b = 0; b < kBatch; ++b) P += b < n ? g.prob[static_cast<size_t>(t) * a.E + es[b]] : 0.f;
            }
#pragma unroll
            for (int b = 0; b < kBatch; ++b) dot[b] = 0.f;
            for (int v = id; v < a.vecs; v += NT) {
                float dy[V::N];
                V::get(a.src[t * a.vecs + v], dy);
                uint4 q[kBatch];
                if (g.dots) {
#pragma unroll
                    for (int b = 0; b < kBatch; ++b)
                        if (rows[b] >= 0) q[b] = load_row(g.rows + static_cast<int64_t>(rows[b]) * a.vecs + v);
                }
                if (a.dst) {                              // (while the rows are on their way)
#pragma unroll
                    for (int b = 0; b < kBatch; ++b) {
                        if (rows[b] < 0) continue;
                        float o[V::N];
#pragma unroll
                        for (int i = 0; i < V::N; ++i) o[i] = gates[b] * dy[i];
                        store_row(a.dst + static_cast<int64_t>(rows[b]) * a.vecs + v, V::put(o));
                    }
                }
                if (g.dots) {
#pragma unroll
                    for (int b = 0; b < kBatch; ++b) {
                        if (rows[b] < 0) continue;
                        float f[V::N];
                        V::get(q[b], f);
#pragma unroll
                        for (int i = 0; i < V::N; ++i) dot[b] = fmaf(dy[i], f[i], dot[b]);
                    }
                }
            }
            if (g.dots) {
#pragma unroll
                for (int b = 0; b < kBatch; ++b) {
                    dot[b] = wave_sum(dot[b]);
                    if (NT > kWave && lane == 0) red[b][wave] = dot[b];
                }
                if constexpr (NT > kWave) __syncthreads();
                if (id == 0) {
#pragma unroll
                    for (int b = 0; b < kBatch; ++b) {
                        if (b >= n) continue;
                        float s = dot[b];
                        if constexpr (NT > kWave) {
                            s = 0.f;
#pragma unroll
                            for (int q = 0; q < kWaves; ++q) s += red[b][q];
                        }
                        dgs[sub][es[b]] = s;
                        gs[sub][es[b]] = gates[b];
                    }
                }
                sync();
            }
            if (n < kBatch) break;
        }
        if (!g.dots) continue;
        sync();
        float G = 0.f;
        if (g.dlogits) {
            // (every wave of the token adds the same numbers in the same order)
            for (int e = lane; e < a.E; e += kWave) G = fmaf(gs[sub][e], dgs[sub][e], G);
            G = wave_sum(G);
        }
        const float rest = P + g.eps > 0.f ? g.eps / (P + g.eps) : 0.f;
        for (int e = id; e < a.E; e += NT) {
            const size_t at = static_cast<size_t>(t) * a.E + e;
            const float dg = dgs[sub][e];
            if (g.dgate) g.dgate[at] = dg;
            if (g.dlogits) {
                const bool on = (a.mask[static_cast<size_t>(t) * a.W + e / kWave] >> (e % kWave)) & 1ull;
                // (none selected: 0 beside NaN probabilities too, as routing leaves them for rows with NaN)
                const float out = any ? g.prob[at] * G * rest : 0.f;
                g.dlogits[at] = on ? fmaf(gs[sub][e], dg - G, -out) : -out;
            }
        }
        sync();
    }
}

int64_t row_blocks(int64_t units) { return std::max<int64_t>(1, std::min<int64_t>(units, int64_t{1} << 20)); }

template <typename T>
RowArgs row_args(const SortCall& c, const void* src, void* dst) {
    const int vecs = c.d * static_cast<int>(sizeof(T)) / 16;
    return RowArgs{c.mask, c.place, c.gate, c.T, c.E, mask_words(c.E), c.cap, vecs, std::max(1, kThreads / vecs),
                   static_cast<const uint4*>(src), static_cast<uint4*>(dst)};
}

}  // namespace

static int chunks_of(int T) {
    const int chunk = T <= kSmallTokens ? kSmallChunk : kChunk;
    return (T + chunk - 1) / chunk;
}
size_t sort_workspace(int32_t T, int E) {
    if (T <= kFusedTokens) return 0;
    return (static_cast<size_t>(chunks_of(T)) + 1) * E * 4;
}

hipError_t launch_sort(const SortCall& c, const void* x, void* rows, int32_t* offsets, int32_t* token, int32_t* place,
                       void* ws, hipStream_t s) {
    const int W = mask_words(c.E), chunks = chunks_of(c.T);
    const bool small = c.T <= kSmallTokens;
    IndexArgs ia{c.mask, c.T, c.E, W, c.cap, nullptr, chunks, nullptr, offsets, token, place};
    if (c.T <= kFusedTokens) {
        small_sort_kernel<<<std::max(1, c.T), kThreads, 0, s>>>(ia, static_cast<const uint4*>(x), static_cast<uint4*>(rows),
                                                                c.d * (c.bf16 ? 2 : 4) / 16);
        return hipGetLastError();
    }
    int32_t* const cnt = static_cast<int32_t*>(ws);
    hipError_t e = hipSuccess;
    if ((c.T + kWave - 1) / kWave * W > kCountPairs) {
        ia.cnt = cnt;
        if (small) count_kernel<kSmallChunk><<<chunks, kSmallChunk, 0, s>>>(c.mask, c.T, c.E, W, cnt);
        else count_kernel<kChunk><<<chunks, kChunk, 0, s>>>(c.mask, c.T, c.E, W, cnt);
        e = hipGetLastError();
    }
    if (e == hipSuccess && !small && chunks > kSumChunks) {
        int32_t* const total = cnt + static_cast<size_t>(chunks) * c.E;
        ia.total = total;
        scan_kernel<<<c.E, kThreads, 0, s>>>(cnt, chunks, c.E, total);
        e = hipGetLastError();
    }
    if (e != hipSuccess) return e;
    if (small) index_kernel<kSmallChunk><<<chunks, kIndexWaves * kWave, 0, s>>>(ia);
    else index_kernel<kChunk><<<chunks, kIndexWaves * kWave, 0, s>>>(ia);
    e = hipGetLastError();
    if (e != hipSuccess || !rows) return e;
    SortCall p = c;
    p.place = place;
    const RowArgs a = c.bf16 ? row_args<uint16_t>(p, x, rows) : row_args<float>(p, x, rows);
    spread_kernel<<<row_blocks((c.T + a.tpb - 1) / a.tpb), kThreads, 0, s>>>(a);
    return hipGetLastError();
}

hipError_t launch_gather(const SortCall& c, const void* rows, void* y, hipStream_t s) {
    const RowArgs a = c.bf16 ? row_args<uint16_t>(c, rows, y) : row_args<float>(c, rows, y);
    const int64_t blocks = row_blocks((c.T + a.tpb - 1) / a.tpb);
    if (c.bf16) {
        if (c.gate) gather_kernel<uint16_t, true><<<blocks, kThreads, 0, s>>>(a);
        else gather_kernel<uint16_t, false><<<blocks, kThreads, 0, s>>>(a);
    } else {
        if (c.gate) gather_kernel<float, true><<<blocks, kThreads, 0, s>>>(a);
        else gather_kernel<float, false><<<blocks, kThreads, 0, s>>>(a);
    }
    return hipGetLastError();
}

hipError_t launch_combine_grad(const SortCall& c, const void* dy, const void* rows, const float* prob, float eps, void* drows,
                               float* dgate, float* dlogits, hipStream_t s) {
    const RowArgs a = c.bf16 ? row_args<uint16_t>(c, dy, drows) : row_args<float>(c, dy, drows);
    const GradArgs g{a, static_cast<const uint4*>(rows), dgate || dlogits, prob, eps, dgate, dlogits};
    const bool one = a.vecs <= kWave;
    const int64_t blocks = row_blocks(one ? (c.T + kWaves - 1) / kWaves : c.T);
    if (c.bf16) {
        if (one) combine_grad_kernel<uint16_t, kWave><<<blocks, kThreads, 0, s>>>(g);
        else combine_grad_kernel<uint16_t, kThreads><<<blocks, kThreads, 0, s>>>(g);
    } else {
        if (one) combine_grad_kernel<float, kWave><<<blocks, kThreads, 0, s>>>(g);
        else combine_grad_kernel<float, kThreads><<<blocks, kThreads, 0, s>>>(g);
    }
    return hipGetLastError();
}

}  // namespace eat
