// Softmax cross entropy of the LM head with its gradients (gfx950).
//
// With z = h W^T over the n rows that count, y their targets:
//   nll_t  = log(1 + sum_{v != y} exp(z_tv - z_ty)),  loss = c sum_t nll_t
//   G_tv   = exp(z_tv - lse_t) off the target, expm1(-nll_t) on it
//   dh     = c G W,   dW = c G^T h,   c = scale / (mean ? n : 1)
// The z of all the rows is never there.  A first pass leaves one (maximum, sum of
// exponentials) pair per row and 128 or 256 columns, and in 16 bits the exponentials of
// the first piece of the vocabulary, over their tile's maximum: G of that piece
// needs one multiplication per entry.  The gradients take the other pieces' z again,
// a piece at a time, whose G is held in bf16 (kPieceBytes at most) for its two
// products.
//
// list_kernel lists the rows that count, gather_kernel copies them together
// (everything after works on n rows, so ignored ones cost nothing and reach
// nothing) and takes their target's logit in fp64; loss_gemm<LSE> makes the
// pairs, row_kernel the NLLs, the softmax denominators and the loss;
// scale_kernel makes G of the first piece, loss_gemm<GRAD> of the others,
// loss_gemm<PART/ROWS> the products of a piece, and join_kernel adds the slices of
// dh.
//
// G in bf16 is off by up to 2^-8 of each entry, that of the first piece by 2^-10 more
// (the exponential's rounding: pack_kept).  Over many rows such errors average
// out against the rounding of the bf16 results; over few they do not (dW of one row
// is its G times a number), so up to kFewRows rows that count have G in two bf16
// parts, and their hidden rows twice: known on the host in calls of so few, else on
// the device, where the parts are further rows of the products (dh of 200 positions,
// d 4096, V 32000, of which 64 count: 129 us of kernels, 119 in one part).
//
// Bounds, measured: three products of 2 n d V operations each (1.06 - 1.18 PFLOP/s
// at 4096 rows, d 4096, V 32000, where a call takes 2.74 ms, 1.16 - 1.26 at 8192 rows,
// V 128256; a library product reaches 1.1 - 1.4); with few rows the one pass over W (1 row, 262 MB:
// 66 us, 4.0 TB/s), then dW's store (131 M entries from one row: 70 us, 3.7
// TB/s); with small vocabularies the launches, five to seven that wait for each
// other (32 rows, d 128, V 1024: 34.5 us).
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "loss_gemm.h"

namespace eat {
namespace {

// One wave per row.  Row t of the call, where it is ignored: its NLL and its
// dh are zero.  Row i of the list: its hidden row, its target and the target's
// logit in fp64 (the NLL would depend most on that logit's rounding); rows
// behind the list up to whole tiles: zeros.  Of up to kFewRows listed rows all is
// there again, kFewRows rows on.  LIST (calls of up to kListedRows
// rows): every workgroup works the list out for itself, a lane per row, instead of a
// launch before this one (~5 us).
constexpr int kGatherWaves = 4, kListedRows = kGatherWaves * kWave;
template <bool LIST>
__global__ __launch_bounds__(kGatherWaves * kWave) void gather_kernel(
    const uint16_t* __restrict__ h, const uint16_t* __restrict__ w, const int32_t* __restrict__ target, int T, int Tpad,
    int d, int V, int ignore, int32_t* rows, int32_t* head, uint16_t* hc, int32_t* tc, double* zt, float* nll, uint16_t* dh) {
    __shared__ uint64_t keep[kGatherWaves];
    const int lane = lane_id(), i = blockIdx.x * kGatherWaves + __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    int n, t = 0;
    if constexpr (LIST) {
        const int at = threadIdx.x;
        const uint64_t b = ballot(at < T && target[at < T ? at : 0] != ignore);
        if (lane == 0) keep[at / kWave] = b;
        __syncthreads();
        n = 0;
#pragma unroll
        for (int k = 0; k < kGatherWaves; ++k) n += __popcll(keep[k]);
        if (i < n) t = nth_token<kGatherWaves>(keep, i);
        if (i < n && lane == 0) rows[i] = t;
        if (i == 0 && lane == 0) {
            head[0] = n;
            head[1] = (n + kBK - 1) / kBK * kBK;
            head[2] = 0;
        }
    } else {
        n = head[0];
        if (i < n) t = rows[i];
    }
    if (i < T && target[i] == ignore) {
        if (nll && lane == 0) nll[i] = 0.f;
        if (dh)
            for (int k = 8 * lane; k < d; k += 8 * kWave)
                *reinterpret_cast<uint4*>(dh + static_cast<size_t>(i) * d + k) = uint4{};
    }
    const bool again = n <= kFewRows;
    if (i >= Tpad || i >= (n + 255) / 256 * 256 || (again && i >= kFewRows && i < 2 * kFewRows)) return;
    const int y = i < n ? target[t] : 0;
    const bool known = y >= 0 && y < V;
    double z = 0.0;
    constexpr int kLoads = 4;                 // 16-byte pieces of each row a lane has in flight
    for (int k0 = 8 * lane; k0 < d; k0 += 8 * kWave * kLoads) {
        uint4 p[kLoads], q[kLoads];
#pragma unroll
        for (int u = 0; u < kLoads; ++u) {    // (pieces past the row load its first)
            const int k = k0 + 8 * kWave * u < d ? k0 + 8 * kWave * u : k0;
            p[u] = *reinterpret_cast<const uint4*>(h + static_cast<size_t>(t) * d + k);
            q[u] = *reinterpret_cast<const uint4*>(w + static_cast<size_t>(known ? y : 0) * d + k);
        }
#pragma unroll
        for (int u = 0; u < kLoads; ++u) {
            const int k = k0 + 8 * kWave * u;
            if (k >= d) break;
            const uint4 row = i < n ? p[u] : uint4{};
            *reinterpret_cast<uint4*>(hc + static_cast<size_t>(i) * d + k) = row;
            if (again && i < kFewRows) *reinterpret_cast<uint4*>(hc + static_cast<size_t>(i + kFewRows) * d + k) = row;
            const uint32_t pw[4] = {p[u].x, p[u].y, p[u].z, p[u].w}, qw[4] = {q[u].x, q[u].y, q[u].z, q[u].w};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                z = fma(static_cast<double>(__uint_as_float(pw[e] << 16)), static_cast<double>(__uint_as_float(qw[e] << 16)), z);
                z = fma(static_cast<double>(__uint_as_float(pw[e] & 0xffff0000u)),
                        static_cast<double>(__uint_as_float(qw[e] & 0xffff0000u)), z);
            }
        }
    }
    z = wave_sum(z);
    if (lane == 0 && i < n) {
        tc[i] = known ? y : -1;
        zt[i] = z;
    }
}

// The row's (maximum, sum) over the column tiles, a lane per row and a wave
// per share of the tiles; then its NLL, its softmax denominator and G at its
// target.  The last workgroup to finish adds up the loss, in row order.
constexpr int kRowWaves = 16, kRowLoads = 8;
__global__ __launch_bounds__(kRowWaves * kWave) void row_kernel(const float2* __restrict__ part, int ntiles, int ldpart,
                                                                int32_t* head, const int32_t* __restrict__ rows,
                                                                const int32_t* __restrict__ tc,
                                                                const double* __restrict__ zt, float scale, int mean,
                                                                float2* stats, double* nllc, float* nll, float* loss,
                                                                float* coef, int32_t* count) {
    __shared__ float2 red[kRowWaves][kWave];
    __shared__ double sums[kRowWaves];
    __shared__ int last;
    const int lane = lane_id(), wave = threadIdx.x / kWave;
    const int n = head[0], blocks = max(1, (n + kWave - 1) / kWave);
    if (static_cast<int>(blockIdx.x) >= blocks) return;
    const int i = blockIdx.x * kWave + lane, is = max(0, min(i, n - 1));
    float m = -INFINITY, s = 0.f;
    auto merge = [&](float2 p) __attribute__((always_inline)) {
        const float hi = fmaxf(m, p.x);
        s = (m == hi ? s : s * __expf(m - hi)) + (p.x == hi ? p.y : p.y * __expf(p.x - hi));
        m = hi;
    };
    // (loads of a row and a tile that exist, all issued before the first use)
    const double z = wave == 0 && n > 0 ? zt[is] : 0.0;
    const int y = wave == 0 && n > 0 ? tc[is] : 0;
    if (n > 0)
        for (int t0 = wave; t0 < ntiles; t0 += kRowLoads * kRowWaves) {
            float2 p[kRowLoads];
#pragma unroll
            for (int u = 0; u < kRowLoads; ++u)
                p[u] = part[static_cast<size_t>(min(t0 + u * kRowWaves, ntiles - 1)) * ldpart + is];
#pragma unroll
            for (int u = 0; u < kRowLoads; ++u)
                if (t0 + u * kRowWaves < ntiles) merge(p[u]);
        }
    red[wave][lane] = float2{m, s};
    __syncthreads();
    double v = 0.0;
    if (wave == 0 && i < n) {
#pragma unroll
        for (int w = 1; w < kRowWaves; ++w) merge(red[w][lane]);
        // (z - z is NaN for an infinite target, as its row's logsumexp less itself)
        const double md = m, rest = s;
        double lse;
        if (z >= md) {
            v = log1p(rest * exp(md - z)) + (z - z);
            lse = z + v;
        } else {
            lse = md + log(rest + exp(z - md));
            v = lse - z;
        }
        if (y < 0) v = lse = NAN;
        stats[i] = float2{static_cast<float>(lse), static_cast<float>(expm1(-v))};
        if (nll) nll[rows[i]] = static_cast<float>(v);
        if (blocks > 1) __hip_atomic_store(nllc + i, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    double a = v;
    if (blocks > 1) {
        if (threadIdx.x == 0)
            last = __hip_atomic_fetch_add(head + 2, 1, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) == blocks - 1;
        __syncthreads();
        if (!last) return;
        a = 0.0;
        for (int r = threadIdx.x; r < n; r += kRowWaves * kWave)
            a += __hip_atomic_load(nllc + r, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    a = wave_sum(a);
    if (lane == 0) sums[wave] = a;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < kRowWaves; ++w) a += sums[w];
        const double c = static_cast<double>(scale) / (mean ? max(n, 1) : 1);
        *loss = static_cast<float>(a * c);
        *coef = static_cast<float>(c);
        if (count) *count = n;
    }
}

// G of the columns whose exponentials the first pass kept, in place (NaN in a row
// and tile with a logit of +inf, whose exponentials are not below 1): a tile of
// the first pass x 64 rows per workgroup, 16 bytes per lane.  Twice the piece's
// bytes against taking its product again (4096 rows of 32000 columns, d 4096:
// see launch_ce).  Rows behind the list up to a whole reduction chunk: zeros.  Up
// to kFewRows rows: in two bf16 parts (the second kFewRows rows on).
constexpr int kScaleThreads = 256, kScaleRows = 64;
template <int NA>
__global__ __launch_bounds__(kScaleThreads) void scale_kernel(const float2* __restrict__ part, int ldpart,
                                                              const float2* __restrict__ stats,
                                                              const int32_t* __restrict__ tc,
                                                              const int32_t* __restrict__ head, uint16_t* g, int64_t ldg) {
    constexpr int V = NA / 8, R = kScaleThreads / V;       // lanes per row, rows at a time
    __shared__ float4 row[kScaleRows];                     // factor, G at the target, target's column (bits)
    const int n = head[0], pad = head[1];
    const int r0 = blockIdx.y * kScaleRows, c0 = blockIdx.x * NA;
    if (r0 >= pad) return;
    const int tid = threadIdx.x;
    if (tid < kScaleRows) {
        const int i = r0 + tid;
        float4 v{0.f, 0.f, __int_as_float(-1), 0.f};
        if (i < n) {
            const float2 st = stats[i];
            const float m = part[static_cast<size_t>(blockIdx.x) * ldpart + i].x;
            v = float4{m == INFINITY ? NAN : m == -INFINITY ? 0.f * st.x : exp_from(tile_ref(m), st.x), st.y,
                       __int_as_float(tc[i] - c0), 0.f};
        }
        row[tid] = v;
    }
    uint16_t* const at = g + (r0 + tid / V) * ldg + c0 + 8 * (tid % V);
    constexpr int K = kScaleRows / R;
    auto scale = [&](auto two) __attribute__((always_inline)) {
        constexpr bool PARTS = decltype(two)::value;
        constexpr int N = PARTS ? K / 2 : K;               // loads of a plane in flight
        uint4 v[N], v2[PARTS ? N : 1];
#pragma unroll
        for (int k0 = 0; k0 < K; k0 += N) {
#pragma unroll
            for (int k = 0; k < N; ++k) {
                v[k] = *reinterpret_cast<const uint4*>(at + (k0 + k) * R * ldg);
                if constexpr (PARTS) v2[k] = *reinterpret_cast<const uint4*>(at + (kFewRows + (k0 + k) * R) * ldg);
            }
            if (k0 == 0) __syncthreads();
#pragma unroll
            for (int k = 0; k < N; ++k) {
                const int r = tid / V + (k0 + k) * R;
                const float4 p = row[r];
                const int rel = __float_as_int(p.z) - 8 * (tid % V);
                const uint32_t w[4] = {v[k].x, v[k].y, v[k].z, v[k].w};
                uint32_t w2[4] = {}, o[4], o2[4];
                if constexpr (PARTS) { w2[0] = v2[k].x; w2[1] = v2[k].y; w2[2] = v2[k].z; w2[3] = v2[k].w; }
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float lo, hi;
                    if constexpr (PARTS) {
                        lo = __uint_as_float(w[e] << 16) + __uint_as_float(w2[e] << 16);
                        hi = __uint_as_float(w[e] & 0xffff0000u) + __uint_as_float(w2[e] & 0xffff0000u);
                    } else {
                        lo = kept_lo(w[e]);
                        hi = kept_hi(w[e]);
                    }
                    lo = rel == 2 * e ? p.y : lo * p.x;
                    hi = rel == 2 * e + 1 ? p.y : hi * p.x;
                    if (r0 + r >= n) lo = hi = 0.f;
                    o[e] = pack_bf16x2(lo, hi);
                    if constexpr (PARTS) o2[e] = pack_bf16x2(bf16_rest(lo), bf16_rest(hi));
                }
                uint16_t* const to = at + (k0 + k) * R * ldg;
                *reinterpret_cast<uint4*>(to) = uint4{o[0], o[1], o[2], o[3]};
                if constexpr (PARTS) *reinterpret_cast<uint4*>(to + kFewRows * ldg) = uint4{o2[0], o2[1], o2[2], o2[3]};
            }
        }
    };
    static_assert(kScaleRows == kFewRows, "one workgroup has all rows of both parts");
    if (n <= kFewRows) scale(std::true_type{});
    else scale(std::false_type{});
}

// dh of the listed rows: its slices (head[3] of them) added in order, times c.
// planes: up to kFewRows rows come in two parts, the second kFewRows rows on.
constexpr int kJoinThreads = 256;
__global__ __launch_bounds__(kJoinThreads) void join_kernel(const float* __restrict__ part, int tile_rows, int direct, int planes,
                                                            const int32_t* __restrict__ head,
                                                            const int32_t* __restrict__ rows, int d,
                                                            const float* __restrict__ coef, uint16_t* dh) {
    const int n = head[0], splits = head[3];
    const bool two = planes && n <= kFewRows;
    if (splits == 1 && direct && !two) return;             // (written as it was finished)
    const int64_t stride = static_cast<int64_t>(((two ? with_parts(n) : n) + tile_rows - 1) / tile_rows) * tile_rows * d;
    const float c = *coef;
    const int64_t total = static_cast<int64_t>(n) * (d / 8);
    for (int64_t at = blockIdx.x * int64_t(kJoinThreads) + threadIdx.x; at < total; at += int64_t(gridDim.x) * kJoinThreads) {
        const int i = static_cast<int>(at / (d / 8)), k = static_cast<int>(at % (d / 8)) * 8;
        const float* p = part + static_cast<size_t>(i) * d + k;
        f32x4 lo = *reinterpret_cast<const f32x4*>(p), hi = *reinterpret_cast<const f32x4*>(p + 4);
        for (int s = 1; s < splits; ++s) {
            lo += *reinterpret_cast<const f32x4*>(p + s * stride);
            hi += *reinterpret_cast<const f32x4*>(p + s * stride + 4);
        }
        if (two) {
            p += static_cast<size_t>(kFewRows) * d;
            for (int s = 0; s < splits; ++s) {
                lo += *reinterpret_cast<const f32x4*>(p + s * stride);
                hi += *reinterpret_cast<const f32x4*>(p + s * stride + 4);
            }
        }
        *reinterpret_cast<uint4*>(dh + static_cast<size_t>(rows[i]) * d + k) =
            uint4{pack_bf16x2(lo[0] * c, lo[1] * c), pack_bf16x2(lo[2] * c, lo[3] * c),
                  pack_bf16x2(hi[0] * c, hi[1] * c), pack_bf16x2(hi[2] * c, hi[3] * c)};
    }
}

// The tile of a product of `rows` x `cols` outputs with one reduction slice:
// Small up to its 64 rows (the operand of `cols` streams past), else the larger
// one of Big and Mid whose rounds over the CUs take less time.  (A chunk costs a
// Big workgroup kBigNs, a Mid one kMidNs.  The loss of 32000 x 4096, Mid | Big:
// 128 rows 62 | 108 us, 200 92 | 105, 300 124 | 114, 512 161 | 125; of 50000 x 2048:
// 128 53 | 58, 200 87 | 61; of 8000 x 1024: 768 38 | 42, 2048 59 | 50.)
enum Size { kSmall, kMid, kBig };
int64_t tiles_of(int64_t rows, int64_t cols, int nb, int na) { return ((rows + nb - 1) / nb) * ((cols + na - 1) / na); }
Size pick_tile(int64_t rows, int64_t cols) {
    if (rows <= Small::NB) return kSmall;
    const int64_t big = (tiles_of(rows, cols, Big::NB, Big::NA) + kCus - 1) / kCus * kBigNs;
    const int64_t mid = (tiles_of(rows, cols, Mid::NB, Mid::NA) + kCus - 1) / kCus * kMidNs;
    return mid < big ? kMid : kBig;
}
constexpr int tile_cols(Size z) { return z == kBig ? Big::NA : Mid::NA; }
static_assert(Mid::NA == Small::NA, "column tiles of 128 or 256");

// dh, whose reduction of `chunks` is split over what CUs its tiles leave: Mid up
// to its two tiles of rows, and while Big has few rounds over the CUs.  (kSmall: Mid
// on G's two planes.  Mid | Big: 50000 x 2048, 128 rows 55 | 92 us, 256 81 | 95, 512
// 144 | 140; 32000 x 4096, 256 100 | 102, 300 154 | 135; 8000 x 1024 in 8 rounds of
// 1024 rows 38 | 45, in 16 of 2048 62 | 64.)
Size dh_tile(int64_t rows, int64_t d, int64_t chunks) {
    if (rows <= Small::NB) return kSmall;
    return rows <= 2 * Mid::NB || tiles_of(rows, d, Big::NB, Big::NA) * chunks <= 8 * kCus ? kMid : kBig;
}

template <bool ACOLS, bool BCOLS, int OUT>
hipError_t launch_sized(Size z, const GemmArgs& g, hipStream_t s) {
    if (z == kBig) return launch_gemm<Big, ACOLS, BCOLS, OUT>(g, s);
    if (z == kMid) return launch_gemm<Mid, ACOLS, BCOLS, OUT>(g, s);
    if constexpr (BCOLS) return launch_gemm<Mid, ACOLS, BCOLS, OUT>(g, s);      // (few entries, not few rows)
    else return launch_gemm<Small, ACOLS, BCOLS, OUT>(g, s);
}

// G held at a time: a piece of the vocabulary whose G takes kPieceBytes at
// most (1.4% of the card's memory) and, with a smaller workspace, what fits,
// from kMinPiece columns on (which take more than kPieceBytes beyond 2^19 rows, 8
// GiB at the most).  The first piece costs a pass over its G, every
// other one its product again: 8192 rows, d 4096, V 128256 (2.1 GB) take 22.0 ms in
// one piece, 25.0 in two, 26.6 in four, 29.0 in 32; 512 rows, d 2048, V 50000 take 396
// us in one, 478 in two, 1108 in 13 (the smallest, too few columns to fill the CUs).
constexpr size_t kPieceBytes = size_t{4} << 30;
constexpr int kMinPiece = 4096, kMaxPiece = 1 << 22;       // (a row of G is addressed with 24 bits)

}  // namespace

CePlan plan_ce(int32_t T, int32_t d, int32_t V, bool dh, bool dw, size_t bytes) {
    CePlan p{};
    p.rows_pad = T <= Small::NB ? Small::NB : (T + Big::NB - 1) / Big::NB * Big::NB;
    const size_t tp = p.rows_pad, planes = T <= Small::NB ? 2 : 1;
    p.tile = tile_cols(pick_tile(T, V));
    p.tiles = (V + p.tile - 1) / p.tile;
    const int vpad = (V + 255) / 256 * 256;
    const int least = std::min(vpad, kMinPiece);
    auto fit = [&](size_t room) {
        return static_cast<int>(
            std::max<size_t>(least, std::min<size_t>({size_t(vpad), size_t(kMaxPiece), room / (2 * tp * planes) / 256 * 256})));
    };
    // dh: room for its slices, a few of many rows (how many there are is chosen on
    // the device, by the rows that count)
    const size_t pool = dh ? std::max<size_t>(tp, std::min<size_t>(16 * tp, 16384)) : 0;
    p.pool_rows = static_cast<int>(pool);
    auto layout = [&](int piece) {
        size_t off = 0;
        auto take = [&](size_t n) { const size_t at = off; off += (n + 255) & ~size_t(255); return at; };
        p.piece = piece;
        p.head = take(16);
        p.coef = take(4);
        p.rows = take(tp * 4);
        p.tc = take(tp * 4);
        p.zt = take(tp * 8);
        p.nllc = take(tp * 8);
        p.stats = take(tp * 8);
        p.hc = take(tp * planes * d * 2);
        p.part = take(tp * p.tiles * 8);
        p.dhp = take(pool * d * 4);
        p.g = off;
        p.total = off + (dh || dw ? tp * planes * piece * 2 : 0);
    };
    layout(fit(kPieceBytes));
    if (p.total <= bytes || (!dh && !dw)) return p;
    layout(least);
    if (bytes > p.total) layout(fit(bytes - p.g));
    return p;
}

hipError_t launch_ce(const CePlan& p, const CeCall& c, char* ws, hipStream_t s) {
    int32_t* const head = reinterpret_cast<int32_t*>(ws + p.head);
    float* const coef = reinterpret_cast<float*>(ws + p.coef);
    int32_t* const rows = reinterpret_cast<int32_t*>(ws + p.rows);
    int32_t* const tc = reinterpret_cast<int32_t*>(ws + p.tc);
    double* const zt = reinterpret_cast<double*>(ws + p.zt);
    double* const nllc = reinterpret_cast<double*>(ws + p.nllc);
    float2* const stats = reinterpret_cast<float2*>(ws + p.stats);
    uint16_t* const hc = reinterpret_cast<uint16_t*>(ws + p.hc);
    float2* const part = reinterpret_cast<float2*>(ws + p.part);
    uint16_t* const gbuf = reinterpret_cast<uint16_t*>(ws + p.g);
    float* const dhp = reinterpret_cast<float*>(ws + p.dhp);
    const int T = c.T, d = c.d, V = c.V;
    const Size zz = pick_tile(T, V), zh = dh_tile(T, d, (std::min(p.piece, V) + kBK - 1) / kBK);
    static_assert(Small::NB == kFewRows, "calls of few rows have one tile of them");
    const int planes = zz == kSmall ? 0 : 1;               // (kSmall: both parts are tiles of their own or folded)

    const int rb = (p.rows_pad + kGatherWaves - 1) / kGatherWaves;
    if (T <= kListedRows) {
        gather_kernel<true><<<rb, kGatherWaves * kWave, 0, s>>>(c.h, c.w, c.target, T, p.rows_pad, d, V, c.ignore, rows,
                                                                head, hc, tc, zt, c.nll, c.dh);
    } else {
        list_kernel<int32_t><<<1, kListThreads, 0, s>>>(c.target, T, c.ignore, rows, head);
        gather_kernel<false><<<rb, kGatherWaves * kWave, 0, s>>>(c.h, c.w, c.target, T, p.rows_pad, d, V, c.ignore, rows,
                                                                 head, hc, tc, zt, c.nll, c.dh);
    }
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    GemmArgs z{};
    z.a = c.w; z.lda = d; z.na = V;
    z.b = hc; z.ldb = d; z.nb = T; z.nb_dev = head;
    z.K = d; z.splits = 1;
    z.part = part; z.ldpart = p.rows_pad; z.target = tc;
    z.out = gbuf; z.ldo = p.piece; z.kept = c.dh || c.dw ? p.piece : 0;
    e = launch_sized<false, false, LSE>(zz, z, s);
    if (e != hipSuccess) return e;
    row_kernel<<<std::max(1, (T + kWave - 1) / kWave), kRowWaves * kWave, 0, s>>>(part, p.tiles, p.rows_pad, head, rows, tc, zt, c.scale,
                                                                    c.mean, stats, nllc, c.nll, c.loss, coef, c.count);
    e = hipGetLastError();
    if (!c.dh && !c.dw) return e;
    for (int v0 = 0; v0 < V && e == hipSuccess; v0 += p.piece) {
        const int nv = std::min(p.piece, V - v0);
        const uint16_t* w = c.w + static_cast<size_t>(v0) * d;
        if (v0 == 0) {
            const dim3 grid((nv + p.tile - 1) / p.tile, p.rows_pad / kScaleRows);
            if (zz == kBig) scale_kernel<Big::NA><<<grid, kScaleThreads, 0, s>>>(part, p.rows_pad, stats, tc, head, gbuf, p.piece);
            else scale_kernel<Mid::NA><<<grid, kScaleThreads, 0, s>>>(part, p.rows_pad, stats, tc, head, gbuf, p.piece);
            e = hipGetLastError();
        } else {
            GemmArgs q = z;
            q.a = w; q.na = nv; q.col0 = v0;
            q.stats = stats;
            e = launch_sized<false, false, GRAD>(zz, q, s);
        }
        if (e == hipSuccess && c.dh) {
            GemmArgs a{};
            a.a = w; a.lda = d; a.na = d; a.a_rows = nv;
            a.b = gbuf; a.ldb = p.piece; a.nb = planes ? std::max(T, 2 * kFewRows) : T; a.nb_dev = head;
            a.planes = planes; a.K = nv; a.splits = 0;
            a.pool_rows = p.pool_rows; a.slice_chunks = std::min(p.piece, V + kBK - 1) / kBK; a.slices_out = head + 3;
            a.direct = p.piece < V ? nullptr : c.dh;
            a.out = dhp; a.ldo = d; a.add = v0 > 0; a.rows = rows; a.coef = coef;
            e = zh == kBig   ? launch_gemm<Big, true, false, PART>(a, s)
                : zh == kMid ? launch_gemm<Mid, true, false, PART>(a, s)
                             : launch_gemm<Mid, true, false, PART, PLANES>(a, s);
        }
        if (e == hipSuccess && c.dw) {
            GemmArgs a{};
            a.a = hc; a.lda = d; a.na = d; a.a_rows = 1 << 30;
            a.b = gbuf; a.ldb = p.piece; a.nb = nv;
            a.k_times = zz == kSmall ? 2 : 1;              // (both planes of G, over both copies of h)
            a.K = p.rows_pad * a.k_times; a.k_dev = head + 1; a.splits = 1; a.planes = planes;
            a.out = c.dw + static_cast<size_t>(v0) * d; a.ldo = d; a.coef = coef;
            e = launch_sized<true, true, ROWS>(pick_tile(nv, d), a, s);
        }
    }
    if (e == hipSuccess && c.dh) {
        const int64_t n8 = static_cast<int64_t>(T) * (d / 8);
        if (n8 > 0)
            join_kernel<<<static_cast<int>(std::min<int64_t>((n8 + kJoinThreads - 1) / kJoinThreads, 2048)), kJoinThreads, 0, s>>>(
                dhp, zh == kSmall ? Small::NB : zh == kMid ? Mid::NB : Big::NB, p.piece < V ? 0 : 1, planes, head, rows, d, coef, c.dh);
        e = hipGetLastError();
    }
    return e;
}

}  // namespace eat
