// Softmax cross entropy of the LM head with its gradients (gfx950).
//
// With z = h W^T over the n rows that count, y their targets:
//   nll_t  = log(1 + sum_{v != y} exp(z_tv - z_ty)),  loss = c sum_t nll_t
//   G_tv   = exp(z_tv - lse_t) off the target, expm1(-nll_t) on it
//   dh     = c G W,   dW = c G^T h,   c = scale / (mean ? n : 1)
// No row of z is kept: a first pass leaves one (maximum, sum of exponentials)
// pair per row and 256 columns, and the gradients take z again, a piece of the
// vocabulary at a time, whose G is held in bf16 (kPieceBytes at most) for its
// two products.
//
// compact_kernel lists the rows that count, gather_kernel copies them together
// (everything after works on n rows, so ignored ones cost nothing and reach
// nothing) and takes their target's logit in fp64; ce_gemm<LSE> makes the
// pairs, row_kernel the NLLs, the softmax denominators and the loss;
// per piece ce_gemm<GRAD> makes G, ce_gemm<PART/ROWS> its products, and
// join_kernel adds the slices of dh.
//
// ce_gemm: C[b][a] = sum_k A[a][k] B[b][k], bf16 operands, fp32 accumulation
// on v_mfma_f32_32x32x16_bf16 (a lane ends with 4 consecutive columns a of one
// row b).  Either operand may be stored with its reduction index as the row
// ("columns": W for dh, G and h for dW): its LDS tile is then [k][index], and
// the fragments come out of transposing LDS reads (ds_read_b64_tr_b16: the 16
// lanes of a group read a 4 x 16 block, 4 lanes a row, and each gets a column of
// it), so no operand is transposed in memory.
#include <math.h>

#include <algorithm>

#include "eat_device.h"
#include "eat_internal.h"

namespace eat {
namespace {

constexpr int kBK = 64;                   // reduction chunk (bf16 elements)
constexpr float kLog2e = 1.44269504088896340736f;

typedef short s16x4 __attribute__((ext_vector_type(4)));

// NA x NB outputs per workgroup, WA x WB waves over them, a ring of STAGES
// chunks in LDS.
template <int NA_, int NB_, int WA_, int WB_, int STAGES_>
struct Tile {
    static constexpr int NA = NA_, NB = NB_, WA = WA_, WB = WB_, STAGES = STAGES_;
    static constexpr int kWaves = WA * WB;
    static constexpr int kThreads = kWaves * kWave;
    static constexpr int FA = NA / (32 * WA), FB = NB / (32 * WB);    // 32-wide fragments per wave
    static constexpr int kA = NA * kBK * 2, kB = NB * kBK * 2;        // bytes of a stage's operands
    static constexpr int kStage = kA + kB;
    static constexpr int kLA = kA / 1024 / kWaves, kLB = kB / 1024 / kWaves;   // 1 KB loads per wave
    static constexpr int kLoads = kLA + kLB;
    static constexpr int kP = STAGES - 1;     // chunks in flight ahead of the one computed
    static_assert(kLA * 1024 * kWaves == kA && kLB * 1024 * kWaves == kB, "loads split evenly over the waves");
    static_assert(FA * 32 * WA == NA && FB * 32 * WB == NB, "fragments cover the tile");
    static_assert(kP >= 1 && kP <= 3, "wait counts cover up to three chunks in flight");
};
using Big = Tile<256, 256, 4, 2, 2>;
using Small = Tile<128, 64, 4, 2, 4>;

enum Out { LSE, GRAD, PART, ROWS };

struct GemmArgs {
    const uint16_t* a;
    const uint16_t* b;
    int lda, ldb;              // elements between stored rows
    int na, nb, K;             // output columns and rows, reduction length (nb, K: upper bounds where *_dev is set)
    const int32_t* nb_dev;     // rows of the output, on the device (or null)
    const int32_t* k_dev;      // reduction length, on the device (or null)
    int a_rows;                // stored rows of a "columns" A operand (later ones read the last)
    int splits;                // slices of the reduction (PART)
    int col0;                  // LSE, GRAD: vocabulary index of column 0
    int xcds;
    void* out;                 // GRAD, ROWS, LSE: bf16; PART: fp32 slices
    int64_t ldo, split_stride;
    int kept;                  // LSE: columns below it leave exp(z - the tile's maximum) in out
    const int32_t* rows;       // ROWS: destination of each output row (or null: itself)
    const float* coef;         // ROWS: factor c
    int add;                   // PART: add to what the slices hold
    float2* part;              // LSE: [column tile][ldpart] (maximum, sum) pairs
    int ldpart;
    const int32_t* target;     // LSE, GRAD: column that is the row's target
    const float2* stats;       // GRAD: (lse log2 e, G at the target) of a row
};

// Operands stored row by row: LDS rows of 128 bytes (64 k), 16-byte slots XORed
// with the row's 256-byte line, so that an MFMA operand read of 16 rows covers
// every bank.
__device__ __forceinline__ int swz_row(int r) { return (static_cast<unsigned>(r) >> 1) & 7; }
// Operands stored by columns: LDS rows of N indices for each of the 64 k.  A
// transposing read takes 64 bytes of each of 4 consecutive k: XORing the slot
// with 4 (k % 4) puts them on different banks.
__device__ __forceinline__ int swz_col(int k) { return (k & 3) << 2; }

// Loads of one operand's part of a chunk: where lane l of load j gets the 16
// bytes that belong at LDS byte 1024 (wave + kWaves j) + 16 l.
template <int N, int L, int WAVES, bool COLS>
struct Operand {
    const char* base;          // uniform: the item's first chunk
    uint32_t ldbytes;
    uint32_t off[L];           // rows: byte offset; columns: that of the index
    int k_last;                // columns: last stored row, from the item's first chunk (for the clamp)

    // first: the tile's first index, count: indices there are (>= 1), k0: the
    // slice's first k, k_rows: stored rows of a columns operand
    __device__ __forceinline__ void set(const uint16_t* p, int ld, int first, int count, int k0, int k_rows) {
        const int lane = lane_id(), wave = threadIdx.x / kWave;
        ldbytes = static_cast<uint32_t>(ld) * 2;
        if constexpr (COLS) {
            base = reinterpret_cast<const char*>(p) + static_cast<size_t>(k0) * ldbytes;
            k_last = k_rows - 1 - k0;
            constexpr int VPR = N / 8;         // 16-byte slots per LDS row
#pragma unroll
            for (int j = 0; j < L; ++j) {
                const int g = (wave + WAVES * j) * 64 + lane;
                const int k = g / VPR, v = (g % VPR) ^ swz_col(k);
                off[j] = static_cast<uint32_t>(min(first + 8 * v, count - 8)) * 2;
            }
        } else {
            base = reinterpret_cast<const char*>(p) + static_cast<size_t>(first) * ldbytes + 2 * static_cast<size_t>(k0);
            k_last = 0;
#pragma unroll
            for (int j = 0; j < L; ++j) {
                const int r = (wave + WAVES * j) * 8 + lane / 8, v = (lane & 7) ^ swz_row(r);
                off[j] = static_cast<uint32_t>(min(r, count - 1 - first)) * ldbytes + 16 * v;
            }
        }
    }
    // chunk c into LDS at `st` (a load is waited for by count: the compiler
    // adds no waits of its own for asm)
    __device__ __forceinline__ void issue(uint8_t* st, int c) const {
        const int lane = lane_id(), wave = threadIdx.x / kWave;
        const char* src = base + (COLS ? static_cast<size_t>(c) * kBK * ldbytes : static_cast<size_t>(c) * kBK * 2);
#pragma unroll
        for (int j = 0; j < L; ++j) {
            uint32_t o = off[j];
            if constexpr (COLS) {
                const int k = ((wave + WAVES * j) * 64 + lane) / (N / 8);
                o += static_cast<uint32_t>(min(k, k_last - c * kBK)) * ldbytes;
            }
            const uint32_t lds = __builtin_amdgcn_readfirstlane(
                static_cast<uint32_t>(reinterpret_cast<uintptr_t>(st + 1024 * (wave + WAVES * j))));
            asm volatile("s_mov_b32 m0, %2\n\tglobal_load_lds_dwordx4 %0, %1"
                         :: "v"(o), "s"(src), "s"(lds) : "memory", "m0");
        }
    }
};

// The operand fragment of indices i0 .. i0 + 31 and reduction elements 16 s ..
// 16 s + 15 of a stage: lane l holds index i0 + l % 32, elements 8 (l / 32) ..
// + 7.
template <int N, bool COLS>
__device__ __forceinline__ bf16x8 fragment(const uint8_t* st, int i0, int s) {
    const int lane = lane_id();
    if constexpr (COLS) {
        const int g = lane >> 4, j = lane & 15;
        const int k = 16 * s + 8 * (g >> 1) + (j >> 2);
        const int slot = ((i0 >> 3) + 2 * (g & 1) + ((j & 3) >> 1)) ^ ((j >> 2) << 2);
        const uint8_t* p = st + k * (2 * N) + 16 * slot + 8 * (j & 1);
        typedef __attribute__((address_space(3))) s16x4* lds_t;
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_t)(p));
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_t)(p + 4 * (2 * N)));
        typedef short s16x8 __attribute__((ext_vector_type(8)));
        return __builtin_bit_cast(bf16x8, (s16x8)__builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    } else {
        const int r = i0 + (lane & 31);
        return *reinterpret_cast<const bf16x8*>(st + r * 128 + (((2 * s + (lane >> 5)) ^ swz_row(r)) << 4));
    }
}

struct Item {
    int a0, b0, sp;
};

// The reference of a row's exponentials over a tile with maximum m (infinite
// where all are -inf, whose sum is 0, or some +inf: then 0).
__device__ __forceinline__ float tile_ref(float m) { return fabsf(m) == INFINITY ? 0.f : m; }

__device__ __forceinline__ float swap_halves(float v) { return __shfl_xor(v, 32, kWave); }

template <class C, bool ACOLS, bool BCOLS, int OUT>
__global__ __launch_bounds__(C::kThreads) void ce_gemm(GemmArgs g) {
    constexpr int FA = C::FA, FB = C::FB;
    __shared__ __attribute__((aligned(1024))) uint8_t ring[C::STAGES * C::kStage];
    const int nb = g.nb_dev ? min(*g.nb_dev, g.nb) : g.nb;
    const int K = g.k_dev ? min(*g.k_dev, g.K) : g.K;
    const int nta = (g.na + C::NA - 1) / C::NA, ntb = (nb + C::NB - 1) / C::NB;
    const int splits = OUT == PART ? g.splits : 1;
    const int chunks = (K + kBK - 1) / kBK;
    const int work = nta * ntb * splits;
    // contiguous parts of the work list per XCD (workgroups are dealt to XCDs
    // round-robin), in it groups of 8 row tiles, column tile by column tile:
    // the workgroups of an XCD that run together share both operands in its L2
    const int xcd = blockIdx.x % g.xcds, slot = blockIdx.x / g.xcds, per_xcd = gridDim.x / g.xcds;
    const int part = (work + g.xcds - 1) / g.xcds;
    const int wbeg = xcd * part, wend = min(work, wbeg + part);
    auto item_at = [&](int wid) __attribute__((always_inline)) {
        const int sp = wid / (nta * ntb);
        int r = wid - sp * nta * ntb;
        const int grp = r / (8 * nta);
        const int gb = min(8, ntb - 8 * grp);
        r -= grp * 8 * nta;
        Item it;
        it.sp = __builtin_amdgcn_readfirstlane(sp);
        it.a0 = __builtin_amdgcn_readfirstlane(r / gb * C::NA);
        it.b0 = __builtin_amdgcn_readfirstlane((8 * grp + r % gb) * C::NB);
        return it;
    };
    int wid = wbeg + slot;
    if (wid >= wend) return;                  // uniform over the workgroup

    const int lane = lane_id(), wave = threadIdx.x / kWave;
    const int l32 = lane & 31, lh = lane >> 5;
    const int arow = 32 * FA * (wave % C::WA), brow = 32 * FB * (wave / C::WA);
    const float coef = OUT == ROWS ? *g.coef : 1.f;

    Operand<C::NA, C::kLA, C::kWaves, ACOLS> oa;
    Operand<C::NB, C::kLB, C::kWaves, BCOLS> ob;
    int nch = 0;
    auto slice = [&](int sp) { return chunks * sp / splits; };     // first chunk of a slice
    auto setup = [&](const Item& it) __attribute__((always_inline)) {
        const int c0 = slice(it.sp);
        oa.set(g.a, g.lda, it.a0, g.na, c0 * kBK, g.a_rows);
        // (every stored row and column of B there is up to whole tiles)
        ob.set(g.b, g.ldb, it.b0, 1 << 30, c0 * kBK, 1 << 30);
    };
    auto issue = [&](int stage, int c) __attribute__((always_inline)) {
        uint8_t* st = ring + stage * C::kStage;
        oa.issue(st, c);
        ob.issue(st + C::kA, c);
    };
    Item cur = item_at(wid);
    setup(cur);
    nch = slice(cur.sp + 1) - slice(cur.sp);
#pragma unroll
    for (int c = 0; c < C::kP; ++c)
        if (c < nch) issue(c, c);
    int sc = 0;                               // stage of the chunk computed next

    for (;;) {
        const int nwid = wid + per_xcd;
        const bool more = nwid < wend;        // uniform
        const Item nxt = more ? item_at(nwid) : cur;
        const bool active = cur.b0 + brow < (OUT == GRAD ? (nb + kBK - 1) / kBK * kBK : nb);
        f32x16 acc[FA][FB];
#pragma unroll
        for (int i = 0; i < FA; ++i)
#pragma unroll
            for (int j = 0; j < FB; ++j) acc[i][j] = f32x16{};

        // one step of the ring: wait for this wave's loads of chunk c, barrier
        // (every wave's have landed, and every wave is done with the stage
        // before), refill that stage, compute
        for (int c = 0; c < nch; ++c) {
            const int after = min(C::kP - 1, nch - 1 - c);
            if (C::kP >= 3 && after >= 2) wait_vm<(C::kP >= 3 ? 2 : 0) * C::kLoads>();
            else if (C::kP >= 2 && after >= 1) wait_vm<(C::kP >= 2 ? 1 : 0) * C::kLoads>();
            else wait_vm<0>();
            lds_barrier();
            const int si = sc == 0 ? C::STAGES - 1 : sc - 1;
            if (c + C::kP < nch) issue(si, c + C::kP);
            const uint8_t* st = ring + sc * C::kStage;
            sc = sc + 1 == C::STAGES ? 0 : sc + 1;
            if (!active) continue;
#pragma unroll
            for (int s = 0; s < kBK / 16; ++s) {
                bf16x8 A[FA], B[FB];
#pragma unroll
                for (int j = 0; j < FB; ++j) B[j] = fragment<C::NB, BCOLS>(st + C::kA, brow + 32 * j, s);
#pragma unroll
                for (int i = 0; i < FA; ++i) A[i] = fragment<C::NA, ACOLS>(st, arow + 32 * i, s);
#pragma unroll
                for (int j = 0; j < FB; ++j)
#pragma unroll
                    for (int i = 0; i < FA; ++i)
                        acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(A[i], B[j], acc[i][j], 0, 0, 0);
            }
        }
        lds_barrier();                        // every wave is done with the ring
        // lane: row cur.b0 + brow + 32 j + l32, columns cur.a0 + arow + 32 i + 8 (q / 4) + 4 lh + q % 4
        uint8_t* const tb = ring + wave * (C::STAGES * C::kStage / C::kWaves);
        static_assert(C::STAGES * C::kStage / C::kWaves >= 4096, "a fragment's rows fit a wave's share of the ring");
        // FA fragments' 32 rows of 64 FA bytes, turned around through the
        // wave's share of LDS so that adjacent lanes store adjacent pieces
        auto store16 = [&](int j, auto val, auto dst, int nv) __attribute__((always_inline)) {
            constexpr int V = 4 * FA;         // 16-byte pieces per row
            auto at = [&](int r, int v) { return r * (64 * FA) + ((v ^ (FA == 2 ? r & 7 : (r >> 1) & 3)) << 4); };
#pragma unroll
            for (int i = 0; i < FA; ++i)
#pragma unroll
                for (int qb = 0; qb < 4; ++qb)
                    *reinterpret_cast<uint2*>(tb + at(l32, 4 * i + qb) + 8 * lh) =
                        uint2{pack_bf16x2(val(i, 4 * qb), val(i, 4 * qb + 1)),
                              pack_bf16x2(val(i, 4 * qb + 2), val(i, 4 * qb + 3))};
            wave_lds_sync();
#pragma unroll
            for (int k = 0; k < 32 * V / 64; ++k) {
                const int r = (64 / V) * k + lane / V, v = lane % V;
                const u32x4 d = *reinterpret_cast<const u32x4*>(tb + at(r, v));
                if (r < nv) *reinterpret_cast<u32x4*>(dst(r) + 8 * v) = d;
            }
            wave_lds_sync();
        };
        if constexpr (OUT == LSE) {
            // the waves' maxima of a row, then its exponentials over the tile's
            // maximum and their sum: the tile's first columns may be kept
            float* const redm = reinterpret_cast<float*>(ring + 4096);       // [WA][NB], beside wave 0's rows
            float* const reds = redm + C::WA * C::NB;
            static_assert(4096 + 8 * C::WA * C::NB <= C::STAGES * C::kStage / C::kWaves, "within wave 0's share");
            const int v0 = cur.a0 + arow + 4 * lh;
            const bool tail = cur.a0 + C::NA > g.na;
            const bool kept = cur.a0 < g.kept;
            const int at = (wave % C::WA) * C::NB + brow + l32;
#pragma unroll
            for (int j = 0; j < FB; ++j) {
                const int row = cur.b0 + brow + 32 * j + l32;
                const int rel = row < nb ? g.target[row] - g.col0 - v0 : -1;      // the target counts as no column
                if (ballot(rel >= 0 && rel < 32 * FA) || tail) {
#pragma unroll
                    for (int i = 0; i < FA; ++i)
#pragma unroll
                        for (int q = 0; q < 16; ++q) {
                            const int v = 32 * i + 8 * (q / 4) + q % 4;
                            if (v == rel || v0 + v >= g.na) acc[i][j][q] = -INFINITY;
                        }
                }
                float m = -INFINITY;
#pragma unroll
                for (int i = 0; i < FA; ++i)
#pragma unroll
                    for (int q = 0; q < 16; ++q) m = fmaxf(m, acc[i][j][q]);
                m = fmaxf(m, swap_halves(m));
                if (lh == 0) redm[at + 32 * j] = m;
            }
            lds_barrier();
#pragma unroll
            for (int j = 0; j < FB; ++j) {
                float m = -INFINITY;
#pragma unroll
                for (int w = 0; w < C::WA; ++w) m = fmaxf(m, redm[w * C::NB + brow + 32 * j + l32]);
                const float ref = tile_ref(m);
                float s = 0.f;
#pragma unroll
                for (int i = 0; i < FA; ++i)
#pragma unroll
                    for (int q = 0; q < 16; ++q) {
                        acc[i][j][q] = __builtin_amdgcn_exp2f(fmaf(acc[i][j][q], kLog2e, -ref * kLog2e));
                        s += acc[i][j][q];
                    }
                s += swap_halves(s);
                if (lh == 0) reds[at + 32 * j] = s;
                const int row0 = cur.b0 + brow + 32 * j;
                if (kept && row0 < nb)
                    store16(j, [&](int i, int q) __attribute__((always_inline)) { return acc[i][j][q]; },
                            [&](int r) { return static_cast<uint16_t*>(g.out) + (row0 + r) * g.ldo + cur.a0 + arow; },
                            nb - row0);
            }
            lds_barrier();
            for (int r = threadIdx.x; r < C::NB; r += C::kThreads) {
                float m = -INFINITY, s = 0.f;
#pragma unroll
                for (int w = 0; w < C::WA; ++w) {
                    m = fmaxf(m, redm[w * C::NB + r]);
                    s += reds[w * C::NB + r];
                }
                if (m == INFINITY && s == s) s = 1.f;      // (some are +inf: the row's NLL is)
                if (cur.b0 + r < nb) g.part[static_cast<size_t>(cur.a0 / C::NA) * g.ldpart + cur.b0 + r] = float2{m, s};
            }
        } else if (active) {
            const int nrow = OUT == GRAD ? (nb + kBK - 1) / kBK * kBK : nb;
#pragma unroll
            for (int j = 0; j < FB; ++j) {
                const int row0 = cur.b0 + brow + 32 * j;
                const int nv = min(32, nrow - row0);
                if (nv <= 0) break;
                if constexpr (OUT == GRAD) {
                    const int row = row0 + l32;
                    const bool live = row < nb;
                    const float2 st = live ? g.stats[row] : float2{0.f, 0.f};
                    const int rel = (live ? g.target[row] : -1) - (g.col0 + cur.a0 + arow + 4 * lh);
                    const int end = live ? g.na - (cur.a0 + arow + 4 * lh) : 0;     // columns of the piece from here on
                    store16(j, [&](int i, int q) __attribute__((always_inline)) {
                        const int v = 32 * i + 8 * (q / 4) + q % 4;
                        float p = __builtin_amdgcn_exp2f(fmaf(acc[i][j][q], kLog2e, -st.x));
                        p = v == rel ? st.y : p;
                        return v < end ? p : 0.f;
                    }, [&](int r) { return static_cast<uint16_t*>(g.out) + (row0 + r) * g.ldo + cur.a0 + arow; }, nv);
                } else if constexpr (OUT == ROWS) {
                    if (cur.a0 + arow >= g.na) break;      // (columns come in multiples of 64)
                    store16(j, [&](int i, int q) __attribute__((always_inline)) { return acc[i][j][q] * coef; },
                            [&](int r) {
                                const int64_t to = g.rows && r < nv ? g.rows[row0 + r] : row0 + r;
                                return static_cast<uint16_t*>(g.out) + to * g.ldo + cur.a0 + arow;
                            }, nv);
                } else {
                    auto at = [&](int r, int v) { return r * 128 + ((v ^ (r & 7)) << 4); };
#pragma unroll
                    for (int i = 0; i < FA; ++i) {
                        const int col = cur.a0 + arow + 32 * i;
                        if (col >= g.na) break;
#pragma unroll
                        for (int qb = 0; qb < 4; ++qb)
                            *reinterpret_cast<f32x4*>(tb + at(l32, 2 * qb + lh)) =
                                f32x4{acc[i][j][4 * qb], acc[i][j][4 * qb + 1], acc[i][j][4 * qb + 2], acc[i][j][4 * qb + 3]};
                        wave_lds_sync();
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            const int r = 8 * k + lane / 8, v = lane % 8;
                            f32x4 d = *reinterpret_cast<const f32x4*>(tb + at(r, v));
                            if (r < nv) {
                                float* const p = static_cast<float*>(g.out) + cur.sp * g.split_stride +
                                                 (row0 + r) * g.ldo + col + 4 * v;
                                if (g.add) d += *reinterpret_cast<const f32x4*>(p);
                                *reinterpret_cast<f32x4*>(p) = d;
                            }
                        }
                        wave_lds_sync();
                    }
                }
            }
        }
        if (!more) break;
        cur = nxt;
        wid = nwid;
        __syncthreads();
        setup(cur);
        nch = slice(cur.sp + 1) - slice(cur.sp);
        sc = 0;
#pragma unroll
        for (int c = 0; c < C::kP; ++c)
            if (c < nch) issue(c, c);
    }
}

// ------------------------------------------------------------- row kernels --

// rows[0 .. n): the rows whose target is not `ignore`, in order; head: {n,
// n rounded up to whole reduction chunks, 0}.  One workgroup: the list is a running sum over the call.
constexpr int kCompactThreads = 1024, kCompactLoads = 8;
__global__ __launch_bounds__(kCompactThreads) void compact_kernel(const int32_t* __restrict__ target, int T, int ignore,
                                                                  int32_t* rows, int32_t* head) {
    constexpr int NW = kCompactThreads / kWave;
    __shared__ int cnt[kCompactLoads][NW];
    const int lane = lane_id(), wave = threadIdx.x / kWave;
    const uint64_t below = lane == 0 ? 0ull : ~0ull >> (kWave - lane);
    int base = 0;
    for (int t0 = 0; t0 < T; t0 += kCompactThreads * kCompactLoads) {
        bool keep[kCompactLoads];
        uint64_t m[kCompactLoads];
#pragma unroll
        for (int i = 0; i < kCompactLoads; ++i) {
            const int t = t0 + i * kCompactThreads + threadIdx.x;
            keep[i] = t < T && target[t < T ? t : 0] != ignore;
        }
#pragma unroll
        for (int i = 0; i < kCompactLoads; ++i) {
            m[i] = ballot(keep[i]);
            if (lane == 0) cnt[i][wave] = __popcll(m[i]);
        }
        __syncthreads();
        for (int i = 0; i < kCompactLoads; ++i) {
            int at = base;
            for (int w = 0; w < NW; ++w) {
                const int c = cnt[i][w];
                at += w < wave ? c : 0;
                base += c;
            }
            if (keep[i]) rows[at + __popcll(m[i] & below)] = t0 + i * kCompactThreads + threadIdx.x;
        }
        __syncthreads();
    }
    if (threadIdx.x == 0) {
        head[0] = base;
        head[1] = (base + kBK - 1) / kBK * kBK;
        head[2] = 0;
    }
}

// One wave per row.  Row t of the call, where it is ignored: its NLL and its
// dh are zero.  Row i of the list: its hidden row, its target and the target's
// logit in fp64 (the NLL would depend most on that logit's rounding); rows
// behind the list up to whole tiles: zeros.
constexpr int kGatherWaves = 4;
__global__ __launch_bounds__(kGatherWaves * kWave) void gather_kernel(
    const uint16_t* __restrict__ h, const uint16_t* __restrict__ w, const int32_t* __restrict__ target, int T, int Tpad,
    int d, int V, int ignore, const int32_t* __restrict__ rows, const int32_t* __restrict__ head, uint16_t* hc,
    int32_t* tc, double* zt, float* nll, uint16_t* dh) {
    const int lane = lane_id(), i = blockIdx.x * kGatherWaves + threadIdx.x / kWave;
    const int n = head[0];
    if (i < T && target[i] == ignore) {
        if (nll && lane == 0) nll[i] = 0.f;
        if (dh)
            for (int k = 8 * lane; k < d; k += 8 * kWave)
                *reinterpret_cast<uint4*>(dh + static_cast<size_t>(i) * d + k) = uint4{};
    }
    if (i >= Tpad || i >= (n + 255) / 256 * 256) return;
    const int t = i < n ? rows[i] : 0;
    const int y = i < n ? target[t] : 0;
    const bool known = y >= 0 && y < V;
    double z = 0.0;
    for (int k = 8 * lane; k < d; k += 8 * kWave) {
        const uint4 p = i < n ? *reinterpret_cast<const uint4*>(h + static_cast<size_t>(t) * d + k) : uint4{};
        const uint4 q = *reinterpret_cast<const uint4*>(w + static_cast<size_t>(known ? y : 0) * d + k);
        *reinterpret_cast<uint4*>(hc + static_cast<size_t>(i) * d + k) = p;
        const uint32_t pw[4] = {p.x, p.y, p.z, p.w}, qw[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            z = fma(static_cast<double>(__uint_as_float(pw[e] << 16)), static_cast<double>(__uint_as_float(qw[e] << 16)), z);
            z = fma(static_cast<double>(__uint_as_float(pw[e] & 0xffff0000u)),
                    static_cast<double>(__uint_as_float(qw[e] & 0xffff0000u)), z);
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
constexpr int kRowWaves = 8;
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
    const int i = blockIdx.x * kWave + lane;
    float m = -INFINITY, s = 0.f;
    auto merge = [&](float2 p) __attribute__((always_inline)) {
        const float hi = fmaxf(m, p.x);
        s = (m == hi ? s : s * __expf(m - hi)) + (p.x == hi ? p.y : p.y * __expf(p.x - hi));
        m = hi;
    };
    if (i < n) {
        for (int t0 = wave; t0 < ntiles; t0 += 8 * kRowWaves) {
            float2 p[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const int t = t0 + u * kRowWaves;
                p[u] = part[static_cast<size_t>(t < ntiles ? t : t0) * ldpart + i];
            }
#pragma unroll
            for (int u = 0; u < 8; ++u)
                if (t0 + u * kRowWaves < ntiles) merge(p[u]);
        }
    }
    red[wave][lane] = float2{m, s};
    __syncthreads();
    if (wave == 0 && i < n) {
        for (int w = 1; w < kRowWaves; ++w) merge(red[w][lane]);
        // (zt - zt is NaN for an infinite target, as its row's logsumexp less itself)
        const double md = m, rest = s, z = zt[i];
        double v, lse;
        if (z >= md) {
            v = log1p(rest * exp(md - z)) + (z - z);
            lse = z + v;
        } else {
            lse = md + log(rest + exp(z - md));
            v = lse - z;
        }
        if (tc[i] < 0) v = lse = NAN;
        nllc[i] = v;
        stats[i] = float2{static_cast<float>(lse * 1.4426950408889634), static_cast<float>(expm1(-v))};
        if (nll) nll[rows[i]] = static_cast<float>(v);
    }
    if (threadIdx.x == 0) {
        __threadfence();
        last = __hip_atomic_fetch_add(head + 2, 1, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) == blocks - 1;
    }
    __syncthreads();
    if (!last) return;
    __threadfence();
    double a = 0.0;
    for (int r = threadIdx.x; r < n; r += kRowWaves * kWave)
        a += __hip_atomic_load(nllc + r, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
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

// G of the columns whose exponentials the first pass kept, in place: a tile of
// the first pass x 64 rows per workgroup, 16 bytes per lane.  Twice the piece's
// bytes against taking its product again (4096 rows of 32000 columns, d 4096:
// see launch_ce).  Rows behind the list up to a whole reduction chunk: zeros.
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
            v = float4{m == -INFINITY ? 0.f * st.x : __builtin_amdgcn_exp2f(fmaf(tile_ref(m), kLog2e, -st.x)), st.y,
                       __int_as_float(tc[i] - c0), 0.f};
        }
        row[tid] = v;
    }
    uint16_t* const at = g + (r0 + tid / V) * ldg + c0 + 8 * (tid % V);
    uint4 v[kScaleRows / R];
#pragma unroll
    for (int k = 0; k < kScaleRows / R; ++k) v[k] = *reinterpret_cast<const uint4*>(at + k * R * ldg);
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kScaleRows / R; ++k) {
        const int r = tid / V + k * R;
        const float4 p = row[r];
        const int rel = __float_as_int(p.z) - 8 * (tid % V);
        const uint32_t w[4] = {v[k].x, v[k].y, v[k].z, v[k].w};
        uint32_t o[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            float lo = __uint_as_float(w[e] << 16) * p.x, hi = __uint_as_float(w[e] & 0xffff0000u) * p.x;
            lo = rel == 2 * e ? p.y : lo;
            hi = rel == 2 * e + 1 ? p.y : hi;
            o[e] = r0 + r < n ? pack_bf16x2(lo, hi) : 0u;
        }
        *reinterpret_cast<uint4*>(at + k * R * ldg) = uint4{o[0], o[1], o[2], o[3]};
    }
}

// dh of the listed rows: its slices added in order, times c.
constexpr int kJoinThreads = 256;
__global__ __launch_bounds__(kJoinThreads) void join_kernel(const float* __restrict__ part, int splits, int64_t stride,
                                                            const int32_t* __restrict__ head,
                                                            const int32_t* __restrict__ rows, int d,
                                                            const float* __restrict__ coef, uint16_t* dh) {
    const int n = head[0];
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
        *reinterpret_cast<uint4*>(dh + static_cast<size_t>(rows[i]) * d + k) =
            uint4{pack_bf16x2(lo[0] * c, lo[1] * c), pack_bf16x2(lo[2] * c, lo[3] * c),
                  pack_bf16x2(hi[0] * c, hi[1] * c), pack_bf16x2(hi[2] * c, hi[3] * c)};
    }
}

struct Geometry {
    int cus, xcds;
};
const Geometry& geometry() {
    static const Geometry g = [] {
        int dev = 0, cus = 0, xccs = 0;
        if (hipGetDevice(&dev) != hipSuccess ||
            hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || cus < 1)
            cus = 256;
        if (hipDeviceGetAttribute(&xccs, hipDeviceAttributeNumberOfXccs, dev) != hipSuccess || xccs < 1 || xccs > cus)
            xccs = 1;
        return Geometry{cus, xccs};
    }();
    return g;
}

// Persistent: a workgroup per CU (the ring fills its LDS) or per item, a
// multiple of the XCD count.
template <class C, bool ACOLS, bool BCOLS, int OUT>
hipError_t launch_gemm(GemmArgs g, hipStream_t s) {
    g.xcds = geometry().xcds;
    const int64_t work = static_cast<int64_t>((g.na + C::NA - 1) / C::NA) * ((g.nb + C::NB - 1) / C::NB) * g.splits;
    if (work == 0) return hipSuccess;
    int64_t blocks = std::min<int64_t>(work, geometry().cus);
    blocks = std::max<int64_t>(g.xcds, (blocks + g.xcds - 1) / g.xcds * g.xcds);
    ce_gemm<C, ACOLS, BCOLS, OUT><<<static_cast<int>(blocks), C::kThreads, 0, s>>>(g);
    return hipGetLastError();
}

// Calls of few rows take the tile of 64 rows, which streams the head.
bool small_call(int T) { return T <= Small::NB; }

// G held at a time: a piece of the vocabulary whose G takes kPieceBytes at
// most (1.4% of the card's memory) and, with a smaller workspace, what fits,
// from kMinPiece columns on.  The first piece costs a pass over its G, every
// other one its product again.
constexpr size_t kPieceBytes = size_t{4} << 30;
constexpr int kMinPiece = 4096;

}  // namespace

CePlan plan_ce(int32_t T, int32_t d, int32_t V, bool dh, bool dw, size_t bytes) {
    CePlan p{};
    p.rows_pad = small_call(T) ? Small::NB : (T + Big::NB - 1) / Big::NB * Big::NB;
    const size_t tp = p.rows_pad;
    p.tile = small_call(T) ? Small::NA : Big::NA;
    p.tiles = (V + p.tile - 1) / p.tile;
    const int vpad = (V + 255) / 256 * 256;
    const int least = std::min(vpad, kMinPiece);
    auto fit = [&](size_t room) {
        return static_cast<int>(std::max<size_t>(least, std::min<size_t>(vpad, room / (2 * tp) / 256 * 256)));
    };
    // dh: slices of the reduction until the CUs have an item each, none under 4 chunks
    const int nb = small_call(T) ? Small::NB : Big::NB;
    const int64_t items = static_cast<int64_t>((T + nb - 1) / nb) * ((d + p.tile - 1) / p.tile);
    p.splits = 1;
    while (dh && items * p.splits * 2 <= 256 && vpad / kBK / (p.splits * 2) >= 4) p.splits *= 2;
    auto layout = [&](int piece) {
        size_t off = 0;
        auto take = [&](size_t n) { const size_t at = off; off += (n + 255) & ~size_t(255); return at; };
        p.piece = piece;
        p.parts = dh && (p.splits > 1 || piece < vpad) ? p.splits : 0;
        p.head = take(16);
        p.coef = take(4);
        p.rows = take(static_cast<size_t>(T) * 4);
        p.tc = take(tp * 4);
        p.zt = take(tp * 8);
        p.nllc = take(tp * 8);
        p.stats = take(tp * 8);
        p.hc = take(tp * d * 2);
        p.part = take(tp * p.tiles * 8);
        p.dhp = take(static_cast<size_t>(p.parts) * tp * d * 4);
        p.g = off;
        p.total = off + (dh || dw ? tp * piece * 2 : 0);
    };
    layout(fit(kPieceBytes));
    if (p.total <= bytes || (!dh && !dw)) return p;
    layout(least < vpad ? least : vpad);
    if (bytes > p.total) layout(std::min(vpad, fit(bytes - p.g)));
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
    const bool small = small_call(T);

    compact_kernel<<<1, kCompactThreads, 0, s>>>(c.target, T, c.ignore, rows, head);
    gather_kernel<<<(p.rows_pad + kGatherWaves - 1) / kGatherWaves, kGatherWaves * kWave, 0, s>>>(
        c.h, c.w, c.target, T, p.rows_pad, d, V, c.ignore, rows, head, hc, tc, zt, c.nll, c.dh);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    GemmArgs z{};
    z.a = c.w; z.lda = d; z.na = V;
    z.b = hc; z.ldb = d; z.nb = T; z.nb_dev = head;
    z.K = d; z.splits = 1;
    z.part = part; z.ldpart = p.rows_pad; z.target = tc;
    z.out = gbuf; z.ldo = p.piece; z.kept = c.dh || c.dw ? p.piece : 0;
    e = small ? launch_gemm<Small, false, false, LSE>(z, s) : launch_gemm<Big, false, false, LSE>(z, s);
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
            if (small) scale_kernel<Small::NA><<<grid, kScaleThreads, 0, s>>>(part, p.rows_pad, stats, tc, head, gbuf, p.piece);
            else scale_kernel<Big::NA><<<grid, kScaleThreads, 0, s>>>(part, p.rows_pad, stats, tc, head, gbuf, p.piece);
            e = hipGetLastError();
        } else {
            GemmArgs q = z;
            q.a = w; q.na = nv; q.col0 = v0;
            q.stats = stats;
            e = small ? launch_gemm<Small, false, false, GRAD>(q, s) : launch_gemm<Big, false, false, GRAD>(q, s);
        }
        if (e == hipSuccess && c.dh) {
            GemmArgs a{};
            a.a = w; a.lda = d; a.na = d; a.a_rows = nv;
            a.b = gbuf; a.ldb = p.piece; a.nb = T; a.nb_dev = head;
            a.K = nv; a.splits = p.splits;
            if (p.parts) {
                a.out = dhp; a.ldo = d; a.split_stride = static_cast<int64_t>(p.rows_pad) * d; a.add = v0 > 0;
                e = small ? launch_gemm<Small, true, false, PART>(a, s) : launch_gemm<Big, true, false, PART>(a, s);
            } else {
                a.out = c.dh; a.ldo = d; a.rows = rows; a.coef = coef;
                e = small ? launch_gemm<Small, true, false, ROWS>(a, s) : launch_gemm<Big, true, false, ROWS>(a, s);
            }
        }
        if (e == hipSuccess && c.dw) {
            GemmArgs a{};
            a.a = hc; a.lda = d; a.na = d; a.a_rows = 1 << 30;
            a.b = gbuf; a.ldb = p.piece; a.nb = nv;
            a.K = p.rows_pad; a.k_dev = head + 1; a.splits = 1;
            a.out = c.dw + static_cast<size_t>(v0) * d; a.ldo = d; a.coef = coef;
            e = launch_gemm<Big, true, true, ROWS>(a, s);
        }
    }
    if (e == hipSuccess && p.parts) {
        const int64_t n8 = static_cast<int64_t>(T) * (d / 8);
        join_kernel<<<static_cast<int>(std::min<int64_t>((n8 + kJoinThreads - 1) / kJoinThreads, 2048)), kJoinThreads, 0, s>>>(
            dhp, p.splits, static_cast<int64_t>(p.rows_pad) * d, head, rows, d, coef, c.dh);
        e = hipGetLastError();
    }
    return e;
}

}  // namespace eat
