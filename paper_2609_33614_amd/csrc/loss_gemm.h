// The products of the losses' gradients (gfx950):
//   C[b][a] = sum_k A[a][k] B[b][k]
// in bf16 with fp32 accumulation on v_mfma_f32_32x32x16_bf16 (a lane ends with
// 4 consecutive columns a of one row b).  Either operand may be stored with
// its reduction index as the row ("columns": the head for dh; G and h for dW):
// its LDS tile is then [k][index], and the fragments come out of transposing
// LDS reads (ds_read_b64_tr_b16: the 16 lanes of a group read a 4 x 16 block, 4
// lanes a row, and each gets a column of it), so no operand is transposed in
// memory.  The kernel's output side is one of Out: the cross entropy's first
// pass (LSE) and its recomputed pieces (GRAD), fp32 slices of a split reduction
// (PART), finished rows (ROWS, ROWS32).
//
// A workgroup has a CU to itself and works a list of tiles; the tiles of an XCD's
// workgroups lie next to each other, so that its L2 holds what they share.  Loads
// go straight to LDS into a ring of half chunks and run ahead over the ends of the
// tiles: a tile's output is written while the next one's operands arrive.  What
// bounds the large tile is the card's power (its clock falls to 1.5 - 1.6 GHz under
// these products): 1.21 - 1.34 PFLOP/s for LSE, 1.24 - 1.29 for dh, 1.05 - 1.22
// for dW, where a library product takes 1.29 - 1.53, 1.26 - 1.40 and 1.00 - 1.15
// (8192 x 4096 x 32768, timed in turn).
//
// The header's kernels are instantiated by ce.hip and balance.hip.
#pragma once
#include <algorithm>

#include "eat_device.h"
#include "eat_internal.h"

namespace eat {
namespace {

constexpr int kBK = 64;                   // reduction chunk (bf16 elements)
constexpr float kLog2e = 1.44269504088896340736f;

typedef short s16x4 __attribute__((ext_vector_type(4)));

// NA x NB outputs per workgroup, WA x WB waves over them.  A chunk is two
// parts, A's and B's, and LDS a ring of SLOTS parts: the two computed and
// kAhead loaded or on their way.
template <int NA_, int NB_, int WA_, int WB_>
struct Tile {
    static constexpr int NA = NA_, NB = NB_, WA = WA_, WB = WB_;
    static constexpr int kWaves = WA * WB;
    static constexpr int kThreads = kWaves * kWave;
    static constexpr int FA = NA / (32 * WA), FB = NB / (32 * WB);    // 32-wide fragments per wave
    static constexpr int kA = NA * kBK * 2, kB = NB * kBK * 2;        // bytes of a chunk's parts
    static constexpr int kSlot = kA > kB ? kA : kB;
    static constexpr int SLOTS = (160 * 1024 / kSlot - 1) | 1;        // odd
    static constexpr int kAhead = SLOTS - 2;
    static constexpr int kLA = kA / 1024 / kWaves, kLB = kB / 1024 / kWaves;   // 1 KB loads per wave
    static constexpr int kShare = 2 * kSlot / kWaves;                 // a wave's bytes of two slots
    static_assert(kLA * 1024 * kWaves == kA && kLB * 1024 * kWaves == kB, "loads split evenly over the waves");
    static_assert(FA * 32 * WA == NA && FB * 32 * WB == NB, "fragments cover the tile");
    static_assert(kAhead >= 3, "a chunk and the next one's first part");
    static_assert(kShare >= 4096 && kShare >= 2048 * FA + 256 * FB, "a fragment's rows and sums fit a wave's share");
    // loads of `parts` parts in a row, the first of them A's
    static constexpr int loads(int parts) { return (parts + 1) / 2 * kLA + parts / 2 * kLB; }
};
using Big = Tile<256, 256, 4, 2>;
using Mid = Tile<128, 128, 4, 2>;
using Small = Tile<128, 64, 4, 2>;

enum Out { LSE, GRAD, PART, ROWS, ROWS32 };

struct GemmArgs {
    const uint16_t* a;
    const uint16_t* b;
    int lda, ldb;              // elements between stored rows
    int na, nb, K;             // output columns and rows, reduction length (nb, K: upper bounds where *_dev is set)
    const int32_t* nb_dev;     // rows of the output, on the device (or null)
    const int32_t* k_dev;      // reduction length, on the device (or null), over k_times
    int k_times;
    int planes;                // 1: up to kFewRows of nb_dev's rows, or of k_dev's, have second parts, kFewRows on, that count too
    int a_rows;                // stored rows of a "columns" A operand (later ones read the last)
    const int32_t* k_rows;     // GATHER: the stored row of A of each reduction element (whole chunks of them)
    int segs, map;             // GROUPS, B by rows: see loss_gemm
    int splits;                // slices of the reduction (PART); 0: chosen on the device (pick_slices)
    int pool_rows, slice_chunks;   // ... by the rows the slices may take and the reduction's chunks
    int32_t* slices_out;       // ... and written there
    void* direct;              // ... and one slice goes there as ROWS (or null)
    int col0;                  // LSE, GRAD: vocabulary index of column 0
    int xcds;
    void* out;                 // GRAD, ROWS, LSE: bf16; ROWS32: fp32; PART: fp32 slices
    int64_t ldo;
    int64_t split_stride;      // PART: between slices (0: the output's whole tiles of rows)
    int kept;                  // LSE: columns below it leave exp(z - the tile's maximum) in out, by pack_kept or in two parts
    const int32_t* rows;       // ROWS, ROWS32: destination of each output row (or null: itself)
    const float* coef;         // ROWS: factor c on the device, or null: factor
    float factor;
    int add;                   // PART: add to what the slices hold
    float2* part;              // LSE: [column tile][ldpart] (maximum, sum) pairs
    int ldpart;
    const int32_t* target;     // LSE, GRAD: column that is the row's target
    const float2* stats;       // GRAD: (lse, G at the target) of a row
};

// The cross entropy keeps its G in two bf16 parts up to this many rows that count.
constexpr int kFewRows = 64;
// Rows there are when the second parts of so few follow as rows of their own.
__device__ __forceinline__ int with_parts(int n) { return n > 0 && n <= kFewRows ? kFewRows + n : n; }


// (uniform: what depends on it branches on scalars)
__device__ __forceinline__ int wave_id() { return __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) / kWave); }

// Operands stored row by row: LDS rows of 128 bytes (64 k), 16-byte slots XORed
// with the row's 256-byte line, so that an MFMA operand read of 16 rows covers
// every bank.
__device__ __forceinline__ int swz_row(int r) { return (static_cast<unsigned>(r) >> 1) & 7; }
// Operands stored by columns: LDS rows of N indices for each of the 64 k.  A
// transposing read takes 64 bytes of each of 4 consecutive k: XORing the slot
// with 4 (k % 4) puts them on different banks.
__device__ __forceinline__ int swz_col(int k) { return (k & 3) << 2; }

// v in scalar registers, ready to be a load's address: a vector instruction's
// write of one wants five wait states before a memory instruction reads it there,
// which the compiler does not count for loads written in asm.
__device__ __forceinline__ uint64_t uniform(uint64_t v) {
    v = static_cast<uint64_t>(static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(static_cast<uint32_t>(v >> 32)))) << 32 |
        static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(static_cast<uint32_t>(v)));
    asm volatile("s_nop 4" : "+s"(v));
    return v;
}

// Loads of one operand's part of a chunk: where lane l of load j gets the 16
// bytes that belong at LDS byte 1024 (wave + WAVES j) + 16 l of the part.
template <int N, int L, int WAVES, bool COLS, bool GATHER = false>
struct Operand {
    uint64_t src;              // uniform: where the chunk begins
    uint32_t step;             // to the next chunk's
    uint32_t ldbytes;
    uint32_t off[L];           // byte offset of the lane's 16 bytes from there (GATHER: from their row)
    int k_last;                // columns: last stored row, from the chunk's first
    const int32_t* rows;       // GATHER: where the reduction rows of the next chunk are stored
    int at[GATHER ? L : 1];    // GATHER: those of the chunk

    // first: the tile's first index, count: indices there are (>= 1), k0: the
    // slice's first k, k_rows: stored rows of a columns operand
    __device__ __forceinline__ void set(const uint16_t* p, int ld, int first, int count, int k0, int k_rows) {
        const int lane = lane_id(), wave = wave_id();
        ldbytes = static_cast<uint32_t>(ld) * 2;
        if constexpr (COLS) {
            src = uniform(reinterpret_cast<uint64_t>(p) + static_cast<uint64_t>(k0) * ldbytes);
            step = kBK * ldbytes;
            k_last = k_rows - 1 - k0;
            constexpr int VPR = N / 8;         // 16-byte slots per LDS row
#pragma unroll
            for (int j = 0; j < L; ++j) {
                const int g = (wave + WAVES * j) * 64 + lane;
                const int k = g / VPR, v = (g % VPR) ^ swz_col(k);
                off[j] = static_cast<uint32_t>(min(first + 8 * v, count - 8)) * 2;
                if constexpr (!GATHER) off[j] += __umul24(min(k, k_last), ldbytes);
            }
        } else {
            src = uniform(reinterpret_cast<uint64_t>(p) + static_cast<uint64_t>(first) * ldbytes + 2 * static_cast<uint64_t>(k0));
            step = kBK * 2;
            k_last = 0;
#pragma unroll
            for (int j = 0; j < L; ++j) {
                const int r = (wave + WAVES * j) * 8 + lane / 8, v = (lane & 7) ^ swz_row(r);
                off[j] = static_cast<uint32_t>(min(r, count - 1 - first)) * ldbytes + 16 * v;
            }
        }
    }
    __device__ __forceinline__ void next() {
        src += step;
        if constexpr (COLS && !GATHER) {
            k_last -= kBK;
            if (k_last < kBK - 1) {            // the last chunk, not a whole one: its last row again
#pragma unroll
                for (int j = 0; j < L; ++j) {
                    const int k = ((wave_id() + WAVES * j) * 64 + lane_id()) / (N / 8);
                    off[j] -= __umul24(max(k - k_last, 0), ldbytes);
                }
            }
        }
    }
    // the stored rows of the chunk at `rows`
    __device__ __forceinline__ void look_up() {
        if constexpr (GATHER) {
#pragma unroll
            for (int j = 0; j < L; ++j) at[j] = rows[((wave_id() + WAVES * j) * 64 + lane_id()) / (N / 8)];
        }
    }
    // load j of the chunk (at: src, in scalar registers) into the part at LDS byte `lds` (+ 1024
    // wave); a load is waited for by count: the compiler adds no waits of its own for asm
    // (nor the wait state between a write of M0 and the load that reads it: s_nop)
    __device__ __forceinline__ void load(uint32_t lds, uint64_t from, int j) const {
        const uint32_t o = off[j];
        if constexpr (GATHER) {
            const uint64_t p = from + static_cast<uint64_t>(at[j]) * ldbytes + o;
            asm volatile("s_add_u32 m0, %1, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off"
                         :: "v"(p), "s"(lds), "n"(1024 * WAVES * j) : "memory", "m0", "scc");
        } else {
            asm volatile("s_add_u32 m0, %2, %3\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1"
                         :: "v"(o), "s"(from), "s"(lds), "n"(1024 * WAVES * j) : "memory", "m0", "scc");
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

// Slices of a reduction of `chunks` over `items` tiles, every slice's `rows` fp32
// rows of `cols` taking tile_rows of the pool_rows there are: the count that
// takes least time, by its rounds over the CUs (about 1650 ns a chunk of the 256 x
// 256 tile, 800 of the smaller ones) and the slices' rows written and read again
// (about 4.5 TB/s).  A slice keeps four chunks.  (The times and the CU count
// only steer the choice.)
constexpr int kCus = 256, kMostSlices = 32;
constexpr int kBigNs = 1650, kMidNs = 800;
__device__ inline int pick_slices(int items, int chunks, int rows, int cols, int tile_rows, int pool_rows, int chunk_ns) {
    int best = 1;
    float least = 0.f;
    const float row_ns = static_cast<float>(rows) * static_cast<float>(cols) * (1.f / 562.f);
    for (int s = 1; s <= kMostSlices && (s == 1 || (s * tile_rows <= pool_rows && 4 * s <= chunks)); ++s) {
        const int each = static_cast<int>(static_cast<float>(chunks + s - 1) / static_cast<float>(s));
        const float cost = static_cast<float>((items * s + kCus - 1) / kCus) * static_cast<float>(each * chunk_ns) +
                           (s > 1 ? static_cast<float>(s) * row_ns : 0.f);
        if (s == 1 || cost < least) { best = s; least = cost; }
    }
    return best;
}
// The reference of a row's exponentials over a tile with maximum m (infinite
// where all are -inf, whose sum is 0, or some +inf: then 0).
__device__ __forceinline__ float tile_ref(float m) { return fabsf(m) == INFINITY ? 0.f : m; }
// exp(z - ref).  The difference comes first: either of them times log2 e may be
// past fp32's range.
__device__ __forceinline__ float exp_from(float z, float ref) { return __builtin_amdgcn_exp2f((z - ref) * kLog2e); }

// Exponentials of 0 to 1 in 16 bits each: fp32's 7 lower exponent bits (the sign and
// the upper one are 0 below 2) and 9 of its digits, two more than bf16 has, so
// that the rounding of what is made of them counts and theirs hardly does.
__device__ __forceinline__ uint32_t pack_kept(float a, float b) {
    const uint32_t x = (__float_as_uint(a) << 2) + 0x8000u, y = (__float_as_uint(b) << 2) + 0x8000u;
    return __builtin_amdgcn_perm(y, x, 0x07060302);        // (the upper halves)
}
__device__ __forceinline__ float kept_lo(uint32_t w) { return __uint_as_float((w & 0xffffu) << 14); }
__device__ __forceinline__ float kept_hi(uint32_t w) { return __uint_as_float((w >> 2) & 0x3fffc000u); }

// What the rounding of v to bf16 leaves.
__device__ __forceinline__ float bf16_rest(float v) { return v - __uint_as_float(pack_bf16x2(v, 0.f) << 16); }

__device__ __forceinline__ float swap_halves(float v) { return __shfl_xor(v, 32, kWave); }

// B may hold numbers of more than bf16's digits as sums of bf16 parts.
//   GROUPS: in groups of 64 indices of 4 parts each ([stored row][group][part]
//     [64], part 3 unused).  B by columns: a tile of 256 is a group, and the
//     products with its first three parts are added into one output row per index.
//     B by rows: the reduction runs over the groups, `segs` chunks of 64 each: chunk
//     i of a group is its part (map >> 4 i) & 15 (A holds the matching rows, chunk
//     by chunk).
//   PLANES: B by rows, 64 of them, and 64 rows on their second parts; the products
//     with both are added into one output row.
enum Fold { WHOLE, GROUPS, PLANES };

template <class C, bool ACOLS, bool BCOLS, int OUT, int FOLD = WHOLE, bool GATHER = false>
__global__ __launch_bounds__(C::kThreads) void loss_gemm(GemmArgs g) {
    constexpr bool kGroupTile = FOLD == GROUPS && BCOLS, kFolds = kGroupTile || FOLD == PLANES;
    static_assert(!kGroupTile || (C::NB == 256 && C::WB == 2), "a group per tile, 32 indices per wave");
    static_assert(FOLD != PLANES || (!BCOLS && C::NB == 128 && C::WB == 2), "two planes per tile, 32 rows per wave");
    constexpr int FA = C::FA, FB = kFolds ? 1 : C::FB;         // fragments of B held, and read
    constexpr int FL = kGroupTile ? 3 : FOLD == PLANES ? 2 : C::FB;
    constexpr int NBO = kFolds ? 64 : C::NB;                   // output rows per tile
    __shared__ __attribute__((aligned(1024))) uint8_t ring[C::SLOTS * C::kSlot];
    const int nb = g.nb_dev ? min(g.planes ? with_parts(*g.nb_dev) : *g.nb_dev, g.nb) : g.nb;
    const int K = g.k_dev ? min((g.planes ? with_parts(*g.k_dev) : *g.k_dev) * g.k_times, g.K) : g.K;
    const int nta = (g.na + C::NA - 1) / C::NA, ntb = (nb + NBO - 1) / NBO;
    const int chunks = (K + kBK - 1) / kBK;
    int splits = 1;
    if constexpr (OUT == PART) {
        splits = g.splits;
        if (splits == 0) {
            splits = __builtin_amdgcn_readfirstlane(pick_slices(nta * ntb, g.slice_chunks, nb, g.na, ntb * NBO,
                                                                g.pool_rows, C::NA == 256 ? kBigNs : kMidNs));
            if (blockIdx.x == 0 && threadIdx.x == 0) *g.slices_out = splits;
        }
    }
    const bool direct = OUT == PART && splits == 1 && g.direct && !(g.planes && *g.nb_dev <= kFewRows);
    const int64_t split_stride = g.split_stride ? g.split_stride : static_cast<int64_t>(ntb) * NBO * g.ldo;
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
        it.b0 = __builtin_amdgcn_readfirstlane((8 * grp + r % gb) * NBO);
        return it;
    };
    int wid = wbeg + slot;
    if (wid >= wend) return;                  // uniform over the workgroup

    const int lane = lane_id(), wave = wave_id();
    const int l32 = lane & 31, lh = lane >> 5;
    const int arow = 32 * FA * (wave % C::WA), brow = 32 * FB * (wave / C::WA);
    const bool parts = C::NB == kFewRows || nb <= kFewRows;     // LSE, GRAD: out in two parts, the second kFewRows rows on
    const float coef = (OUT == ROWS || OUT == ROWS32 || OUT == PART) ? (g.coef ? *g.coef : g.factor) : 1.f;

    auto slice = [&](int sp) { return chunks * sp / splits; };     // first chunk of a slice

    // The stream of loads: the parts A, B, A, B, ... of the chunks of this
    // workgroup's items, on into the next item while the last chunks of one are
    // computed and stored.  After the first A it goes by pairs, the B of the last
    // A and the A after it.  Behind the last chunk (`ended`) the pairs load that one
    // again, into slots nothing reads, so that the waits are constants; a workgroup
    // whose items have no chunks never loads (nor meets).
    Operand<C::NA, C::kLA, C::kWaves, ACOLS, GATHER> oa;
    Operand<C::NB, C::kLB, C::kWaves, BCOLS> ob;
    int iwid = wid - per_xcd, left = 1;       // the last A's item, chunks from it on
    int cb = 0, bfirst = 0;                   // GROUPS by rows: B's chunk and first row
    Item item{};
    bool fresh = false, ended = false;        // the last A is its item's first; there is none after it
    const uint32_t lds0 = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(ring)) + 1024 * wave;
    int islot = 0;                            // the slot loaded next
    auto next_a = [&]() __attribute__((always_inline)) {
        fresh = false;
        if (--left > 0) {
            oa.next();
            return;
        }
        for (iwid += per_xcd; iwid < wend; iwid += per_xcd) {          // the next item that has chunks
            item = item_at(iwid);
            const int c0 = slice(item.sp);
            left = slice(item.sp + 1) - c0;
            if (left == 0) continue;
            oa.set(g.a, g.lda, item.a0, g.na, GATHER ? 0 : c0 * kBK, g.a_rows);
            if constexpr (GATHER) {
                oa.step = 0;
                oa.rows = g.k_rows + c0 * kBK;
                oa.look_up();
            }
            fresh = true;
            return;
        }
        ended = true;
    };
    auto looked_up = [&]() __attribute__((always_inline)) {   // after A's loads: the next chunk's rows
        if constexpr (GATHER) {
            if (!ended && left > 1) {
                oa.rows += kBK;
                oa.look_up();
            }
        }
    };
    auto next_pair = [&]() __attribute__((always_inline)) {
        if (ended) return;
        if (fresh) {
            // (every stored row and column of B there is up to whole tiles)
            ob.set(g.b, g.ldb, item.b0 / NBO * C::NB, 1 << 30, slice(item.sp) * kBK, 1 << 30);
            cb = 0;
            bfirst = item.b0;
        } else {
            ob.next();
            ++cb;
        }
        next_a();
    };
    auto slot_at = [&](int ahead) __attribute__((always_inline)) {
        const int sl = islot + ahead;
        return (sl >= C::SLOTS ? sl - C::SLOTS : sl) * C::kSlot;
    };
    auto advance = [&](int parts) __attribute__((always_inline)) {
        islot += parts;
        if (islot >= C::SLOTS) islot -= C::SLOTS;
    };
    uint32_t ldsa = lds0, ldsb = 0;           // the pair's slots and sources
    uint64_t srca = 0, srcb = 0;
    auto pair_slots = [&]() __attribute__((always_inline)) {
        ldsb = lds0 + slot_at(0);
        ldsa = lds0 + slot_at(1);
        advance(2);
        srca = uniform(oa.src);
        srcb = uniform(ob.src);
        if constexpr (FOLD == GROUPS && !BCOLS) {        // the group's part that meets A's chunk (splits is 1: chunks from 0 on)
            const int c = cb / g.segs * 4 + ((g.map >> (4 * (cb % g.segs))) & 15);
            srcb = uniform(reinterpret_cast<uint64_t>(g.b + static_cast<size_t>(bfirst) * g.ldb) + c * (kBK * 2));
        }
    };
    // load q of a pair: B's, then A's
    auto pair_load = [&](int q) __attribute__((always_inline)) {
        if (q < C::kLB) ob.load(ldsb, srcb, q);
        else oa.load(ldsa, srca, q - C::kLB);
    };
    // Waits until at most the loads of the parts behind the chunk met next, and
    // `stores` output stores issued since, are still in flight (vector memory operations complete
    // in issue order for this counter; counting fewer only waits longer).
    auto wait_parts = [&](int stores) __attribute__((always_inline)) {
        constexpr int N = C::loads(C::kAhead - 2);
        if (stores == 0) wait_vm<N>();
        else if (stores < 8) wait_vm<N + 1>();
        else if (stores < 16) wait_vm<N + 8>();
        else wait_vm<N + 16>();
    };
    next_a();
    if (!ended) {
        srca = uniform(oa.src);
#pragma unroll
        for (int j = 0; j < C::kLA; ++j) oa.load(ldsa, srca, j);
        looked_up();
        advance(1);
#pragma unroll 1
        for (int i = 0; i < (C::kAhead - 1) / 2; ++i) {
            next_pair();
            pair_slots();
#pragma unroll
            for (int q = 0; q < C::kLA + C::kLB; ++q) pair_load(q);
            looked_up();
        }
    }
    int slot0 = 0;                            // slot of the chunk met next
    int stored = 0;                           // output stores since the loads it awaits

    for (;;) {
        const Item cur = item_at(wid);
        const int nch = slice(cur.sp + 1) - slice(cur.sp);
        const bool active = cur.b0 + brow < (OUT == GRAD ? (nb + kBK - 1) / kBK * kBK : nb);
        // what the epilogue needs of the rows, before the loads it would wait behind
        int target[FB];
        float2 stats[FB];
#pragma unroll
        for (int j = 0; j < FB; ++j) {
            const int row = cur.b0 + brow + 32 * j + l32;
            if constexpr (OUT == LSE || OUT == GRAD) target[j] = nb > 0 ? g.target[min(row, nb - 1)] : 0;
            if constexpr (OUT == GRAD) stats[j] = nb > 0 ? g.stats[min(row, nb - 1)] : float2{};
        }
        f32x16 acc[FA][FB];
#pragma unroll
        for (int i = 0; i < FA; ++i)
#pragma unroll
            for (int j = 0; j < FB; ++j) acc[i][j] = f32x16{};

        // The ring's step to a chunk: wait for this wave's loads of it, barrier
        // (every wave's have landed, and every wave has read the chunk before),
        // refill that one's slots.  It comes before the last of the 4 products of the
        // chunk before, whose fragments are in registers, so the matrix cores
        // have work while the waves meet and read on; inside a chunk the
        // fragments of a product are read during the one before.
        bf16x8 A[2][FA], B[2][FL];
        const uint8_t *sa = ring, *sb = ring;
        auto read = [&](int p, int s) __attribute__((always_inline)) {
#pragma unroll
            for (int j = 0; j < FL; ++j) B[p][j] = fragment<C::NB, BCOLS>(sb, brow + (kFolds ? 64 : 32) * j, s);
#pragma unroll
            for (int i = 0; i < FA; ++i) A[p][i] = fragment<C::NA, ACOLS>(sa, arow + 32 * i, s);
        };
        auto product = [&](int p, int j, int i) __attribute__((always_inline)) {
            f32x16& c16 = acc[i][kFolds ? 0 : j];
            c16 = __builtin_amdgcn_mfma_f32_32x32x16_bf16(A[p][i], B[p][j], c16, 0, 0, 0);
        };
        auto products = [&](int p) __attribute__((always_inline)) {
#pragma unroll
            for (int j = 0; j < FL; ++j)
#pragma unroll
                for (int i = 0; i < FA; ++i) product(p, j, i);
        };
        constexpr int kReads = FA * (ACOLS ? 2 : 1) + FL * (BCOLS ? 2 : 1), kProducts = FA * FL;
        constexpr int kPerProduct = (kReads + kProducts - 1) / kProducts;
        auto spread = [&]() __attribute__((always_inline)) {      // reads evenly between the products
#pragma unroll
            for (int m = 0; m < kProducts; ++m) {
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                __builtin_amdgcn_sched_group_barrier(0x100, kPerProduct, 0);
            }
            __builtin_amdgcn_sched_barrier(0);
        };
        auto meet = [&](int stores) __attribute__((always_inline)) {
            wait_parts(stores);
            lds_barrier();
            sa = ring + slot0 * C::kSlot;
            slot0 = slot0 + 1 == C::SLOTS ? 0 : slot0 + 1;
            sb = ring + slot0 * C::kSlot;
            slot0 = slot0 + 1 == C::SLOTS ? 0 : slot0 + 1;
            next_pair();
            pair_slots();
        };
        auto first_three = [&]() __attribute__((always_inline)) {
            read(1, 1);
            products(0);
            spread();
            read(0, 2);
            products(1);
            spread();
            read(1, 3);
            products(0);
            spread();
        };
        constexpr int kPair = C::kLA + C::kLB;
        if (nch > 0) {
            meet(stored);
            read(0, 0);
#pragma unroll
            for (int q = 0; q < kPair; ++q) pair_load(q);
            looked_up();
            for (int c = 1; c < nch; ++c) {
                first_three();
                meet(0);
                read(0, 0);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int m = 0; m < kProducts; ++m) {
                    product(1, m / FA, m % FA);
                    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                    for (int q = m * kPair / kProducts; q < (m + 1) * kPair / kProducts; ++q) pair_load(q);
                    __builtin_amdgcn_sched_barrier(0);
                }
                looked_up();
            }
            first_three();
            products(1);
        }
        lds_barrier();                        // every wave is done with the ring's two next slots
        stored = 0;
        // lane: row cur.b0 + brow + 32 j + l32, columns cur.a0 + arow + 32 i + 8 (q / 4) + 4 lh + q % 4
        auto share = [&](int w) __attribute__((always_inline)) {      // wave w's bytes of those slots
            return ring + slot_at(w >= C::kWaves / 2) + w % (C::kWaves / 2) * C::kShare;
        };
        uint8_t* const tb = share(wave);
        // FA fragments' 32 rows of 64 FA bytes, turned around through the
        // wave's share of LDS so that adjacent lanes store adjacent pieces
        auto as_bf16 = [](float a, float b) __attribute__((always_inline)) { return pack_bf16x2(a, b); };
        auto store16 = [&](int j, auto val, auto dst, int nv, auto pack) __attribute__((always_inline)) {
            constexpr int V = 4 * FA;         // 16-byte pieces per row
            auto at = [&](int r, int v) { return r * (64 * FA) + ((v ^ (FA == 1 ? (r >> 1) & 3 : r & (4 * FA - 1))) << 4); };
#pragma unroll
            for (int i = 0; i < FA; ++i)
#pragma unroll
                for (int qb = 0; qb < 4; ++qb)
                    *reinterpret_cast<uint2*>(tb + at(l32, 4 * i + qb) + 8 * lh) =
                        uint2{pack(val(i, 4 * qb), val(i, 4 * qb + 1)), pack(val(i, 4 * qb + 2), val(i, 4 * qb + 3))};
            wave_lds_sync();
#pragma unroll
            for (int k = 0; k < 32 * V / 64; ++k) {
                if ((64 / V) * k >= nv) break;
                const int r = (64 / V) * k + lane / V, v = lane % V;
                const u32x4 d = *reinterpret_cast<const u32x4*>(tb + at(r, v));
                // (past the caches, which the operands that are read again need: dW
                // of 32000 x 4096 from one row took 121 us through them and 70 so,
                // a router gradient of 16384 x 4096 290 and 246; nothing got slower)
                if (r < nv) __builtin_nontemporal_store(d, reinterpret_cast<u32x4*>(dst(r) + 8 * v));
                ++stored;
            }
            wave_lds_sync();
        };
        if constexpr (OUT == LSE) {
            // the waves' maxima of a row, then its exponentials over the tile's
            // maximum and their sum: the tile's first columns may be kept
            auto sums = [&](int w) { return reinterpret_cast<float*>(share(w) + 2048 * FA); };   // [2][32 FB] of wave w
            const int wb = wave / C::WA;
            const int v0 = cur.a0 + arow + 4 * lh;
            const bool tail = cur.a0 + C::NA > g.na;
            const bool kept = cur.a0 < g.kept;
#pragma unroll
            for (int j = 0; j < FB; ++j) {
                const int rel = target[j] - g.col0 - v0;                // the target counts as no column
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
                if (lh == 0) sums(wave)[32 * j + l32] = m;
            }
            lds_barrier();
#pragma unroll
            for (int j = 0; j < FB; ++j) {
                float m = -INFINITY;
#pragma unroll
                for (int w = 0; w < C::WA; ++w) m = fmaxf(m, sums(C::WA * wb + w)[32 * j + l32]);
                const float ref = tile_ref(m);
                float s = 0.f;
#pragma unroll
                for (int i = 0; i < FA; ++i)
#pragma unroll
                    for (int q = 0; q < 16; ++q) {
                        acc[i][j][q] = exp_from(acc[i][j][q], ref);
                        s += acc[i][j][q];
                    }
                s += swap_halves(s);
                if (lh == 0) sums(wave)[32 * (FB + j) + l32] = s;
                const int row0 = cur.b0 + brow + 32 * j;
                if (kept && row0 < nb) {
                    auto to = [&](int r) { return static_cast<uint16_t*>(g.out) + (row0 + r) * g.ldo + cur.a0 + arow; };
                    auto value = [&](int i, int q) __attribute__((always_inline)) { return acc[i][j][q]; };
                    if (parts) {
                        store16(j, value, to, nb - row0, as_bf16);
                        store16(j, [&](int i, int q) __attribute__((always_inline)) { return bf16_rest(acc[i][j][q]); },
                                [&](int r) { return to(r) + kFewRows * g.ldo; }, nb - row0, as_bf16);
                    } else {
                        store16(j, value, to, nb - row0, [](float a, float b) __attribute__((always_inline)) { return pack_kept(a, b); });
                    }
                }
            }
            lds_barrier();
            for (int r = threadIdx.x; r < C::NB; r += C::kThreads) {
                const int rb = r / (32 * FB), at = r % (32 * FB);
                float m = -INFINITY, s = 0.f;
#pragma unroll
                for (int w = 0; w < C::WA; ++w) {
                    m = fmaxf(m, sums(C::WA * rb + w)[at]);
                    s += sums(C::WA * rb + w)[32 * FB + at];
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
                    const float2 st = stats[j];
                    const int rel = target[j] - (g.col0 + cur.a0 + arow + 4 * lh);
                    const int end = live ? g.na - (cur.a0 + arow + 4 * lh) : 0;     // columns of the piece from here on
                    auto grad = [&](int i, int q) __attribute__((always_inline)) {
                        const int v = 32 * i + 8 * (q / 4) + q % 4;
                        float p = exp_from(acc[i][j][q], st.x);
                        p = v == rel ? st.y : p;
                        return v < end ? p : 0.f;
                    };
                    auto to = [&](int r) { return static_cast<uint16_t*>(g.out) + (row0 + r) * g.ldo + cur.a0 + arow; };
                    store16(j, grad, to, nv, as_bf16);
                    if (parts)
                        store16(j, [&](int i, int q) __attribute__((always_inline)) { return bf16_rest(grad(i, q)); },
                                [&](int r) { return to(r) + kFewRows * g.ldo; }, nv, as_bf16);
                } else if (OUT == ROWS || direct) {
                    if (cur.a0 + arow >= g.na) break;      // (columns come in multiples of 64)
                    store16(j, [&](int i, int q) __attribute__((always_inline)) { return acc[i][j][q] * coef; },
                            [&](int r) {
                                const int64_t to = g.rows && r < nv ? g.rows[row0 + r] : row0 + r;
                                return static_cast<uint16_t*>(direct ? g.direct : g.out) + to * g.ldo + cur.a0 + arow;
                            }, nv, as_bf16);
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
                            if (8 * k >= nv) break;
                            ++stored;
                            const int r = 8 * k + lane / 8, v = lane % 8;
                            f32x4 d = *reinterpret_cast<const f32x4*>(tb + at(r, v));
                            if (r < nv && OUT == ROWS32) {
                                const int64_t to = g.rows ? g.rows[row0 + r] : row0 + r;
                                *reinterpret_cast<f32x4*>(static_cast<float*>(g.out) + to * g.ldo + col + 4 * v) = d * coef;
                            } else if (r < nv) {
                                float* const p = static_cast<float*>(g.out) + cur.sp * split_stride +
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
        wid += per_xcd;
        if (wid >= wend) break;
    }
    wait_vm<0>();                             // (the last pairs' loads land before the LDS is another's)
}

// rows[0 .. n): the indices t < T whose key is not `skip`, in order, and the
// last of them again up to a whole reduction chunk; head: {n, n rounded up to
// whole chunks, 0}.  One workgroup of kListThreads: the list is a running count over the call.
// A thread takes 16 bytes of keys at a time, so that 4096 fp32-sized keys are
// one round of loads and one scan.
constexpr int kListThreads = 1024;
template <typename Key>
__device__ __forceinline__ void list_rows(const Key* __restrict__ key, int T, Key skip, int32_t* rows, int32_t* head) {
    constexpr int NW = kListThreads / kWave, N = 16 / sizeof(Key);
    __shared__ int cnt[2][NW];
    __shared__ int lastrow;
    const int lane = lane_id(), wave = threadIdx.x / kWave;
    const bool wide = reinterpret_cast<uintptr_t>(key) % 16 == 0;
    int base = 0, flip = 0;
    for (int t0 = 0; t0 < T; t0 += kListThreads * N, flip ^= 1) {
        const int t = t0 + threadIdx.x * N;
        alignas(16) Key k[N];
        if (wide && t + N <= T) {
            *reinterpret_cast<uint4*>(k) = *reinterpret_cast<const uint4*>(key + t);
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) k[i] = t + i < T ? key[t + i] : skip;
        }
        int c = 0;
#pragma unroll
        for (int i = 0; i < N; ++i) c += k[i] != skip;
        const int upto = wave_scan(c);
        if (lane == kWave - 1) cnt[flip][wave] = upto;
        __syncthreads();               // (the other half of cnt was last read before the round before's barrier)
        int sum = wave_scan(lane < NW ? cnt[flip][lane] : 0);
        const int total = __builtin_amdgcn_readlane(sum, NW - 1);
        int at = base + upto - c + (wave ? __builtin_amdgcn_readlane(sum, wave - 1) : 0);
        base += total;
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (k[i] != skip) {
                rows[at] = t + i;
                if (++at == base) lastrow = t + i;
            }
    }
    __syncthreads();
    const int pad = (base + kBK - 1) / kBK * kBK;
    for (int i = base + threadIdx.x; i < pad; i += kListThreads) rows[i] = lastrow;
    if (threadIdx.x == 0) {
        head[0] = base;
        head[1] = pad;
        head[2] = 0;
    }
}
template <typename Key>
__global__ __launch_bounds__(kListThreads) void list_kernel(const Key* __restrict__ key, int T, Key skip, int32_t* rows,
                                                            int32_t* head) {
    list_rows(key, T, skip, rows, head);
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
template <class C, bool ACOLS, bool BCOLS, int OUT, int FOLD = WHOLE, bool GATHER = false>
hipError_t launch_gemm(GemmArgs g, hipStream_t s) {
    constexpr int kRows = (FOLD == GROUPS && BCOLS) || FOLD == PLANES ? 64 : C::NB;
    g.xcds = geometry().xcds;
    const int64_t work = static_cast<int64_t>((g.na + C::NA - 1) / C::NA) * ((g.nb + kRows - 1) / kRows) *
                         (g.splits ? g.splits : std::max(1, std::min(kMostSlices, g.slice_chunks / 4)));
    if (work == 0) return hipSuccess;
    int64_t blocks = std::min<int64_t>(work, geometry().cus);
    blocks = std::max<int64_t>(g.xcds, (blocks + g.xcds - 1) / g.xcds * g.xcds);
    loss_gemm<C, ACOLS, BCOLS, OUT, FOLD, GATHER><<<static_cast<int>(blocks), C::kThreads, 0, s>>>(g);
    return hipGetLastError();
}

}  // namespace
}  // namespace eat
