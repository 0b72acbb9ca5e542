"""The addresses that the losses' GEMM loads from, on the CPU.

Operands go to LDS by loads the compiler does not see through, along a stream
that runs on over a workgroup's items, so an address that is off would fault
the GPU.  The parts of csrc/loss_gemm.h that choose the addresses (the tile
table, Operand, the item order and the load stream) are compiled here with g++ as
they stand, the loads themselves replaced by a check, and run for every
workgroup, wave and lane of a launch: each 16 bytes must lie in the operands'
buffers and each LDS block in the ring.
"""
import os
import re
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "paper_2609_33614_amd", "csrc", "loss_gemm.h")

PRELUDE = r"""
#include <algorithm>
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <type_traits>
#include <vector>
#define __device__
#define __forceinline__ inline
#define __builtin_amdgcn_readfirstlane(x) (x)
using std::max; using std::min;
struct Dim { int x; };
static Dim blockIdx, threadIdx, gridDim;
struct float2 { float x, y; };
constexpr int kWave = 64, kBK = 64;
inline int lane_id() { return threadIdx.x % 64; }
inline int wave_id() { return threadIdx.x / 64; }
inline uint64_t uniform(uint64_t v) { return v; }
static void fail(const char* what, uint64_t v) {
    printf("BAD %s %llx block %d thread %d\n", what, (unsigned long long)v, blockIdx.x, threadIdx.x);
    exit(1);
}
inline uint32_t __umul24(uint32_t a, uint32_t b) {
    if (a >> 24 || b >> 24) fail("24-bit product", a);
    return a * b;
}
static uint64_t lo[2], hi[2];
static uint32_t ring_end;
static long loads;
static void note(uint64_t p, uint32_t lds) {
    ++loads;
    bool ok = false;
    for (int i = 0; i < 2; ++i) ok |= p >= lo[i] && p + 16 <= hi[i];
    if (!ok || p % 16) fail("load", p);
    if (lds + 1024 > ring_end) fail("ring block", lds);
}
"""

KERNEL = r"""
template <class C, bool ACOLS, bool BCOLS, int OUT, int FOLD = WHOLE, bool GATHER = false>
void stream(GemmArgs g) {
%(consts)s
    uint8_t* const ring = nullptr;
%(items)s
    const int wave = wave_id();
%(stream)s
%(prologue)s
    for (; wid < wend; wid += per_xcd) {
        const Item cur = item_at(wid);
        const int nch = slice(cur.sp + 1) - slice(cur.sp);
        for (int c = 0; c < nch; ++c) {
            next_pair();
            pair_slots();
            for (int q = 0; q < C::kLA + C::kLB; ++q) pair_load(q);
            looked_up();
        }
    }
}

template <class C, bool ACOLS, bool BCOLS, int OUT, int FOLD = WHOLE, bool GATHER = false>
long launch(GemmArgs g, uint64_t a_bytes, uint64_t b_bytes) {
    constexpr int kRows = (FOLD == GROUPS && BCOLS) || FOLD == PLANES ? 64 : C::NB;
    g.xcds = 8;
    const long work = (long)((g.na + C::NA - 1) / C::NA) * ((g.nb + kRows - 1) / kRows) * (g.splits ? g.splits : kCus);
    if (!work) return 0;
    const long blocks = max<long>(8, (min<long>(work, 256) + 7) / 8 * 8);
    lo[0] = (uint64_t)g.a; hi[0] = lo[0] + a_bytes;
    lo[1] = (uint64_t)g.b; hi[1] = lo[1] + b_bytes;
    ring_end = C::SLOTS * C::kSlot;
    gridDim.x = (int)blocks;
    loads = 0;
    for (blockIdx.x = 0; blockIdx.x < blocks; ++blockIdx.x)
        for (threadIdx.x = 0; threadIdx.x < C::kThreads; ++threadIdx.x) stream<C, ACOLS, BCOLS, OUT, FOLD, GATHER>(g);
    return loads;
}

static const uint16_t* const A = (const uint16_t*)0x100000000000ull;
static const uint16_t* const B = (const uint16_t*)0x300000000000ull;

// the launches of one cross-entropy call of n counted rows out of T
template <class C>
void ce(int T, int n, int d, int V, int rows_pad, int piece, int pool) {
    int32_t head[4] = {n, (n + 63) / 64 * 64, 0, 0}, slices = 0;
    GemmArgs z{};
    z.a = A; z.lda = d; z.na = V; z.b = B; z.ldb = d; z.nb = T; z.nb_dev = head; z.K = d; z.splits = 1;
    long total = launch<C, false, false, LSE>(z, 2ull * V * d, 2ull * rows_pad * d);
    for (int v0 = 0; v0 < V; v0 += piece) {
        const int nv = min(piece, V - v0);
        GemmArgs a{};
        a.a = A; a.lda = d; a.na = d; a.a_rows = nv; a.b = B; a.ldb = piece; a.nb = T; a.nb_dev = head; a.K = nv;
        a.pool_rows = pool; a.slice_chunks = min(piece, V + 63) / 64; a.slices_out = &slices;
        // (Small: G and h in two planes, the larger tiles)
        constexpr bool kSmall = C::NB == 64;
        const int planes = kSmall ? 2 : 1;
        if constexpr (kSmall) total += launch<Mid, true, false, PART, PLANES>(a, 2ull * nv * d, 4ull * rows_pad * piece);
        else total += launch<C, true, false, PART>(a, 2ull * nv * d, 2ull * rows_pad * piece);
        GemmArgs w{};
        w.a = A; w.lda = d; w.na = d; w.a_rows = 1 << 30; w.b = B; w.ldb = piece; w.nb = nv;
        w.K = rows_pad * planes; w.k_dev = head + 1; w.k_times = planes; w.splits = 1;
        using W = std::conditional_t<kSmall, Mid, C>;
        total += launch<W, true, true, ROWS>(w, 2ull * planes * rows_pad * d, 2ull * planes * rows_pad * piece);
        if constexpr (kSmall) total += launch<Big, true, true, ROWS>(w, 4ull * rows_pad * d, 4ull * rows_pad * piece);
    }
    printf("ce T %d n %d d %d V %d: %ld loads\n", T, n, d, V, total);
}

// the products of one balance call of n valid tokens out of T, x in `parts` parts
void balance(int T, int n, int E, int d, int splits, bool gather, int parts, int segs, int map) {
    const int groups = (E + 63) / 64, pad = (T + 255) / 256 * 256, padn = (n + 63) / 64 * 64;
    int32_t head[3] = {n, padn, 0};
    std::vector<int32_t> rows(pad, 1 << 30);
    for (int i = 0; i < padn; ++i) rows[i] = n ? (int)((long)min(i, n - 1) * T / n) : 0;
    GemmArgs g{};
    g.a = A; g.lda = g.na = parts * d; g.a_rows = parts == 1 ? T : 1 << 30; g.k_rows = rows.data();
    g.b = B; g.ldb = 256 * groups; g.nb = E; g.K = (T + 63) / 64 * 64; g.k_dev = head + 1; g.k_times = 1;
    g.splits = splits;
    const uint64_t a_bytes = parts == 1 ? 2ull * T * d : 2ull * pad * parts * d, b_bytes = 512ull * pad * groups;
    long total = gather ? launch<Big, true, true, PART, GROUPS, true>(g, a_bytes, b_bytes)
                        : launch<Big, true, true, PART, GROUPS, false>(g, a_bytes, b_bytes);
    GemmArgs x{};
    x.segs = segs; x.map = map; x.K = x.a_rows = groups * segs * 64; x.a = A; x.lda = x.na = d;
    x.b = B; x.ldb = 256 * groups; x.nb = T; x.nb_dev = head; x.splits = 1;
    total += launch<Big, true, false, ROWS, GROUPS>(x, 2ull * x.K * d, b_bytes);
    printf("balance T %d n %d E %d d %d: %ld loads\n", T, n, E, d, total);
}

int main() {
%(calls)s
    puts("ALL IN BOUNDS");
}
"""


def program(calls: str, header: str = None) -> str:
    """C++ source that makes ``calls`` (of ce<Tile>(...) and balance(...))."""
    s = header if header is not None else open(HEADER).read()

    def cut(begin, end):
        i = s.index(begin)
        return s[i:s.index(end, i)]

    operand = cut("// Loads of one operand's part of a chunk", "// The operand fragment of indices")
    operand = re.sub(r'asm volatile\("s_add_u32 m0, %1.*?;', "note(p, lds + 1024 * WAVES * j);", operand, flags=re.S)
    operand = re.sub(r'asm volatile\("s_add_u32 m0, %2.*?;', "note(from + o, lds + 1024 * WAVES * j);", operand, flags=re.S)
    assert operand.count("note(") == 2 and "asm volatile" not in operand
    parts = {
        "consts": cut("    constexpr bool kGroupTile =", "    __shared__ __attribute__((aligned(1024))) uint8_t ring"),
        "items": cut("    const int nb = g.nb_dev ?", "    const int lane = lane_id(), wave = wave_id();"),
        "stream": cut("    auto slice = [&](int sp)", "    // Waits until at most the loads of the parts behind"),
        "prologue": cut("    next_a();\n    if (", "    int slot0 = 0;"),
        "calls": calls,
    }
    kernel = KERNEL
    for k, v in parts.items():
        kernel = kernel.replace(f"%({k})s", v)
    return (PRELUDE + cut("template <int NA_, int NB_, int WA_, int WB_>\nstruct Tile", "enum Out {")
            + cut("enum Out {", "// (uniform: what depends on it")
            + cut("__device__ __forceinline__ int swz_row", "__device__ __forceinline__ uint64_t uniform")
            + operand + cut("enum Fold {", "template <class C") + cut("struct Item {", "// The reference of a row's exponentials") + kernel)


def run(tmp_path, calls: str, header: str = None):
    """(exit status, output) of the program."""
    src, exe = str(tmp_path / "loads.cpp"), str(tmp_path / "loads")
    open(src, "w").write(program(calls, header))
    subprocess.run(["g++", "-O2", "-std=c++17", "-w", src, "-o", exe], check=True)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    return r.returncode, r.stdout
