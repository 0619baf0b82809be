// Product of 8-bit matrices under power-of-two block scales, on gfx950's scaled matrix instructions.
//
//   C[m, n] = sum over blocks b of 2^(ea[m, b] + ew[n, b]) * sum over the block's 128 k of a[m, k] w[n, k]      in float32, rounded to bf16
//
// v_mfma_scale_f32_16x16x128_f8f6f4 takes 128 k of 16 rows of either operand, a whole block, and a scale byte for each row, so the scales
// cost no instruction of their own but the reads that bring them.
//
// A workgroup of 4 waves owns a BM x BN tile and a slice of K, and walks it in slabs of 128 k: rows of 128 bytes, which go straight into
// LDS (buffer_load ... lds: no staging registers), the 16-byte chunks XOR-swizzled by the row so that no bank conflicts arise.  Slabs go in
// half slabs - the rows that one half of every wave's tile needs of A, and one half of W - through a ring of NS of them.  All fragments
// of a half slab are in registers before its products begin, so a place is free again half a slab after it was waited for; one
// barrier per half slab waits for the one that is needed next, never for all loads in flight.  Scale bytes lie [block][row], so those of
// a tile are a few hundred bytes side by side for each slab; each wave fetches one slab's of the next four.
//
// Measured, us: 2048 x 55296 x 5120 443 to 463 (2.5 to 2.6 PFLOP/s: the matrix pipe is busy 68 % of the time at 1.6 GHz, the clock under these
// operands), 96 x 55296 x 5120 53 (5.3 TB/s), 573 x 3584 x 18944 in six slices 43 and 8 for their sums.
#include <algorithm>
#include <type_traits>

#include "fp8.h"

namespace {

typedef __attribute__((ext_vector_type(8))) int i32x8;
typedef __attribute__((ext_vector_type(4))) int i32x4;
typedef f32x4 f32x4_a4 __attribute__((aligned(4)));   // the caller's rows are aligned to their elements only
typedef u32x4 u32x4_a2 __attribute__((aligned(2)));

constexpr int CHUNKS = FP8_BLOCK / 16;   // 16-byte chunks of a row of a slab
constexpr int NUM_XCD = 8;
constexpr int GROUP_M = 8;

struct Fp8Args {
    const unsigned char *A, *As, *W, *Ws;   // codes and scale bytes
    int a_pitch, w_pitch;                   // rows of the scales
    int M, N, K, split, per, tiles_m, tiles_n;
    bf16_t* out;
    float* partial;                         // [split][M][N] where split > 1
};

// x / d of a uniform x >= 0, off by one at most below 2^23 before the correction.
__device__ __forceinline__ int fast_div(int x, int d) {
    const int q = (int)((float)x * __builtin_amdgcn_rcpf((float)d));
    const int r = x - q * d;
    return __builtin_amdgcn_readfirstlane(q + (r >= d ? 1 : 0) - (r < 0 ? 1 : 0));
}

// Workgroup -> (row tile, column tile, K slice): each of the 8 XCDs, to which workgroups are dealt in turn, gets a contiguous range of
// tiles, walked M-fastest in groups of 8 row tiles, so that the workgroups that share a weight panel share an L2.
struct Tile { int tm, tn, ks; };
__device__ __forceinline__ Tile tile_of(int bid, const Fp8Args& g) {
    const int total = g.tiles_m * g.tiles_n * g.split, q = total / NUM_XCD, r = total % NUM_XCD, xcd = bid % NUM_XCD;
    const int lin = xcd * q + (xcd < r ? xcd : r) + bid / NUM_XCD, slice = g.tiles_m * g.tiles_n;
    Tile c;
    c.ks = g.split == 1 ? 0 : fast_div(lin, slice);
    const int t = lin - c.ks * slice;
    if (g.tiles_m == 1) {
        c.tm = 0;
        c.tn = t;
        return c;
    }
    const int size = GROUP_M * g.tiles_n, grp = fast_div(t, size), first = grp * GROUP_M;
    const int gm = g.tiles_m - first < GROUP_M ? g.tiles_m - first : GROUP_M, in = t - grp * size;
    c.tn = fast_div(in, gm);
    c.tm = first + in - c.tn * gm;
    return c;
}

template <int BM, int BN, int WM, int WN>
struct Shape {
    static constexpr int WTM = BM / WM, WTN = BN / WN;                   // wave tile
    static constexpr int MI = WTM / 16, NI = WTN / 16;
    static constexpr int HA = BM / 2, HB = BN / 2;                       // rows of a half slab
    static constexpr int QA = HA / 4, QB = HB / 4;                       // rows that one wave loads
    static constexpr int LA = QA / 8, LB = QB / 8;                       // load instructions of a wave: 8 rows of 128 bytes
    static constexpr int LOADS = LA + LB;
    static constexpr int SLOT = (HA + HB) * FP8_BLOCK;                   // bytes
    static constexpr bool TWO = BM * BN <= 128 * 128;                    // two workgroups on a compute unit
    static constexpr int SCALES = 2 * 4 * 512;                           // two groups of four slabs: 256 rows of A, 256 of W
    static constexpr int CAP = (TWO ? 80 : 160) * 1024 - SCALES;
    static constexpr int NS = CAP / SLOT < 6 ? CAP / SLOT : 6;           // half slabs in LDS
    static constexpr int LDS = SCALES + NS * SLOT;
    static_assert(WM * WN == 4 && QA % 8 == 0 && QB % 8 == 0 && NS >= 3, "four waves load whole groups of rows");
    static_assert((WTM / 2) % 16 == 0 && (WTN / 2) % 32 == 0, "halves of whole sub-tiles, pairs of columns");
    static_assert((WTM / 2) % QA == 0 && (WTN / 2) % QB == 0, "the rows that a wave loads lie in one wave tile");
};

// LDS rows are 128 bytes; chunk c of row r is stored at chunk position c ^ key: the 16 rows of a fragment have, two by two, 8 different
// keys.  Fragment row i of sub-tile s is row 16 s + i of A, and row 32 (s / 2) + 8 (i / 4) + 4 (s % 2) + i % 4 of W: a lane, which
// holds columns 4 q .. 4 q + 3 of a sub-tile of the product, then has eight neighbouring columns in two of them.
__device__ __forceinline__ int key_a(int row) { return (row >> 1) & 7; }
__device__ __forceinline__ int key_w(int row) { return ((row >> 1) & 1) | (((row >> 3) & 3) << 1); }

// The matrix instructions are inline assembly: the builtin has separate accumulator operands in and out, and the register allocator
// fills the loop with moves between them.  The compiler therefore does not know the wait states round them:
//   * what else touches their accumulators: every accumulator passes through acc_fence before the loop and behind it;
//   * two behind a vector instruction that writes a code or a scale.  Codes come straight from LDS.  Scales are bytes, which the compiler
//     zero-extends with an instruction of its own, at the head of the loop for those that came over its end; so each is pinned as a whole
//     register at the end of the quadrant that reads it, two wait states before the next.  (Two in front of every matrix instruction
//     instead cost 1 to 3.5 %: 4096 x 3584 x 3584 49.6 -> 51.2 us, 2048 x 55296 x 5120 447 -> 452; like this 49.7 and 446.)
// That nothing else of the kind stands in the loops is looked up in the assembly by tests/test_matrix_asm_waits_host.py; run it, and the exact
// products on every tile, after a change of compiler or flags.
template <typename S>
__device__ __forceinline__ void acc_fence(f32x4 (&acc)[S::MI][S::NI]) {
    asm volatile("s_nop 15\n\ts_nop 15" ::: "memory");
#pragma unroll
    for (int mi = 0; mi < S::MI; ++mi)
#pragma unroll
        for (int ni = 0; ni < S::NI; ++ni) {
            if (S::TWO) asm volatile("" : "+v"(acc[mi][ni]));
            else asm volatile("" : "+a"(acc[mi][ni]));
        }
}

template <int V>
constexpr std::integral_constant<int, V> I{};

// all but the last N loads of this wave have landed and its LDS reads are done; so are the other waves'
template <int N>
__device__ __forceinline__ void dma_barrier() {
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

// Stores of a tile.  GUARD: it reaches past column N.
template <typename S, bool PARTIAL, bool GUARD>
__device__ __forceinline__ void store_tile(const f32x4 (&acc)[S::MI][S::NI], const Fp8Args& g, int ks, int row0, int col0) {
    // a lane holds columns 8 q .. 8 q + 7 of the 32 that two sub-tiles make; col0 counts them in
#pragma unroll
    for (int mi = 0; mi < S::MI; ++mi) {
        const int m = row0 + mi * 16;
        if (m >= g.M) continue;
#pragma unroll
        for (int j = 0; j < S::NI / 2; ++j) {
            const int n = col0 + 32 * j;
            const f32x4 lo = acc[mi][2 * j], hi = acc[mi][2 * j + 1];
            if constexpr (PARTIAL) {
                float* to = g.partial + ((size_t)ks * g.M + m) * g.N + n;
                if (!GUARD || n + 8 <= g.N) {
                    reinterpret_cast<f32x4_a4*>(to)[0] = lo;
                    reinterpret_cast<f32x4_a4*>(to)[1] = hi;
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        if (n + e < g.N) to[e] = e < 4 ? lo[e % 4] : hi[e % 4];
                }
            } else {
                bf16_t* to = g.out + (size_t)m * g.N + n;
                if (!GUARD || n + 8 <= g.N) {
                    *reinterpret_cast<u32x4_a2*>(to) = u32x4{pack_bf16x2(lo.x, lo.y), pack_bf16x2(lo.z, lo.w), pack_bf16x2(hi.x, hi.y), pack_bf16x2(hi.z, hi.w)};
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        if (n + e < g.N) to[e] = f32_to_bf16(e < 4 ? lo[e % 4] : hi[e % 4]);
                }
            }
        }
    }
}

// STREAM: nobody else reads this tile's weights (a single row tile), they bypass the caches.
template <int BM, int BN, int WM, int WN, bool PARTIAL, bool STREAM>
__device__ __forceinline__ void gemm_tile(const Fp8Args& g, unsigned char* smem) {
    using S = Shape<BM, BN, WM, WN>;
    constexpr int MH = S::MI / 2, NH = S::NI / 2, NS = S::NS;
    const int K = g.K;
    const Tile tc = tile_of(blockIdx.x, g);
    const int m0 = tc.tm * BM, n0 = tc.tn * BN, blocks = K / FP8_BLOCK;
    const int b0 = tc.ks * g.per, KT = b0 + g.per < blocks ? g.per : blocks - b0;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave / WN, wn = wave % WN, lrow = lane & 15, lk = lane >> 4;

    auto rsrc = [&](const unsigned char* base, unsigned bytes) {
        const unsigned long long p = reinterpret_cast<unsigned long long>(base);
        return i32x4{__builtin_amdgcn_readfirstlane((int)(unsigned)p), __builtin_amdgcn_readfirstlane((int)(p >> 32)),
                     __builtin_amdgcn_readfirstlane((int)bytes), 0x00020000};
    };
    // Rows past the last one lie behind their descriptor's end: no request is made for them, and zeros arrive.
    const int rows_a = g.M - m0 < BM ? g.M - m0 : BM, rows_w = g.N - n0 < BN ? g.N - n0 : BN;
    i32x4 ra = rsrc(g.A + (size_t)m0 * K, (unsigned)rows_a * (unsigned)K), rb = rsrc(g.W + (size_t)n0 * K, (unsigned)rows_w * (unsigned)K);
    const int a_bytes = ra[2], b_bytes = rb[2];
    // scales of this slice's blocks from the tile's first row on, cut to the array's end
    auto scale_rsrc = [&](const unsigned char* base, int pitch, int first) {
        const size_t at = (size_t)b0 * pitch + first, end = (size_t)blocks * pitch, left = end - at;
        return rsrc(base + at, (unsigned)(left < 0x7fffffffu ? left : 0x7fffffffu));
    };
    const i32x4 rsa = scale_rsrc(g.As, g.a_pitch, m0), rsb = scale_rsrc(g.Ws, g.w_pitch, n0);
    // offsets of a lane's chunks: half slab row x -> tile row (x / (WT / 2)) * WT + half * WT / 2 + x % (WT / 2)
    unsigned va[2][S::LA], vb[2][S::LB];
    {
        const int qa = wave * S::QA, qb = wave * S::QB;
        const int ta = qa / (S::WTM / 2) * S::WTM + qa % (S::WTM / 2), tb = qb / (S::WTN / 2) * S::WTN + qb % (S::WTN / 2);
        const int r = lane >> 3, c = lane & 7;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
#pragma unroll
            for (int i = 0; i < S::LA; ++i)
                va[h][i] = (unsigned)(ta + h * S::WTM / 2 + 8 * i + r) * (unsigned)K + (c ^ key_a(qa + 8 * i + r)) * 16 + (unsigned)b0 * FP8_BLOCK;
#pragma unroll
            for (int i = 0; i < S::LB; ++i)
                vb[h][i] = (unsigned)(tb + h * S::WTN / 2 + 8 * i + r) * (unsigned)K + (c ^ key_w(qb + 8 * i + r)) * 16 + (unsigned)b0 * FP8_BLOCK;
        }
    }
    const unsigned lds0 = (unsigned)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)smem;
    const unsigned lds_a = lds0 + S::SCALES + wave * S::QA * 128, lds_b = lds0 + S::SCALES + S::HA * 128 + wave * S::QB * 128;
    // load i of a half slab (A rows ha, W rows hb) into the slot at byte `slot`
    auto dma = [&](int i, int ha, int hb, unsigned slot, int koff) {
        if (i < S::LA) {
            asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds"
                         ::"s"(lds_a + slot + i * 1024), "v"(va[ha][i]), "s"(ra), "s"(koff));
            return;
        }
        const int j = i - S::LA;
        if (STREAM)
            asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen nt lds"
                         ::"s"(lds_b + slot + j * 1024), "v"(vb[hb][j]), "s"(rb), "s"(koff));
        else
            asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds"
                         ::"s"(lds_b + slot + j * 1024), "v"(vb[hb][j]), "s"(rb), "s"(koff));
    };
    // this wave's slab of scales among the four from `first` on: 256 rows of A and of W, four a lane; slabs past the last one bring bytes
    // that nothing uses
    auto scale_dma = [&](int first) {
        const int kt = first + wave;
        const unsigned to = lds0 + (unsigned)(first >> 2 & 1) * 2048u + wave * 512u;
        // in the lane's offset, which the descriptor's bound sees: the last block's may reach past the array
        const unsigned at_a = (unsigned)kt * (unsigned)g.a_pitch + lane * 4, at_w = (unsigned)kt * (unsigned)g.w_pitch + lane * 4;
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, 0 offen lds" ::"s"(to), "v"(at_a), "s"(rsa));
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, 0 offen lds" ::"s"(to + 256u), "v"(at_w), "s"(rsb));
    };

    f32x4 acc[S::MI][S::NI];
#pragma unroll
    for (int mi = 0; mi < S::MI; ++mi)
#pragma unroll
        for (int ni = 0; ni < S::NI; ++ni) acc[mi][ni] = f32x4{0.f, 0.f, 0.f, 0.f};
    i32x8 fa[S::MI], fb[S::NI];
    int ea[S::MI], eb[S::NI];
    const u32x4* L = reinterpret_cast<const u32x4*>(smem + S::SCALES);
    const int key = (lrow >> 1) & 7, w_row = 8 * (lrow >> 2) + (lrow & 3);   // both keys of fragment row lrow are this one
    const int src_a = (wm * (S::WTM / 2) + lrow) * CHUNKS, src_b = (S::HA + wn * (S::WTN / 2) + w_row) * CHUNKS;
    const unsigned char *scale_a = smem + wm * S::WTM + lrow, *scale_b = smem + 256 + wn * S::WTN + w_row;
    auto scale_at = [](int kt) { return (kt >> 2 & 1) * 2048 + (kt & 3) * 512; };
    auto put = [](i32x8& f, int half, u32x4 x) {
#pragma unroll
        for (int e = 0; e < 4; ++e) f[4 * half + e] = (int)x[e];
    };
    // read i of half h of A (W): 2 MH (2 NH) chunks, then the scales.  Which 32 of a block's k a lane holds does not matter, as long as both
    // operands agree: chunks lk and lk + 4.
    auto read_a = [&](int h, int i, unsigned slot, int kt) {
        if (i < 2 * MH) put(fa[h * MH + i / 2], i & 1, L[slot / 16 + src_a + i / 2 * 16 * CHUNKS + ((lk + (i & 1) * 4) ^ key)]);
        else ea[h * MH + i - 2 * MH] = scale_a[scale_at(kt) + h * (S::WTM / 2) + (i - 2 * MH) * 16];
    };
    auto read_b = [&](int h, int i, unsigned slot, int kt) {
        const int ni = i < 2 * NH ? i / 2 : i - 2 * NH, row = ni / 2 * 32 + ni % 2 * 4;
        if (i < 2 * NH) put(fb[h * NH + ni], i & 1, L[slot / 16 + src_b + row * CHUNKS + ((lk + (i & 1) * 4) ^ key)]);
        else eb[h * NH + ni] = scale_b[scale_at(kt) + h * (S::WTN / 2) + row];
    };

    // Products of a slab: four quadrants of the wave's tile, each with one new half of A or W:
    //   even slabs   A0W0 | read W1,  A0W1 | read A1,  A1W1 | read the next slab's A0,  A1W0 | read its W1
    //   odd slabs    A0W1 | read W0,  A0W0 | read A1,  A1W0 | read the next slab's A0,  A1W1 | read its W0
    // Half slab p is what quadrants 2p - 2 and 2p - 1 read: A half p % 2 and W half (p ^ (p >> 1)) & 1 of slab p / 2.  While
    // half slab p is multiplied, p + 1 is read and p + NS is loaded into the place of p.
    // Slabs past the last one are loaded from descriptors of no bytes, which takes no request.
    auto until = [&](int k) {
        ra[2] = k < KT ? a_bytes : 0;
        rb[2] = k < KT ? b_bytes : 0;
        return (k < KT ? k : KT - 1) * FP8_BLOCK;
    };
    scale_dma(0);
#pragma unroll
    for (int p = 0; p < NS; ++p) {
        const int koff = until(p / 2);
#pragma unroll
        for (int i = 0; i < S::LOADS; ++i) dma(i, p & 1, (p ^ (p >> 1)) & 1, p * S::SLOT, koff);
    }
    dma_barrier<(NS - 1) * S::LOADS>();
#pragma unroll
    for (int i = 0; i < 3 * MH; ++i) read_a(0, i, 0, 0);
#pragma unroll
    for (int i = 0; i < 3 * NH; ++i) read_b(0, i, 0, 0);
    acc_fence<S>(acc);
    dma_barrier<(NS - 2) * S::LOADS>();

    unsigned rd = S::SLOT, wr = 0;   // places of half slabs p + 1 and p
    // One quadrant: rows half ma times columns half nb.  Spread over the first three quarters of its matrix instructions, so that the
    // barrier finds the reads done: the fragments of half rh of A or W of slab kt, and loads [l0, l1) of half slab p + NS.
    auto quadrant = [&](auto ma, auto nb, auto rd_a, auto rh, int kt, auto l0, auto l1, auto ha, auto hb, int koff) {
        constexpr int NM = MH * NH, SPAN = (NM * 3 + 3) / 4;
        constexpr int NR = rd_a() ? 3 * MH : 3 * NH, NL = l1() - l0(), OPS = NR + NL;
#pragma unroll
        for (int i = 0; i < NM; ++i) {
            const int nr = i / MH, mi = ma() * MH + (nr & 1 ? MH - 1 - i % MH : i % MH), ni = nb() * NH + nr;
            if (S::TWO)
                asm volatile("v_mfma_scale_f32_16x16x128_f8f6f4 %0, %1, %2, %0, %3, %4 op_sel_hi:[0,0,0]"
                             : "+v"(acc[mi][ni]) : "v"(fb[ni]), "v"(fa[mi]), "v"(eb[ni]), "v"(ea[mi]));
            else
                asm volatile("v_mfma_scale_f32_16x16x128_f8f6f4 %0, %1, %2, %0, %3, %4 op_sel_hi:[0,0,0]"
                             : "+a"(acc[mi][ni]) : "v"(fb[ni]), "v"(fa[mi]), "v"(eb[ni]), "v"(ea[mi]));
            const int j0 = i < SPAN ? i * OPS / SPAN : OPS, j1 = i + 1 < SPAN ? (i + 1) * OPS / SPAN : OPS;
#pragma unroll
            for (int j = j0; j < j1; ++j) {
                const int nl = j * NL / OPS;   // loads among the operations before j
                if ((j + 1) * NL / OPS > nl) dma(l0() + nl, ha(), hb(), wr, koff);
                else if (rd_a()) read_a(rh(), j - nl, rd, kt);
                else read_b(rh(), j - nl, rd, kt);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int i = 0; i < (rd_a() ? MH : NH); ++i) asm volatile("" : "+v"(rd_a() ? ea[rh() * MH + i] : eb[rh() * NH + i]));
        asm volatile("s_nop 1");
    };
    auto half_end = [&]() {
        dma_barrier<(NS - 2) * S::LOADS>();
        __builtin_amdgcn_sched_barrier(0);
        wr = rd;
        rd = rd + S::SLOT == NS * S::SLOT ? 0u : rd + S::SLOT;
        asm volatile("" : "+s"(rd), "+s"(wr));   // one address per operand, not one for every place of the ring
    };
    auto slab = [&](auto parity, int kt) {
        constexpr int B = decltype(parity)::value;   // the columns half this slab begins with
        constexpr int P0 = 2 * B, P1 = 2 * B + 1;    // p modulo 4
        constexpr int N0 = (P0 + NS) & 3, N1 = (P1 + NS) & 3, H0 = (N0 ^ (N0 >> 1)) & 1, H1 = (N1 ^ (N1 >> 1)) & 1;
        constexpr int LH = S::LOADS / 2;
        // scales: four slabs ahead of their first use at the least, three and a half behind the last one of those they replace
        if (B == 0 && (kt & 3) == 0 && kt + 4 < KT) scale_dma(kt + 4);
        const int o0 = until(kt + NS / 2);           // half slab p + NS lies in slab (p + NS) / 2
        quadrant(I<0>, I<B>, I<0>, I<B ^ 1>, kt, I<0>, I<LH>, I<(N0 & 1)>, I<H0>, o0);
        quadrant(I<0>, I<B ^ 1>, I<1>, I<1>, kt, I<LH>, I<S::LOADS>, I<(N0 & 1)>, I<H0>, o0);
        half_end();
        const int o1 = until(kt + (1 + NS) / 2);
        quadrant(I<1>, I<B ^ 1>, I<1>, I<0>, kt + 1, I<0>, I<LH>, I<(N1 & 1)>, I<H1>, o1);
        quadrant(I<1>, I<B>, I<0>, I<B ^ 1>, kt + 1, I<LH>, I<S::LOADS>, I<(N1 & 1)>, I<H1>, o1);
        half_end();
    };
    for (int kt = 0;;) {
        slab(I<0>, kt);
        if (++kt >= KT) break;
        slab(I<1>, kt);
        if (++kt >= KT) break;
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // no load may land after this workgroup's LDS is another's
    acc_fence<S>(acc);
    const int row0 = m0 + wm * S::WTM + lrow, col0 = n0 + wn * S::WTN + 8 * lk;
    if (__builtin_expect(n0 + BN > g.N, 0)) store_tile<S, PARTIAL, true>(acc, g, tc.ks, row0, col0);
    else store_tile<S, PARTIAL, false>(acc, g, tc.ks, row0, col0);
}

template <int BM, int BN, int WM, int WN, bool PARTIAL, bool STREAM>
__global__ __launch_bounds__(256, (Shape<BM, BN, WM, WN>::TWO ? 2 : 1)) void gemm_fp8_kernel(const Fp8Args g) {
    extern __shared__ __align__(16) unsigned char smem[];
    gemm_tile<BM, BN, WM, WN, PARTIAL, STREAM>(g, smem);
}

// ------------------------------------------------------------------ up to 16 rows
// Weights that one launch's latency outweighs.  Nothing is staged: a wave takes 16 columns and up to U blocks of 128 k, 2 KB of weights a block
// straight into the operand registers of one matrix instruction, all on their way before the first is used; the WAVES waves of a
// workgroup share the blocks and add up in LDS.  One launch, no partial results.  Lane (i, q) = (lane % 16, lane / 16) holds the 32 k from 32 q
// on of row i, on both sides.
// QUANT: the rows are bf16 and become codes on the way, in every workgroup again, which spares the launch that would do it once.
struct RowsArgs {
    const unsigned char *a, *a_scales;   // of codes
    const bf16_t* x;                     // of bf16 rows
    const unsigned char *w, *w_scales;
    bf16_t* out;
    int m, n, k, columns, a_pitch, w_pitch;
};

template <int WAVES, int U, bool QUANT>
__device__ __forceinline__ void rows_tile(const RowsArgs& g, f32x4 (*red)[64]) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), i = lane & 15, q = lane >> 4;
    const int n0 = blockIdx.x * 16, blocks = g.columns / FP8_BLOCK, mine = (blocks - wave + WAVES - 1) / WAVES;   // wave, wave + WAVES, ...
    // rows past the last one are the last one again: no request of their own, not stored
    const size_t row = i < g.m ? i : g.m - 1, col = n0 + i < g.n ? n0 + i : g.n - 1;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    if (mine > 0) {
        u32x4 w[U][2], a[U][QUANT ? 4 : 2];
        int ew[U], ea[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int b = wave + (u < mine ? u : mine - 1) * WAVES;   // past the end: the last block again, not used
            const u32x4* wp = reinterpret_cast<const u32x4*>(g.w + col * g.columns + (size_t)b * FP8_BLOCK + q * 32);
            w[u][0] = __builtin_nontemporal_load(wp);
            w[u][1] = __builtin_nontemporal_load(wp + 1);
            ew[u] = g.w_scales[(size_t)b * g.w_pitch + col];
            if constexpr (QUANT) {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int c = b * FP8_BLOCK + q * 32 + j * 8;
                    a[u][j] = *reinterpret_cast<const u32x4*>(g.x + row * g.k + (c < g.k ? c : 0));
                }
            } else {
                const u32x4* ap = reinterpret_cast<const u32x4*>(g.a + row * g.columns + (size_t)b * FP8_BLOCK + q * 32);
                a[u][0] = ap[0];
                a[u][1] = ap[1];
                ea[u] = g.a_scales[(size_t)b * g.a_pitch + row];
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            i32x8 fw, fa;
            if constexpr (QUANT) {
                unsigned top = 0;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if ((wave + u * WAVES) * FP8_BLOCK + q * 32 + j * 8 >= g.k) a[u][j] = u32x4{0u, 0u, 0u, 0u};   // zeros behind k
                    top = max(top, bf16_amax(a[u][j]));
                }
                if (__builtin_amdgcn_ballot_w64(top >= BF16_INF) != 0) {   // of the finite ones
                    top = 0;
#pragma unroll
                    for (int j = 0; j < 4; ++j) top = max(top, bf16_amax_finite(a[u][j]));
                }
                top = max(top, (unsigned)__shfl_xor((int)top, 16, 64));
                top = max(top, (unsigned)__shfl_xor((int)top, 32, 64));
                ea[u] = fp8_scale_byte(top);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const u32x2 c = fp8_codes_of(a[u][j], ea[u]);
                    fa[2 * j] = (int)c.x;
                    fa[2 * j + 1] = (int)c.y;
                }
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) fa[e] = (int)a[u][e / 4][e % 4];
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) fw[e] = (int)w[u][e / 4][e % 4];
            if (u < mine) acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fw, fa, acc, 0, 0, 0, ew[u], 0, ea[u]);
        }
    }
    red[wave][lane] = acc;
    __syncthreads();
    // lane (i, q) of the result: row i, columns 4 q .. 4 q + 3; the waves in order
    if (wave != 0 || i >= g.m) return;
#pragma unroll
    for (int v = 1; v < WAVES; ++v) acc += red[v][lane];
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (n0 + 4 * q + e < g.n) g.out[(size_t)i * g.n + n0 + 4 * q + e] = f32_to_bf16(acc[e]);
}

template <int WAVES, int U, bool QUANT>
__global__ __launch_bounds__(WAVES * 64) void fp8_rows_kernel(const RowsArgs g) {
    __shared__ f32x4 red[WAVES][64];
    rows_tile<WAVES, U, QUANT>(g, red);
}

// The slices' sums, in order, eight columns of the flattened result a thread.
__global__ __launch_bounds__(256) void fp8_sum_kernel(const float* __restrict__ partial, int split, long count, bf16_t* __restrict__ out) {
    const long i = ((long)blockIdx.x * 256 + threadIdx.x) * 8;
    if (i >= count) return;
    if (i + 8 <= count) {
        f32x4 lo = reinterpret_cast<const f32x4_a4*>(partial + i)[0], hi = reinterpret_cast<const f32x4_a4*>(partial + i)[1];
#pragma unroll 4
        for (int s = 1; s < split; ++s) {
            lo += reinterpret_cast<const f32x4_a4*>(partial + s * count + i)[0];
            hi += reinterpret_cast<const f32x4_a4*>(partial + s * count + i)[1];
        }
        *reinterpret_cast<u32x4_a2*>(out + i) = u32x4{pack_bf16x2(lo.x, lo.y), pack_bf16x2(lo.z, lo.w), pack_bf16x2(hi.x, hi.y), pack_bf16x2(hi.z, hi.w)};
        return;
    }
    for (long j = i; j < count; ++j) {
        float sum = partial[j];
        for (int s = 1; s < split; ++s) sum += partial[s * count + j];
        out[j] = f32_to_bf16(sum);
    }
}

template <int BM, int BN, int WM, int WN, bool PARTIAL, bool STREAM>
int launch(const Fp8Args& g, hipStream_t s) {
    auto kern = gemm_fp8_kernel<BM, BN, WM, WN, PARTIAL, STREAM>;
    constexpr int lds = Shape<BM, BN, WM, WN>::LDS;
    static bool attr_set = false;
    if (!attr_set) {   // per kernel; idempotent, so a race only repeats the call
        LAPS_HIP(hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, lds));
        attr_set = true;
    }
    hipLaunchKernelGGL(kern, dim3(g.tiles_m * g.tiles_n * g.split), dim3(256), lds, s, g);
    LAPS_LAUNCH_CHECK();
    return LAPS_OK;
}

template <int BM, int BN, int WM, int WN>
int launch_tile(const Fp8Args& g, hipStream_t s) {
    if (g.tiles_m == 1) return g.split > 1 ? launch<BM, BN, WM, WN, true, true>(g, s) : launch<BM, BN, WM, WN, false, true>(g, s);
    return g.split > 1 ? launch<BM, BN, WM, WN, true, false>(g, s) : launch<BM, BN, WM, WN, false, false>(g, s);
}

template <bool QUANT>
int launch_rows(const RowsArgs& g, hipStream_t s) {
    const int blocks = g.columns / FP8_BLOCK;
    const dim3 grid((g.n + 15) / 16);
    // As few waves as hold all blocks at once; 16 columns, 1 row, us (waves, blocks a wave): 512 x 256 2.0 (4, 1), 2.4 (16, 1); 1000 x 1024
    // 2.9 (8, 1), 3.3 (4, 2); 2048 x 2048 3.8 (16, 1), 4.9 (8, 4); 3584 x 3584 5.4 (16, 2), 5.6 (8, 4).
    if (blocks <= 4) hipLaunchKernelGGL((fp8_rows_kernel<4, 1, QUANT>), grid, dim3(256), 0, s, g);
    else if (blocks <= 8) hipLaunchKernelGGL((fp8_rows_kernel<8, 1, QUANT>), grid, dim3(512), 0, s, g);
    else if (blocks <= 16) hipLaunchKernelGGL((fp8_rows_kernel<16, 1, QUANT>), grid, dim3(1024), 0, s, g);
    else if (blocks <= 32) hipLaunchKernelGGL((fp8_rows_kernel<16, 2, QUANT>), grid, dim3(1024), 0, s, g);
    else {
        laps_set_error("gemm_fp8: %d blocks of k are too many for the kernel of few rows", blocks);
        return LAPS_EINVAL;
    }
    LAPS_LAUNCH_CHECK();
    return LAPS_OK;
}

// fill, slab: microseconds a workgroup takes besides its slabs, and for one; part: share of the slabs' time that goes away on an empty chip;
// pair: time of two workgroups on a compute unit over that of two alone (0: one fits); live: share of the slabs' time that rows of
// nothing spare.  Fitted, with the constants of laps_fp8_plan, to 6300 launches above 128 rows (15 weights from 512 x 12800 to 55296 x 5120, cold, at
// 15 row counts to 4096, every tile and up to 20 slices): 9 % rms; the plans are 1.5 % behind the best one measured in the mean, 15 of
// 223 products more than 10 % (573 x 7168 x 5120 41 us instead of 34).
struct TileDef {
    int bm, bn;
    float fill, slab, part, pair, live;
};
constexpr TileDef kTiles[] = {
    {64, 128, 2.00f, 0.395f, 0.18f, 0.86f, 0.01f},    // 0: 4 waves of 32 x 64
    {64, 256, 1.95f, 0.633f, 0.12f, 1.00f, 0.00f},    // 1: of 64 x 64; up to 64 rows only
    {128, 128, 2.57f, 0.486f, 0.20f, 1.00f, 0.00f},   // 2: of 64 x 64
    {128, 256, 4.68f, 0.860f, 0.29f, 0.00f, 0.00f},   // 3: of 128 x 64
    {192, 256, 6.56f, 1.026f, 0.21f, 0.00f, 0.07f},   // 4: of 96 x 128
    {256, 128, 5.12f, 0.792f, 0.16f, 0.00f, 0.26f},   // 5: of 128 x 64
    {256, 192, 6.77f, 1.027f, 0.16f, 0.00f, 0.20f},   // 6: of 64 x 192
    {256, 256, 8.56f, 1.273f, 0.19f, 0.00f, 0.15f},   // 7: of 128 x 128
    {16, 16, 0.f, 0.f, 0.f, 0.f, 0.f},                // 8: fp8_rows_kernel
};
constexpr int kNumTiles = sizeof(kTiles) / sizeof(kTiles[0]), kRowsCfg = 8;
constexpr size_t kPartialCap = (size_t)256 << 20;   // bytes of an automatic split's sums

long tiles_of(int cfg, int m, int n) { return ((long)m + kTiles[cfg].bm - 1) / kTiles[cfg].bm * (((long)n + kTiles[cfg].bn - 1) / kTiles[cfg].bn); }

// Up to 128 rows: the weights' stream, and for narrow ones the latency of a few slabs.
Fp8Plan few_rows_plan(int m, int n, int blocks) {
    auto plan = [&](int cfg, long split) {
        while (split > 1 && (size_t)split * m * n * sizeof(float) > kPartialCap) --split;
        split = std::max(1L, split);
        const int per = (int)((blocks + split - 1) / split);
        return Fp8Plan{cfg, (blocks + per - 1) / per, per};
    };
    // Up to 16 rows of weights that fit the chip in one go: one launch without sums (1 row of codes, us, with / without this kernel: 3584 x 3584
    // 5.4 / 7.1, 2048 x 2048 3.8 / 6.0, 512 x 256 2.0 / 3.1, 8192 x 2048 6.1 / 7.4, 16384 x 512 3.8 / 4.3; beyond the line 4608 x 3584 8.0 / 7.5,
    // 5120 x 5120 12.7 / 8.8, 37888 x 3584 30 / 27).
    const long narrow = (n + 15L) / 16;
    if (m <= 16 && blocks <= 32 && narrow * blocks <= 8192 && (blocks <= 16 || narrow <= 256)) return {kRowsCfg, 1, blocks};
    const long tiles = (n + 127L) / 128, wide = (n + 255L) / 256;
    // A unit takes in A beside the weights, so the widest tile that still gives every unit one; where columns are few, K slices, of 5
    // slabs at least, which cost a launch and their sums (3 us) and pay from 20 slabs on (64 rows, us: 5120 x 5120 in 1 / 3 / 5 slices 22 / 15.4 /
    // 13.7, 3584 x 18944 in 4 / 9 25.3 / 20.2, 9000 x 2048 in 1 / 3 10.5 / 11.9).
    if (m <= 64) {
        if (tiles <= 256) return plan(0, blocks >= 20 ? std::min(256 / tiles, blocks / 5L) : 1);
        return plan(wide <= 256 ? 1 : 0, 1);
    }
    // 65 to 128 rows on half the chip's units at most: two tiles of 64 rows in slices of 9 slabs at least, while a slice is short enough that
    // reading the weights twice does not show (128 rows: 5120 x 5120 13.9 on 64 rows in 3 slices, 16.8 on 128 in 6; 3584 x 18944 25.8 and 26.6;
    // 5120 x 27648 48.9 in 3 and 40.0 in 6).
    if (2 * tiles <= 256) {
        const long split = blocks >= 20 ? std::max(1L, std::min(256 / (2 * tiles), blocks / 9L)) : 1;
        if (blocks <= 48 * split) return plan(0, split);
    }
    if (tiles <= 256) return plan(2, blocks >= 20 ? std::min(256 / tiles, blocks / 9L) : 1);
    return plan(wide <= 256 ? 3 : 2, 1);
}

}  // namespace

void laps_fp8_tile_dims(int cfg, int* bm, int* bn) {
    *bm = cfg >= 0 && cfg < kNumTiles ? kTiles[cfg].bm : 0;
    *bn = cfg >= 0 && cfg < kNumTiles ? kTiles[cfg].bn : 0;
}

Fp8Plan laps_fp8_plan(int m, int n, int k) {
    const int blocks = k / FP8_BLOCK;
    if (m <= 128) return few_rows_plan(m, n, blocks);
    // Above 128 rows: workgroups on the busiest unit times what one takes, not less than the weights take from HBM; a split adds a launch and
    // its sums written and read back.
    auto moved = [](double b) { return std::min(b, 64e6) / 6.66e6 + std::max(0.0, b - 64e6) / 10.9e6; };
    const double mn = (double)m * n;
    double best = 1e30;
    Fp8Plan pick = {7, 1, blocks};
    for (int cfg = 0; cfg < kRowsCfg; ++cfg) {
        if (cfg == 1) continue;
        const TileDef& t = kTiles[cfg];
        const long tiles = tiles_of(cfg, m, n), rows = ((long)m + t.bm - 1) / t.bm;
        const double slab = t.slab * (1 - t.live * (1 - (double)m / ((double)rows * t.bm)));
        for (int s = 1; s <= 20 && s <= std::max(1, blocks / 2); ++s) {
            const int per = (blocks + s - 1) / s;
            if ((blocks + per - 1) / per != s) continue;
            if (s > 1 && (tiles * s > 512 || 4.0 * s * mn > (double)kPartialCap)) break;
            const long wgs = tiles * s, deep = (wgs + 255) / 256;
            const double all = per * slab, last = (wgs - (deep - 1) * 256) / 256.0;
            double us;
            if (t.pair > 0) us = deep / 2 * (t.fill + 2 * t.pair * all) + deep % 2 * (t.fill + all * (1 - t.part * (1 - std::min(1.0, wgs / 256.0))));
            else us = (deep - 1) * (t.fill + all) + t.fill + all * (1 - t.part * (1 - last));
            us = 1.6 + std::max(us, 3.4 + (double)n * k / 3.8e6);
            if (s > 1) us += 3.2 + moved(8.0 * s * mn + 2.0 * mn);
            if (us < best) {
                best = us;
                pick = {cfg, s, per};
            }
        }
    }
    return pick;
}

int laps_launch_gemm_fp8(const Fp8Plan& p, const unsigned char* a, const unsigned char* a_scales, const unsigned char* w,
                         const unsigned char* w_scales, bf16_t* out, int m, int n, int k, float* partial, hipStream_t s) {
    int bm, bn;
    laps_fp8_tile_dims(p.cfg, &bm, &bn);
    if (bm == 0) {
        laps_set_error("gemm_fp8: no tile %d", p.cfg);
        return LAPS_EINVAL;
    }
    if (p.cfg == kRowsCfg) return launch_rows<false>({a, a_scales, nullptr, w, w_scales, out, m, n, k, k, (int)fp8_pitch(m), (int)fp8_pitch(n)}, s);
    const Fp8Args g = {a, a_scales, w, w_scales, (int)fp8_pitch(m), (int)fp8_pitch(n), m, n, k, p.split, p.per, (m + bm - 1) / bm, (n + bn - 1) / bn,
                       out, partial};
    int rc = LAPS_EINVAL;
    switch (p.cfg) {
        case 0: rc = launch_tile<64, 128, 2, 2>(g, s); break;
        case 1: rc = launch_tile<64, 256, 1, 4>(g, s); break;
        case 2: rc = launch_tile<128, 128, 2, 2>(g, s); break;
        case 3: rc = launch_tile<128, 256, 1, 4>(g, s); break;
        case 4: rc = launch_tile<192, 256, 2, 2>(g, s); break;
        case 5: rc = launch_tile<256, 128, 2, 2>(g, s); break;
        case 6: rc = launch_tile<256, 192, 4, 1>(g, s); break;
        case 7: rc = launch_tile<256, 256, 2, 2>(g, s); break;
    }
    LAPS_TRY(rc);
    if (p.split > 1) {
        const long count = (long)m * n;
        hipLaunchKernelGGL(fp8_sum_kernel, dim3((unsigned)((count + 2047) / 2048)), dim3(256), 0, s, partial, p.split, count, out);
        LAPS_LAUNCH_CHECK();
    }
    return LAPS_OK;
}

// Quantised on the way, where that beats a launch of its own: up to 8 rows, or a block a wave (3584 x 3584 at 1 / 4 / 16 rows 6.5 / 7.0 / 10.1 us, in
// two launches 8.6 / 8.6 / 9.6; 2048 x 2048 at 16 5.8 and 7.4).
bool laps_fp8_takes_bf16_rows(const Fp8Plan& p, const bf16_t* x, int m, int k) {
    return p.cfg == kRowsCfg && (m <= 8 || p.per <= 16) && k % 8 == 0 && (reinterpret_cast<uintptr_t>(x) & 15) == 0;
}

int laps_launch_linear_fp8_rows(const bf16_t* x, const unsigned char* w, const unsigned char* w_scales, bf16_t* out, int m, int n, int k, hipStream_t s) {
    return launch_rows<true>({nullptr, nullptr, x, w, w_scales, out, m, n, k, (int)fp8_columns(k), (int)fp8_pitch(m), (int)fp8_pitch(n)}, s);
}
