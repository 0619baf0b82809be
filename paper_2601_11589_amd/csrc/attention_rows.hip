// Attention over the 4-bit or 8-bit cache for few query rows a sequence: single tokens, drafted tokens, the shortest turns.
//
//   O = softmax(Q K^T / sqrt(hd)) V over the cached keys, row t of a sequence seeing keys <= H + t
//
// One pass over the keys with a running maximum and sum a row.  What bounds it is the cache: 8.5 * hd bytes of K in 4 bits, 16 * hd in 8, and
// as many of V for 16 keys of a kv head, and 4 * 16 * hd flops for each of the G query heads that share them.  So nothing is staged: a wave
// walks the keys 32 at a time (two pages), and every load is one 16-byte piece a lane, 1 KB of a page a wave, straight into the
// operand registers of 16x16x32 matrix instructions.  Over 4 bits:
//
//   S^T = K Q^T   lane (i, g) = (lane % 16, lane / 16) holds key i and head_dim indices hd/4 g .. hd/4 g + hd/4 - 1: its piece of the page
//                 [16 keys][hd / 2 bytes].  Which index is which of the instruction's 32 does not matter as long as Q's registers agree.
//   O^T = V^T P^T the result above leaves lane (i, g) with row i's scores of keys 4g .. 4g + 3 of both pages; those eight are its
//                 share of the second product's 32 keys, and V's pages are laid out for that: [hd / 8][16 keys][8 values], four keys of
//                 the same eight (hd 64: four) head_dim indices a lane.  No value changes lanes.
//
// Codes become bf16 operands exactly (one instruction a pair, the scale included; over 4 bits two permutes a pair of V's to bring keys
// side by side).  The query rows are the G heads of a kv head for each of the sequence's new tokens, 16 a block.
// Weights are rounded to bf16, which the second product takes, and their sum is that of the rounded ones, so that they add up to one; scores,
// sums, O and partial results are float32.  That makes outputs 1.1 to 1.4 times as far from 64 bits as float32 weights would (1.8e-3 to
// 2.3e-3 of the output against 1.6e-3 to 1.7e-3, most of it the output's own rounding), the same as over bf16 pools.
// 8 bits (KV8): 16 * hd bytes of K and of V for 16 keys, two pieces a lane of either: K's page is [16 keys][hd], a lane's pieces are
// 16 g .. 16 g + 15 of every 64; V's [hd / 4][4 key groups][4][4 keys], a dword is four keys of an index, side by side already.  One scale a
// page and kv head.  32B, 64 tokens over 4096 keys 86 us (6.2 TB/s), over 512 to 8191 115 (4.9); 7B, two tokens over 100000 keys and
// more 49 (4.8): HBM.  16 sequences of 16 tokens over 2048 keys 34, of 64 83: a vector instruction is active in 44 % of the time, the matrix
// pipe in 23 %.
// Four waves of a workgroup take every fourth pair of pages and add up in LDS.  Few sequences over long keys: a sequence's keys go out
// in parts of equal length to workgroups of their own, and a second kernel adds those, in order.
#include "attention_rows.h"
#include "fp8.h"
#include "kv4.h"

#include <climits>
#include <type_traits>

namespace {

constexpr int WAVES = 4;
constexpr int STEP = 2 * LAPS_PAGE;   // keys a wave takes at a time
static_assert(WAVES * STEP == LAPS_KV4_ROUND, "a step for every wave");
constexpr int MAX_PARTS = 96;         // a resident workgroup a place for 8 (sequence, kv head) pairs
constexpr float MOST = 256.f;   // sum of eight weights above which the reference moves

typedef unsigned char byte_t;

// New tokens, cached tokens and first row of a sequence, cut to what the arrays can hold; false: nothing to do.
struct SeqRange { int rs, L, H; };
__device__ __forceinline__ bool seq_range(int seq, const int* cu, const int* seq_len, const int* prefix_len, int n_tokens,
                                          int max_pages, SeqRange* r) {
    const int rs = cu[seq], cap = cu[seq + 1] - rs;
    int L = seq_len ? seq_len[seq] : cap;
    L = L < cap ? L : cap;
    if (L <= 0 || rs < 0 || L > n_tokens - rs) return false;
    r->rs = rs;
    r->L = L;
    r->H = laps_dev_clamp_prefix(prefix_len[seq], L, max_pages);
    return true;
}

// Of either cache, whatever the name.
__device__ __forceinline__ int part_steps(int kv_len, int max_pages, int parts, int min_parts, int* used) {
    return laps_kv4_part_rounds(kv_len, max_pages, parts, min_parts, used) * WAVES;
}

// One step's codes and scales as they come from the pools.
template <int HD, bool KV8>
struct Piece {
    unsigned k[2][HD / 32], ks[2];   // [page]: HD / 4 codes of key i, the dword with their group's scale byte
    u32x4 v[2];                      // eight codes (HD 64: four of them used) of keys 4g .. 4g + 3
    unsigned vs[2];                  // those keys' scale bytes
};
template <int HD>
struct Piece<HD, true> {
    u32x4 k[2][HD / 64];             // [page]: codes of key i, 16 of every 64
    u32x4 v[2][HD / 64];             // four head_dim indices of every 64, keys 4g .. 4g + 3 of each a dword
    unsigned ks[2], vs[2];           // the page's scale bytes, each in a dword of four kv heads'
};

// O += V^T P^T.  8-bit pools: by hand, with one operand for what O was and what it is.  The builtin has two, and with twice the pieces of a
// step in registers the allocator no longer gets by without moves and spills: two blocks of rows 25 spills at 2 waves a SIMD, now none.
// The compiler does not know what such an instruction needs before and behind it: the two wait states behind vector instructions that
// made its operands stand here, those before O is used otherwise are o_settle's.  That O is not moved between the bodies of the loop, where no
// o_settle stands, is looked up in the assembly by tests/test_matrix_asm_waits_host.py: run it after a change of compiler or flags.
template <bool KV8>
__device__ __forceinline__ void add_product(f32x4& o, bf16x8 v, bf16x8 p) {
    if constexpr (KV8) asm volatile("s_nop 1\n\tv_mfma_f32_16x16x32_bf16 %0, %1, %2, %0" : "+v"(o) : "v"(v), "v"(p));
    else o = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, p, o, 0, 0, 0);
}
template <bool KV8, int NR, int DL>
__device__ __forceinline__ void o_settle(f32x4 (&o)[NR][DL]) {
    if constexpr (KV8) {
        asm volatile("s_nop 15\n\ts_nop 15" ::: "memory");
#pragma unroll
        for (int a = 0; a < NR; ++a)
#pragma unroll
            for (int j = 0; j < DL; ++j) asm volatile("" : "+v"(o[a][j]));
    }
}

// 8-bit pools, several blocks of rows: those of a (sequence, part, kv head) read the same keys and go to one XCD one after the other, in n
// groups where there are too few of these for the 8 XCDs to share evenly.  Against kv heads side by side, which 4-bit blocks want (they
// share lines): 32B, 64 sequences of 16 tokens over 2000 keys 113 -> 94 us, 16 of 64 over 2048 88 -> 76, 7B, two of 17 over 60000 81 -> 64.
struct RowsGroups {
    int n, blocks;   // blocks of a group
    __host__ __device__ RowsGroups(int units, int row_blocks) {
        n = (64 + units - 1) / units;
        n = n < row_blocks ? n : row_blocks;
        blocks = (row_blocks + n - 1) / n;
    }
};

// NR: blocks of 16 rows that share what is read and unpacked.
// Waves a SIMD: as many as registers allow, 3 (4 bits, one block) or 2.  8 bits have twice the pieces of a step in registers; with one block
// they go two steps ahead at 2 waves rather than one step ahead at 3: 32B, 64 tokens over 4096 keys each 112 -> 98 us, over 512 to
// 8191 130 -> 114 (two and three parts a sequence; the loads alone, without the work on them, took 92 of the first).
// Four blocks that share what is unpacked, at one wave a SIMD, are not kept: 32B, 16 sequences of 17 to 64 tokens over 512 to 4096 keys
// 88 us and, with the next step's scores among this one's exponentials, 92; two blocks 78.
template <int HD, int NR, bool KV8>
__global__ __launch_bounds__(WAVES * 64, NR == 1 && !KV8 ? 3 : 2) void attn_rows_kernel(
    const bf16_t* __restrict__ q, bf16_t* __restrict__ out, const byte_t* __restrict__ k_pool, const byte_t* __restrict__ v_pool,
    const int* __restrict__ cu, const int* __restrict__ seq_len, const int* __restrict__ prefix_len,
    const int* __restrict__ page_table, int max_pages, int n_seq, int n_tokens, int n_q, int n_kv, int n_pool_pages, int row_blocks, int more_rows,
    int parts, int min_parts, float scale_log2e, float* __restrict__ part_o, float* __restrict__ part_ml) {
    constexpr int AHEAD = KV8 && NR == 1 ? 2 : 1;   // steps whose loads are on their way behind the one that is worked on
    constexpr int KS = HD / 32;        // matrix instructions of a page's scores
    constexpr int DL = HD / 16;        // head_dim indices of a lane of V, and of the result's 16 rows each
    constexpr int BLOCK = kv4_block(HD), CODES = kv4_codes(HD), ROWS = 16 * NR;
    __shared__ __align__(16) float red_o[WAVES][16][HD + 4];
    __shared__ float red_ml[WAVES][2][16];

    // Workgroup b runs on XCD b % 8.  The kv heads of a (sequence, part, row block) go to one XCD side by side: a page's heads are
    // neighbours in memory and a block is 8.5 (4.25) lines of 128 bytes, so that each fetches a line that the next one needs too.
    const int G = n_q / n_kv;
    int bid = blockIdx.x, rb0 = 0;
    if constexpr (KV8 && NR > 1) {   // the launch several times over, for the last row_blocks blocks of a sequence first
        const int launch = gridDim.x / more_rows;
        rb0 = (more_rows - 1 - bid / launch) * row_blocks;
        bid %= launch;
    }
    int kvh = bid / 8 % n_kv, rest = bid / 8 / n_kv * 8 + bid % 8;
    if constexpr (KV8 && NR > 1) {
        const RowsGroups grp(n_seq * parts * n_kv, row_blocks);
        const int at = bid / 8, unit = at / grp.blocks * 8 + bid % 8, rb = unit % grp.n + at % grp.blocks * grp.n;
        if (rb >= row_blocks) return;
        rb0 += rb;
        kvh = unit / grp.n % n_kv;
        rest = unit / grp.n / n_kv;
    } else {
        rb0 = rest % row_blocks;
        rest /= row_blocks;
    }
    const int part = rest % parts, seq = rest / parts;
    if (seq >= n_seq) return;
    SeqRange r;
    if (!seq_range(seq, cu, seq_len, prefix_len, n_tokens, max_pages, &r)) return;
    const int n_rows = r.L * G, kv_len = r.H + r.L;
    int used;
    const int each = part_steps(kv_len, max_pages, parts, min_parts, &used);
    if (part >= used) return;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), i = lane & 15, g = lane >> 4;
    const int need = (kv_len + LAPS_PAGE - 1) / LAPS_PAGE, n_pages = need < max_pages ? need : max_pages;
    const int* pt = page_table + (size_t)seq * max_pages;
    const unsigned k_turn = (8 * (HD == 128 ? g : 2 * (i & 1) + (g >> 1)) + 9) & 31;   // right rotation that brings the lane's scale byte up
    // 8-bit pools: a lane's places in a block, and that of the scales' dword from there (in a vector register: scalar loads return in any
    // order, so that each wait for one is for those of the next step too)
    [[maybe_unused]] const unsigned kv8_lane_k = i * HD + g * 16, kv8_lane_v = i * 64 + g * 16;
    [[maybe_unused]] const int kv8_turn = 8 * (kvh & 3);
    [[maybe_unused]] unsigned kv8_lane_s = (n_kv - kvh) * kv8_codes(HD) + (kvh & ~3);
    [[maybe_unused]] const int kv8_bytes = kv8_lane_s + 4;   // from the block to the end of that dword
    asm volatile("" : "+v"(kv8_lane_s));
    const int v_chunk = HD == 128 ? i : i >> 1, v_group = i / (KV4_GROUP / DL), o_group = g * 4 * DL / KV4_GROUP;

    for (int rb = rb0; rb * ROWS < n_rows; rb += KV8 && NR > 1 ? row_blocks * more_rows : row_blocks) {
        const int last_row = rb * ROWS + ROWS - 1 < n_rows ? rb * ROWS + ROWS - 1 : n_rows - 1;
        const int vis_min = r.H + rb * ROWS / G, kv_end = r.H + last_row / G + 1;  // seen by every row, by the last row
        int limit[NR];                                                             // last key this lane's rows see
        bf16x8 qf[NR][KS];
#pragma unroll
        for (int a = 0; a < NR; ++a) {
            const int row = rb * ROWS + 16 * a + i, rc = row < n_rows ? row : n_rows - 1, tq = rc / G;
            limit[a] = r.H + tq;
            const u32x4* qp = reinterpret_cast<const u32x4*>(q + (size_t)(r.rs + tq) * n_q * HD + (size_t)(kvh * G + rc - tq * G) * HD);
#pragma unroll
            for (int kk = 0; kk < KS; ++kk) qf[a][kk] = __builtin_bit_cast(bf16x8, qp[KV8 ? kk / 2 * 8 + g * 2 + kk % 2 : g * KS + kk]);
        }
        f32x4 o[NR][DL];
        float m_run[NR], l_run[NR];   // reference in log2 units (the same in the four lanes of a row), this lane's sum
#pragma unroll
        for (int a = 0; a < NR; ++a) {
            m_run[a] = -INFINITY;
            l_run[a] = 0.f;
#pragma unroll
            for (int j = 0; j < DL; ++j) o[a][j] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
        int nan_key = INT_MAX;        // first key with a NaN group in this lane's v_group, where not every row sees it

        const int s_begin = part * each + wave;
        int s_end = (kv_end + STEP - 1) / STEP;
        s_end = s_end < (part + 1) * each ? s_end : (part + 1) * each;
        const int n_steps = s_begin < s_end ? (s_end - s_begin + WAVES - 1) / WAVES : 0;

        int ids = 0;   // page ids of the next 32 steps, one a lane
        auto fetch_ids = [&](int n) {
            int p = 2 * (s_begin + (n + (lane >> 1)) * WAVES) + (lane & 1);
            p = p < n_pages ? p : n_pages - 1;                 // past the end: any page, masked below
            const int id = pt[p];
            ids = (id > 0 && id < n_pool_pages) ? id : 0;      // unset, or not a page of the pool
            asm volatile("" : "+v"(ids));   // waited for here: behind the join it would be waited for at every step, with all loads in flight
        };
        // 4 bits, up to 16 rows a sequence: keys are read once and past the caches, 2.3 GB 418 -> 378 us (6.0 TB/s; 280 MB that the memory-side
        // cache held from the call before 52 -> 58).  More rows: other blocks of theirs read the same keys.
        auto codes = [](const auto* from) { return NR == 1 ? __builtin_nontemporal_load(from) : *from; };
        // 8-bit pools: steps past the last one go through descriptors of no bytes, which takes no request.
        auto load = [&](int n, Piece<HD, KV8>& x) {
            [[maybe_unused]] const int bytes = n < n_steps ? kv8_bytes : 0;
            if ((n & 31) == 0) fetch_ids(n);
#pragma unroll
            for (int p = 0; p < 2; ++p) {
                const int page = __builtin_amdgcn_readlane(ids, 2 * (n & 31) + p);
                if constexpr (KV8) {   // through descriptors of the block: its base in scalar registers, a lane's place in one vector register
                    const size_t at = (size_t)page * kv8_page(n_kv, HD) + (size_t)kvh * kv8_codes(HD);
                    auto block = [&](const byte_t* pool) { return __builtin_amdgcn_make_buffer_rsrc(const_cast<byte_t*>(pool + at), 0, bytes, 0x00020000); };
                    const __amdgpu_buffer_rsrc_t kb = block(k_pool), vb = block(v_pool);
                    // past the caches (nt) V alone, on the same terms: a load of K takes (head_dim 128) 64 bytes of each of its 128-byte lines, and
                    // the other half would be fetched again
                    constexpr int PAST = NR == 1 ? 2 : 0;
#pragma unroll
                    for (int u = 0; u < HD / 64; ++u) {
                        x.k[p][u] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(kb, kv8_lane_k + u * 64, 0, 0));
                        x.v[p][u] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(vb, kv8_lane_v + u * 1024, 0, PAST));
                    }
                    x.ks[p] = __builtin_amdgcn_raw_buffer_load_b32(kb, kv8_lane_s, 0, 0);
                    x.vs[p] = __builtin_amdgcn_raw_buffer_load_b32(vb, kv8_lane_s, 0, 0);
                } else {
                    const size_t at = ((size_t)page * n_kv + kvh) * BLOCK;
                    const byte_t *kb = k_pool + at, *vb = v_pool + at;
                    if constexpr (HD == 128) {
                        const u32x4 w = codes(reinterpret_cast<const u32x4*>(kb) + i * 4 + g);
#pragma unroll
                        for (int kk = 0; kk < 4; ++kk) x.k[p][kk] = w[kk];
                    } else {
                        const u32x2 w = codes(reinterpret_cast<const u32x2*>(kb) + i * 4 + g);
                        x.k[p][0] = w.x;
                        x.k[p][1] = w.y;
                    }
                    x.ks[p] = reinterpret_cast<const unsigned*>(kb + CODES)[HD == 128 ? i : i >> 1];
                    x.v[p] = codes(reinterpret_cast<const u32x4*>(vb) + v_chunk * 4 + g);
                    x.vs[p] = reinterpret_cast<const unsigned*>(vb + CODES)[v_group * 4 + g];
                }
            }
        };
        auto compute = [&](int n, Piece<HD, KV8>& x) {
            const int key0 = (s_begin + n * WAVES) * STEP;
            f32x4 s[NR][2];
#pragma unroll
            for (int p = 0; p < 2; ++p) {
                const float ks = KV8 ? fp8_scale(x.ks[p] >> kv8_turn & 255u)
                                     : __uint_as_float(__builtin_amdgcn_alignbit(x.ks[p], x.ks[p], k_turn));   // the byte to bits 23 to 30
#pragma unroll
                for (int a = 0; a < NR; ++a) s[a][p] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int kk = 0; kk < KS; ++kk) {
                    bf16x8 kf;
                    if constexpr (KV8) kf = __builtin_bit_cast(bf16x8, fp8_eight(x.k[p][kk / 2][kk % 2 * 2], x.k[p][kk / 2][kk % 2 * 2 + 1], ks));
                    else kf = __builtin_bit_cast(bf16x8, kv4_eight(x.k[p][kk], ks));
#pragma unroll
                    for (int a = 0; a < NR; ++a) s[a][p] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[a][kk], s[a][p], 0, 0, 0);
                }
            }
            if (key0 + STEP - 1 > vis_min) {   // some row does not see all of these keys
#pragma unroll
                for (int p = 0; p < 2; ++p) {
                    const int k4 = key0 + p * LAPS_PAGE + 4 * g;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
#pragma unroll
                        for (int a = 0; a < NR; ++a)
                            if (k4 + e > limit[a]) s[a][p][e] = -INFINITY;   // whatever it was, NaN included
                        // V of a key that a row does not see has weight zero, which a NaN would survive: slots past the sequence's end
                        // hold anything, and a NaN group of a key before it shows in the rows that see it only
                        if constexpr (KV8) {   // a token's head is NaN as a whole or not at all
                            if (k4 + e >= kv_len || (x.v[p][0].x >> (8 * e) & 127u) == 127u) {
                                if (k4 + e < kv_len) nan_key = k4 + e < nan_key ? k4 + e : nan_key;
#pragma unroll
                                for (int u = 0; u < HD / 64; ++u) x.v[p][u] &= ~(255u << (8 * e));
                            }
                        } else {
                            const unsigned byte = (x.vs[p] >> (8 * e)) & 255u;
                            if (k4 + e >= kv_len || byte == 255u) {
                                if (k4 + e < kv_len) nan_key = k4 + e < nan_key ? k4 + e : nan_key;
                                x.v[p][e] = 0u;
                                x.vs[p] &= ~(255u << (8 * e));
                            }
                        }
                    }
                }
            }
            // The reference that the exponentials subtract is the row's maximum as of some earlier step.  It moves when the weights it
            // gives add up to more than MOST (or when there is none yet): no maximum is taken in the other steps, and the exchange between a
            // row's four lanes and the rescale of O are rare.  The quotient O / l does not depend on it; weights stay far from
            // float32's range, and since the maximum never falls below the reference, so does l.
            bf16x8 pf[NR];
            float sum[NR];   // of the weights as the second product sees them
            auto weights = [&](int a) {
                const float m_sub = m_run[a] == -INFINITY ? 0.f : m_run[a];   // a row that has seen no key yet
                sum[a] = 0.f;
#pragma unroll
                for (int p = 0; p < 2; ++p)
#pragma unroll
                    for (int e = 0; e < 4; e += 2) {
                        bf16x2 w;
                        w.x = (__bf16)__builtin_amdgcn_exp2f(__builtin_fmaf(s[a][p][e], scale_log2e, -m_sub));
                        w.y = (__bf16)__builtin_amdgcn_exp2f(__builtin_fmaf(s[a][p][e + 1], scale_log2e, -m_sub));
                        pf[a][4 * p + e] = w.x;
                        pf[a][4 * p + e + 1] = w.y;
                        sum[a] = __builtin_amdgcn_fdot2_f32_bf16(w, bf16x2{(__bf16)1.f, (__bf16)1.f}, sum[a], false);
                    }
            };
            bool move = false;
#pragma unroll
            for (int a = 0; a < NR; ++a) {
                weights(a);
                move = move || sum[a] > MOST || m_run[a] == -INFINITY;
            }
            if (__builtin_amdgcn_ballot_w64(move) != 0) {
                o_settle<KV8>(o);
#pragma unroll
                for (int a = 0; a < NR; ++a) {
                    float mx = fmaxf(fmaxf(fmaxf(s[a][0].x, s[a][0].y), fmaxf(s[a][0].z, s[a][0].w)),
                                     fmaxf(fmaxf(s[a][1].x, s[a][1].y), fmaxf(s[a][1].z, s[a][1].w))) * scale_log2e;
                    mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
                    mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
                    const float m_new = fmaxf(m_run[a], mx);
                    const float alpha = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m_run[a] - m_new);
                    l_run[a] *= alpha;
#pragma unroll
                    for (int j = 0; j < DL; ++j) o[a][j] *= alpha;
                    m_run[a] = m_new;
                    weights(a);
                }
            }
#pragma unroll
            for (int a = 0; a < NR; ++a) l_run[a] += sum[a];
            if constexpr (KV8) {   // the keys lie side by side already
                const float vs0 = fp8_scale(x.vs[0] >> kv8_turn & 255u), vs1 = fp8_scale(x.vs[1] >> kv8_turn & 255u);
#pragma unroll
                for (int j = 0; j < DL; ++j) {
                    const u32x2 lo = fp8_four(x.v[0][j / 4][j % 4], vs0), hi = fp8_four(x.v[1][j / 4][j % 4], vs1);
                    const bf16x8 vf = __builtin_bit_cast(bf16x8, u32x4{lo.x, lo.y, hi.x, hi.y});
#pragma unroll
                    for (int a = 0; a < NR; ++a) add_product<KV8>(o[a][j], vf, pf[a]);
                }
            } else {
                // codes of one head_dim pair of the eight keys, then the keys side by side
                auto pair_of_keys = [&](auto B) {
                    constexpr int b = decltype(B)::value;
                    unsigned w[8];
#pragma unroll
                    for (int p = 0; p < 2; ++p) {
                        auto word = [&](int e) { return HD == 128 ? x.v[p][e] : x.v[p][e] >> (16 * (i & 1)); };
                        w[4 * p + 0] = kv4_pair<b>(word(0), kv4_scale<0>(x.vs[p]));
                        w[4 * p + 1] = kv4_pair<b>(word(1), kv4_scale<1>(x.vs[p]));
                        w[4 * p + 2] = kv4_pair<b>(word(2), kv4_scale<2>(x.vs[p]));
                        w[4 * p + 3] = kv4_pair<b>(word(3), kv4_scale<3>(x.vs[p]));
                    }
                    u32x4 lo, hi;
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        lo[k] = __builtin_amdgcn_perm(w[2 * k + 1], w[2 * k], 0x05040100u);
                        hi[k] = __builtin_amdgcn_perm(w[2 * k + 1], w[2 * k], 0x07060302u);
                    }
#pragma unroll
                    for (int a = 0; a < NR; ++a) {
                        o[a][2 * b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, lo), pf[a], o[a][2 * b], 0, 0, 0);
                        o[a][2 * b + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, hi), pf[a], o[a][2 * b + 1], 0, 0, 0);
                    }
                };
                pair_of_keys(std::integral_constant<int, 0>{});
                pair_of_keys(std::integral_constant<int, 1>{});
                if constexpr (HD == 128) {
                    pair_of_keys(std::integral_constant<int, 2>{});
                    pair_of_keys(std::integral_constant<int, 3>{});
                }
            }
        };
        // The next step is on its way while one is worked on; two buffers in turn.  Past the last step the last one is loaded again:
        // with a branch round the loads every wait would be for all of them.
        if (n_steps > 0) {
            Piece<HD, KV8> x, y;
            [[maybe_unused]] Piece<HD, KV8> z;
            auto load_at = [&](int n, Piece<HD, KV8>& to) { load(KV8 || n < n_steps ? n : n_steps - 1, to); };
            load_at(0, x);
#pragma unroll
            for (int a = 0; a < NR; ++a)
#pragma unroll
                for (int kk = 0; kk < KS; ++kk) asm volatile("" : "+v"(qf[a][kk]));   // as ids: the loop must find Q arrived
            if constexpr (AHEAD == 2) {
                load_at(1, y);
                for (int n = 0;;) {
                    load_at(n + 2, z);
                    __builtin_amdgcn_sched_barrier(0);
                    compute(n, x);
                    if (++n >= n_steps) break;
                    load_at(n + 2, x);
                    __builtin_amdgcn_sched_barrier(0);
                    compute(n, y);
                    if (++n >= n_steps) break;
                    load_at(n + 2, y);
                    __builtin_amdgcn_sched_barrier(0);
                    compute(n, z);
                    if (++n >= n_steps) break;
                }
            } else for (int n = 0;;) {
                load_at(n + 1, y);
                __builtin_amdgcn_sched_barrier(0);   // loads first: mixed with the work, their registers get copied behind waits
                compute(n, x);
                if (++n >= n_steps) break;
                load_at(n + 1, x);
                __builtin_amdgcn_sched_barrier(0);
                compute(n, y);
                if (++n >= n_steps) break;
            }
        }

        o_settle<KV8>(o);
        // ---- NaN groups of keys that not every row sees
        nan_key = min(nan_key, __shfl_xor(nan_key, 16, 64));
        nan_key = min(nan_key, __shfl_xor(nan_key, 32, 64));
        const int nan_from = KV8 ? nan_key : __shfl(nan_key, o_group * (KV4_GROUP / DL), 64);
#pragma unroll
        for (int a = 0; a < NR; ++a) {
            if (rb * ROWS + 16 * a >= n_rows) break;
            if (nan_from <= limit[a]) {
#pragma unroll
                for (int j = 0; j < DL; ++j) o[a][j] += __builtin_nanf("");
            }
            // ---- the four waves' results: lane (i, g) holds row i, head_dim indices 4 DL g + DL e + j (8 bits: 64 (j / 4) + 16 g + 4 e + j % 4)
            l_run[a] += __shfl_xor(l_run[a], 16, 64);
            l_run[a] += __shfl_xor(l_run[a], 32, 64);
            __syncthreads();   // the rows before are read
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int j = 0; j < DL; j += 4)
                    *reinterpret_cast<f32x4*>(&red_o[wave][i][KV8 ? 16 * j + 16 * g + 4 * e : (4 * g + e) * DL + j]) = f32x4{o[a][j][e], o[a][j + 1][e], o[a][j + 2][e], o[a][j + 3][e]};
            if (g == 0) {
                red_ml[wave][0][i] = m_run[a];
                red_ml[wave][1][i] = l_run[a];
            }
            __syncthreads();
            constexpr int PER = 16 * HD / (WAVES * 64);   // values a thread finishes
            const int fr = tid / (HD / PER), fd = tid % (HD / PER) * PER, frow = rb * ROWS + 16 * a + fr;
            if (frow < n_rows) {
                float m_all = red_ml[0][0][fr];
#pragma unroll
                for (int w = 1; w < WAVES; ++w) m_all = fmaxf(m_all, red_ml[w][0][fr]);
                const float m_sub = m_all == -INFINITY ? 0.f : m_all;   // no key seen here, or NaN scores only
                float l_all = 0.f, v[PER];
#pragma unroll
                for (int k = 0; k < PER; ++k) v[k] = 0.f;
#pragma unroll
                for (int w = 0; w < WAVES; ++w) {
                    const float f = __builtin_amdgcn_exp2f(red_ml[w][0][fr] - m_sub);
                    l_all += f * red_ml[w][1][fr];
#pragma unroll
                    for (int k = 0; k < PER; ++k) v[k] += f * red_o[w][fr][fd + k];
                }
                const int ft = frow / G;
                const size_t at = (size_t)(r.rs + ft) * n_q + kvh * G + frow - ft * G;   // (row, query head) of the batch
                if (used == 1) {
                    const float inv = 1.f / l_all;
#pragma unroll
                    for (int k = 0; k < PER; k += 4) {
                        u32x2 w;
                        w.x = pack_bf16x2(v[k] * inv, v[k + 1] * inv);
                        w.y = pack_bf16x2(v[k + 2] * inv, v[k + 3] * inv);
                        *reinterpret_cast<u32x2*>(out + at * HD + fd + k) = w;
                    }
                } else {
#pragma unroll
                    for (int k = 0; k < PER; k += 4)
                        *reinterpret_cast<f32x4*>(part_o + (at * parts + part) * HD + fd + k) = f32x4{v[k], v[k + 1], v[k + 2], v[k + 3]};
                    if (fd == 0) {
                        part_ml[(at * parts + part) * 2] = m_all;
                        part_ml[(at * parts + part) * 2 + 1] = l_all;
                    }
                }
            }
        }
    }
}

// Adds the parts of a sequence's keys: out = sum_p 2^(m_p - M) O_p / sum_p 2^(m_p - M) l_p, M = max_p m_p, each of 8 groups of
// HD / 4 lanes a run of the parts, the groups in order.  A workgroup takes one query head of one sequence, a row after the other.
template <int HD>
__global__ __launch_bounds__(8 * HD / 4) void attn_rows_merge_kernel(bf16_t* __restrict__ out, const float* __restrict__ part_o,
                                                                     const float* __restrict__ part_ml, const int* __restrict__ cu,
                                                                     const int* __restrict__ seq_len,
                                                                     const int* __restrict__ prefix_len, int max_pages,
                                                                     int n_tokens, int n_q, int parts, int min_parts) {
    constexpr int LANES = HD / 4, GROUPS = 8;
    static_assert(MAX_PARTS % GROUPS == 0 && MAX_PARTS <= 128, "two parts a lane, as many registers as a group has parts");
    __shared__ float weight[MAX_PARTS], l_all;
    __shared__ f32x4 red[GROUPS][LANES];
    const int head = blockIdx.x % n_q, seq = blockIdx.x / n_q, tid = threadIdx.x, c = tid % LANES, grp = tid / LANES;
    SeqRange r;
    if (!seq_range(seq, cu, seq_len, prefix_len, n_tokens, max_pages, &r)) return;
    int used;
    part_steps(r.H + r.L, max_pages, parts, min_parts, &used);
    if (used == 1) return;   // written by the attention kernel
    for (int t = blockIdx.y; t < r.L; t += gridDim.y) {
        const size_t at = ((size_t)(r.rs + t) * n_q + head) * parts;
        const int run = (used + GROUPS - 1) / GROUPS, p0 = grp * run;   // at most 12 parts a group, all on their way before any is used
        f32x4 v[MAX_PARTS / GROUPS];
#pragma unroll
        for (int p = 0; p < MAX_PARTS / GROUPS; ++p)
            if (p < run) v[p] = reinterpret_cast<const f32x4*>(part_o + (at + (p0 + p < used ? p0 + p : used - 1)) * HD)[c];
        if (tid < 64) {   // one wave: parts tid and tid + 64
            float m[2], l[2];
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const int p = tid + 64 * k;
                m[k] = p < used ? part_ml[(at + p) * 2] : -INFINITY;
                l[k] = p < used ? part_ml[(at + p) * 2 + 1] : 0.f;
            }
            float m_all = fmaxf(m[0], m[1]);
#pragma unroll
            for (int k = 32; k > 0; k >>= 1) m_all = fmaxf(m_all, __shfl_xor(m_all, k, 64));
            const float m_sub = m_all == -INFINITY ? 0.f : m_all;
            float sum = 0.f;
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const float f = __builtin_amdgcn_exp2f(m[k] - m_sub);
                if (tid + 64 * k < MAX_PARTS) weight[tid + 64 * k] = f;
                sum += f * l[k];
            }
#pragma unroll
            for (int k = 32; k > 0; k >>= 1) sum += __shfl_xor(sum, k, 64);
            if (tid == 0) l_all = sum;
        }
        __syncthreads();
        f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int p = 0; p < MAX_PARTS / GROUPS; ++p)
            if (p < run && p0 + p < used) acc += weight[p0 + p] * v[p];
        red[grp][c] = acc;
        __syncthreads();
        if (grp == 0) {
#pragma unroll
            for (int k = 1; k < GROUPS; ++k) acc += red[k][c];
            const float inv = 1.f / l_all;
            u32x2 w;
            w.x = pack_bf16x2(acc.x * inv, acc.y * inv);
            w.y = pack_bf16x2(acc.z * inv, acc.w * inv);
            *reinterpret_cast<u32x2*>(out + ((size_t)(r.rs + t) * n_q + head) * HD + 4 * c) = w;
        }
        __syncthreads();
    }
}

// The same for at most FEW_PARTS parts: HD / 4 lanes take a (row, query head), all its parts at once, no exchange between lanes.
// Attention with this merge / with the one above, us: 14B, 16 times 4 tokens over 4000 keys in 2 / 4 / 8 parts 23.9 / 23.3 / 29.5 and
// 29.3 / 28.2 / 33.6; 32B, 64 tokens over 4000 in 8 parts 68.3 and 72.5, 4 turns of 32 37.3 and 46.6; 7B, one token 11.1 and 10.8.
constexpr int FEW_PARTS = 8, FEW_THREADS = 256;
template <int HD>
__global__ __launch_bounds__(FEW_THREADS) void attn_rows_merge_few_kernel(bf16_t* __restrict__ out, const float* __restrict__ part_o,
                                                                          const float* __restrict__ part_ml,
                                                                          const int* __restrict__ cu, const int* __restrict__ seq_len,
                                                                          const int* __restrict__ prefix_len, int max_pages,
                                                                          int n_tokens, int n_q, int parts, int min_parts) {
    constexpr int LANES = HD / 4, GROUPS = FEW_THREADS / LANES;
    const int seq = blockIdx.x, c = threadIdx.x % LANES;
    SeqRange r;
    if (!seq_range(seq, cu, seq_len, prefix_len, n_tokens, max_pages, &r)) return;
    int used;
    part_steps(r.H + r.L, max_pages, parts, min_parts, &used);
    if (used == 1) return;   // written by the attention kernel
    const long items = (long)r.L * n_q, first = (long)r.rs * n_q;
    for (long it = (long)blockIdx.y * GROUPS + threadIdx.x / LANES; it < items; it += (long)gridDim.y * GROUPS) {
        const size_t at = (size_t)(first + it) * parts;
        f32x4 v[FEW_PARTS];
        float m[FEW_PARTS], l[FEW_PARTS];
#pragma unroll
        for (int p = 0; p < FEW_PARTS; ++p) {
            m[p] = -INFINITY;
            l[p] = 0.f;
            v[p] = f32x4{0.f, 0.f, 0.f, 0.f};
            if (p < used) {
                v[p] = reinterpret_cast<const f32x4*>(part_o + (at + p) * HD)[c];
                m[p] = part_ml[(at + p) * 2];
                l[p] = part_ml[(at + p) * 2 + 1];
            }
        }
        float m_all = m[0];
#pragma unroll
        for (int p = 1; p < FEW_PARTS; ++p) m_all = fmaxf(m_all, m[p]);
        const float m_sub = m_all == -INFINITY ? 0.f : m_all;
        f32x4 acc = {0.f, 0.f, 0.f, 0.f};
        float l_all = 0.f;
#pragma unroll
        for (int p = 0; p < FEW_PARTS; ++p) {
            const float f = __builtin_amdgcn_exp2f(m[p] - m_sub);
            acc += f * v[p];
            l_all += f * l[p];
        }
        const float inv = 1.f / l_all;
        u32x2 w;
        w.x = pack_bf16x2(acc.x * inv, acc.y * inv);
        w.y = pack_bf16x2(acc.z * inv, acc.w * inv);
        *reinterpret_cast<u32x2*>(out + (first + it) * HD + 4 * c) = w;
    }
}

template <int HD, bool KV8>
int launch_rows(const RowsAttn& a, const RowsPlan& p, float* part, hipStream_t s) {
    const float scale_log2e = 1.4426950408889634f / sqrtf((float)HD);
    float* part_ml = part ? part + (size_t)a.n_tokens * a.n_q * p.parts * HD : nullptr;
    auto kern = p.row_tiles == 1 ? attn_rows_kernel<HD, 1, KV8> : attn_rows_kernel<HD, 2, KV8>;
    int wgs = (a.n_seq * p.parts * p.row_blocks + 7) / 8 * 8 * a.n_kv;
    if (KV8 && p.row_tiles > 1) {
        const int units = a.n_seq * p.parts * a.n_kv;
        const RowsGroups grp(units, p.row_blocks);
        wgs = (units * grp.n + 7) / 8 * 8 * grp.blocks * p.more_rows;
    }
    hipLaunchKernelGGL(kern, dim3(wgs), dim3(WAVES * 64), 0, s, a.q, a.out, a.k_pool,
                       a.v_pool, a.cu, a.seq_len, a.prefix_len, a.page_table, a.max_pages, a.n_seq, a.n_tokens, a.n_q, a.n_kv, a.n_pool_pages,
                       p.row_blocks, p.more_rows, p.parts, p.min_parts, scale_log2e, part, part_ml);
    LAPS_LAUNCH_CHECK();
    const int rows = (a.n_tokens + a.n_seq - 1) / a.n_seq;   // of a sequence, in the mean
    if (p.parts > FEW_PARTS) {
        hipLaunchKernelGGL(attn_rows_merge_kernel<HD>, dim3(a.n_q * a.n_seq, rows < 64 ? rows : 64), dim3(8 * HD / 4), 0, s, a.out, part, part_ml,
                           a.cu, a.seq_len, a.prefix_len, a.max_pages, a.n_tokens, a.n_q, p.parts, p.min_parts);
        LAPS_LAUNCH_CHECK();
    } else if (p.parts > 1) {
        const long wgs = ((long)rows * a.n_q * HD / 4 + FEW_THREADS - 1) / FEW_THREADS;
        hipLaunchKernelGGL(attn_rows_merge_few_kernel<HD>, dim3(a.n_seq, wgs < 4096 ? wgs : 4096), dim3(FEW_THREADS), 0, s, a.out, part, part_ml,
                           a.cu, a.seq_len, a.prefix_len, a.max_pages, a.n_tokens, a.n_q, p.parts, p.min_parts);
        LAPS_LAUNCH_CHECK();
    }
    return LAPS_OK;
}

}  // namespace

// Blocks of 128 or 256 rows read and unpack the keys once for all of them, but pay for their padding, their longer fill and their
// work-item table; here every 32 rows unpack them again.  This kernel / blocks, graph replays, us: 32B, 16 sequences of 4 / 16 / 64 / 96
// tokens over 2048 keys 18 / 31 / 73 / 109 and 37 / 44 / 80 / 90 (128 to 1920 workgroups), 64 of 8 / 16 / 24 over 2000 58 / 84 / 111 and
// 80 / 88 / 94 (1024 to 2048), of 8 / 16 over 300 22 / 30 and 21 / 24; one of 128 over 16000 70 and 100 (160).
// Where the rule is off: it does not look at the keys, and the largest launches it takes lose over long ones (32B, 800 tokens over 4000 /
// 16000 / 64000 keys 97 / 312 / 1180 and 100 / 282 / 1013; 7B, 1170 tokens 104 / 315 / 1175 and 108 / 288 / 1030; 32B, 16 turns of 40 over
// 16000 323 and 262, 4 of 200 318 and 276).  Fewer than 256 workgroups of 128 rows have no blocks to go to: over bf16 pools their key ranges are
// split.  And rows count by their mean: a long turn among single tokens is walked block after block by the few workgroups of
// a sequence (32B, 95 tokens over 512 to 8100 keys 98 us, a turn of 350 over 4000 65, both in one call 1620, in blocks 363; 7B,
// 127 tokens 72, a turn of 900 100, both 3008, in blocks 334).  8 bits, the same lengths: 165, 72 and 1011; 131, 119 and 1992; where the
// mean is up to 16 rows there are no surplus workgroups either (7B, 239 tokens over 512 to 4096 keys 109, a turn of 300 over 4000 53, both 3532).
// Two calls, one for the tokens and one for the turn, take the sum of theirs.
// 8 bits, this kernel / blocks: 32B, 16 sequences of 17 to 64 tokens over 512 to 4096 keys 78 / 81 us, 16 of 64 over 2048 76 / 81, 64 of 8 / 16 /
// 32 over 2000 71 / 94 / 144 and 87 / 95 / 152, 4 of 200 over 16000 359 / 294; 7B, 12 of 60 to 120 over 100 to 3000 75 / 72.
bool laps_attn_takes_rows(int n_seq, int n_tokens, int n_q, int n_kv) {
    const long rows = (long)n_tokens * (n_q / n_kv), blocks = (rows + 32L * n_seq - 1) / (32L * n_seq);
    return rows <= 16L * n_seq || blocks * n_seq * n_kv <= 1024;
}

RowsPlan laps_attn_rows_plan(int bits, int n_seq, int n_tokens, int n_q, int n_kv, int max_pages) {
    const long rows = (long)n_tokens * (n_q / n_kv);
    const int tiles = rows > 16L * n_seq ? 2 : 1;
    long blocks = (rows + 16L * tiles * n_seq - 1) / (16L * tiles * n_seq);
    const long most = (1L << 20) / ((long)n_seq * n_kv);   // a grid of a million workgroups at most; they walk the blocks that are left
    blocks = blocks < most ? blocks : (most > 1 ? most : 1);
    const long rounds = ((long)max_pages * LAPS_PAGE + LAPS_KV4_ROUND - 1) / LAPS_KV4_ROUND;   // of the longest sequence the table holds
    // One workgroup a place on the chip where the sequences are alike (3 or 2 are resident a unit; with 32 rows one is better than two
    // with their merge); more parts where the table allows sequences long enough for the longest one to outlast the others.  32B, 64
    // tokens over 4096 keys each, 1 / 2 / 4 parts 47.8 / 51.3 / 58 us; over 512 to 8191 70.1 / 68.3 / 72, up to 3 by length 64.7; 96 over
    // 16 to 1300 1 / 2 parts 20.5 / 26.2.  16 times 8 tokens over 2048 keys 1 / 2 / 3 parts 25.9 / 25.2 / 29.0; 7B, 20 times 8 to 40 over
    // 64 to 10000 1 / 2 parts 86 / 67.
    // Tables of up to 8 rounds: one launch without a merge takes no longer (one token over 900 keys 9.0 us in 1 part, 9.3 in 8; 16 tokens
    // over 500 keys 7.6 and 10.7).
    // The caps on the longest sequence's parts (rounds / 16, / 10) are coarse: 14B, 16 times 4 tokens over 4000 / 8000 / 16000 keys take 26.3 /
    // 37.9 / 62.2 by the rule (3 / 6 / 8 parts), 23.8 / 33.1 / 54.4 in 4 parts, 23.8 / 36.1 / 61.1 in 2, 39.8 / 49.6 / 71.6 in 12; 32B, 32 tokens
    // over 2000 / 4000 / 8000 19.2 / 29.5 / 54.7 by the rule, 15.9 / 27.0 / 50.5 in 1.  One long history among short ones keeps
    // the parts that the batch leaves it: 32B, 95 tokens over 100 to 2000 keys and one over 100000 274 in 2 parts, 114 in 16, with
    // which the same table without a long one takes 76 instead of 42.
    // 8 bits: as many workgroups again for the longer turns of a ragged batch, ahead of the others, where they find nothing to do in an even
    // one.  With / without: 32B, five draws of 16 turns of 17 to 64 tokens over 512 to 4096 keys 84 / 82, 86 / 104, 93 / 97, 90 / 104, 70 / 75 us, 12 of
    // 9 to 100 over 100 to 3000 59 / 68, 40 of 4 to 20 over 20 to 2000 45 / 52; 7B, 20 of 8 to 40 over 64 to 10000 103 / 117; even ones the same but
    // 64 of 8 tokens over 2000 keys 78 / 74.  Behind the others 89, 93, 91, 85, 61 and 60, 46, 109; beside the blocks of the same keys they
    // cost even batches half their time (64 of 8 over 2000 110); three and four times as many are like two.
    const int more_rows = bits == 8 && tiles == 2 && n_seq > 1 && blocks * n_seq * n_kv <= (1 << 18) ? 2 : 1;
    if (rounds <= 8) return {tiles, (int)blocks, more_rows, 1, 1};
    const long units = blocks * n_seq * n_kv, places = tiles == 1 ? (bits == 8 ? 512 : 768) : 256;
    auto within = [](long n, long most) { return n < most ? (n > 1 ? n : 1) : most; };
    const long min_parts = within(within(places / units, rounds / 2), MAX_PARTS);
    // 8 bits, one block of rows (two workgroups are resident a unit), at most 1 / 1024 / 1536 workgroups over all parts: 32B, 64 tokens over
    // 4096 keys each 88 / 98 / 98 us, over 512 to 8191 117 / 128 / 114; 14B, 96 over 512 to 8191 164 / 164 / 180; 32B, 40 over 100 to 16000
    // 163 / 127 / 141; two over 100000 in 51 by each.
    const long more = tiles == 2 ? 1024 : bits == 4 ? 1536 : units < 512 ? 1024 : 1;
    const long parts = within(within(more / units, rounds / (tiles == 1 ? 16 : 10)), MAX_PARTS);
    return {tiles, (int)blocks, more_rows, (int)(parts > min_parts ? parts : min_parts), (int)min_parts};
}

size_t laps_attn_rows_bytes(const RowsPlan& p, int n_tokens, int n_q, int hd) {
    return p.parts > 1 ? (size_t)n_tokens * n_q * p.parts * (hd + 2) * sizeof(float) : 0;
}

int laps_launch_attn_rows(const RowsAttn& a, const RowsPlan& p, float* partial, hipStream_t s) {
    auto launch = a.hd == 128 ? (a.bits == 8 ? launch_rows<128, true> : launch_rows<128, false>) : (a.bits == 8 ? launch_rows<64, true> : launch_rows<64, false>);
    return launch(a, p, partial, s);
}
