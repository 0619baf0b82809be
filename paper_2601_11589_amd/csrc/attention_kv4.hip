// Attention over the 4-bit cache for few query rows a sequence: single tokens, drafted tokens, the shortest turns.
//
//   O = softmax(Q K^T / sqrt(hd)) V over the cached keys, row t of a sequence seeing keys <= H + t
//
// One pass over the keys with a running maximum and sum a row.  What bounds it is the cache: 8.5 * hd bytes of K and as many of V for
// 16 keys of a kv head, and 4 * 16 * hd flops for each of the G query heads that share them.  So nothing is staged: a wave walks the
// keys 32 at a time (two pages), and every load is one 16-byte piece a lane, 1 KB of a page a wave, straight into the
// operand registers of 16x16x32 matrix instructions:
//
//   S^T = K Q^T   lane (i, g) = (lane % 16, lane / 16) holds key i and head_dim indices hd/4 g .. hd/4 g + hd/4 - 1: its piece of the page
//                 [16 keys][hd / 2 bytes].  Which index is which of the instruction's 32 does not matter as long as Q's registers agree.
//   O^T = V^T P^T the result above leaves lane (i, g) with row i's scores of keys 4g .. 4g + 3 of both pages; those eight are its
//                 share of the second product's 32 keys, and V's pages are laid out for that: [hd / 8][16 keys][8 values], four keys of
//                 the same eight (hd 64: four) head_dim indices a lane.  No value changes lanes.
//
// Codes become bf16 operands exactly (one instruction a pair, the group's scale included; two permutes a pair of V's to bring keys
// side by side).  The query rows are the G heads of a kv head for each of the sequence's new tokens, 16 a block.
// Weights are rounded to bf16, which the second product takes, and their sum is that of the rounded ones, so that they add up to one; scores,
// sums, O and partial results are float32.  That makes outputs 1.1 to 1.4 times as far from 64 bits as float32 weights would (1.8e-3 to
// 2.3e-3 of the output against 1.6e-3 to 1.7e-3, most of it the output's own rounding), the same as over bf16 pools.
// Four waves of a workgroup take every fourth pair of pages and add up in LDS.  Few sequences over long keys: a sequence's keys go out
// in parts of equal length to workgroups of their own, and a second kernel adds those, in order.
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

__device__ __forceinline__ int part_steps(int kv_len, int max_pages, int parts, int min_parts, int* used) {
    return laps_kv4_part_rounds(kv_len, max_pages, parts, min_parts, used) * WAVES;
}

// One step's codes and scales as they come from the pools.
template <int HD>
struct Piece {
    unsigned k[2][HD / 32], ks[2];   // [page]: HD / 4 codes of key i, the dword with their group's scale byte
    u32x4 v[2];                      // eight codes (HD 64: four of them used) of keys 4g .. 4g + 3
    unsigned vs[2];                  // those keys' scale bytes
};

// NR: blocks of 16 rows that share what is read and unpacked.
template <int HD, int NR>
__global__ __launch_bounds__(WAVES * 64, NR == 1 ? 3 : 2) void attn_rows_kernel(
    const bf16_t* __restrict__ q, bf16_t* __restrict__ out, const byte_t* __restrict__ k_pool, const byte_t* __restrict__ v_pool,
    const int* __restrict__ cu, const int* __restrict__ seq_len, const int* __restrict__ prefix_len,
    const int* __restrict__ page_table, int max_pages, int n_seq, int n_tokens, int n_q, int n_kv, int n_pool_pages, int row_blocks, int parts,
    int min_parts, float scale_log2e, float* __restrict__ part_o, float* __restrict__ part_ml) {
    constexpr int KS = HD / 32;        // matrix instructions of a page's scores
    constexpr int DL = HD / 16;        // head_dim indices of a lane of V, and of the result's 16 rows each
    constexpr int BLOCK = kv4_block(HD), CODES = kv4_codes(HD), ROWS = 16 * NR;
    __shared__ __align__(16) float red_o[WAVES][16][HD + 4];
    __shared__ float red_ml[WAVES][2][16];

    // Workgroup b runs on XCD b % 8.  The kv heads of a (sequence, part, row block) go to one XCD side by side: a page's heads are
    // neighbours in memory and a block is 8.5 (4.25) lines of 128 bytes, so that each fetches a line that the next one needs too.
    const int G = n_q / n_kv, kvh = blockIdx.x / 8 % n_kv, rest = blockIdx.x / 8 / n_kv * 8 + blockIdx.x % 8;
    const int rb0 = rest % row_blocks, part = rest / row_blocks % parts, seq = rest / row_blocks / parts;
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
    const int v_chunk = HD == 128 ? i : i >> 1, v_group = i / (KV4_GROUP / DL), o_group = g * 4 * DL / KV4_GROUP;

    for (int rb = rb0; rb * ROWS < n_rows; rb += row_blocks) {
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
            for (int kk = 0; kk < KS; ++kk) qf[a][kk] = __builtin_bit_cast(bf16x8, qp[g * KS + kk]);
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
        // Up to 16 rows a sequence: keys are read once and past the caches, 2.3 GB 418 -> 378 us (6.0 TB/s; 280 MB that the memory-side cache
        // held from the call before 52 -> 58).  More rows: other blocks of theirs read the same keys.
        auto codes = [](const auto* from) { return NR == 1 ? __builtin_nontemporal_load(from) : *from; };
        auto load = [&](int n, Piece<HD>& x) {
            if ((n & 31) == 0) fetch_ids(n);
#pragma unroll
            for (int p = 0; p < 2; ++p) {
                const int page = __builtin_amdgcn_readlane(ids, 2 * (n & 31) + p);
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
        };
        auto compute = [&](int n, Piece<HD>& x) {
            const int key0 = (s_begin + n * WAVES) * STEP;
            f32x4 s[NR][2];
#pragma unroll
            for (int p = 0; p < 2; ++p) {
                const float ks = __uint_as_float(__builtin_amdgcn_alignbit(x.ks[p], x.ks[p], k_turn));   // the byte to bits 23 to 30
#pragma unroll
                for (int a = 0; a < NR; ++a) s[a][p] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int kk = 0; kk < KS; ++kk) {
                    const bf16x8 kf = __builtin_bit_cast(bf16x8, kv4_eight(x.k[p][kk], ks));
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
                        const unsigned byte = (x.vs[p] >> (8 * e)) & 255u;
                        if (k4 + e >= kv_len || byte == 255u) {
                            if (k4 + e < kv_len) nan_key = k4 + e < nan_key ? k4 + e : nan_key;
                            x.v[p][e] = 0u;
                            x.vs[p] &= ~(255u << (8 * e));
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
        };
        // The next step is on its way while one is worked on; two buffers in turn.  Past the last step the last one is loaded again:
        // with a branch round the loads every wait would be for all of them.
        if (n_steps > 0) {
            Piece<HD> x, y;
            auto load_at = [&](int n, Piece<HD>& to) { load(n < n_steps ? n : n_steps - 1, to); };
            load_at(0, x);
#pragma unroll
            for (int a = 0; a < NR; ++a)
#pragma unroll
                for (int kk = 0; kk < KS; ++kk) asm volatile("" : "+v"(qf[a][kk]));   // as ids: the loop must find Q arrived
            for (int n = 0;;) {
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

        // ---- NaN groups of keys that not every row sees
        nan_key = min(nan_key, __shfl_xor(nan_key, 16, 64));
        nan_key = min(nan_key, __shfl_xor(nan_key, 32, 64));
        const int nan_from = __shfl(nan_key, o_group * (KV4_GROUP / DL), 64);
#pragma unroll
        for (int a = 0; a < NR; ++a) {
            if (rb * ROWS + 16 * a >= n_rows) break;
            if (nan_from <= limit[a]) {
#pragma unroll
                for (int j = 0; j < DL; ++j) o[a][j] += __builtin_nanf("");
            }
            // ---- the four waves' results: lane (i, g) holds row i, head_dim indices 4 DL g + DL e + j
            l_run[a] += __shfl_xor(l_run[a], 16, 64);
            l_run[a] += __shfl_xor(l_run[a], 32, 64);
            __syncthreads();   // the rows before are read
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int j = 0; j < DL; j += 4)
                    *reinterpret_cast<f32x4*>(&red_o[wave][i][(4 * g + e) * DL + j]) = f32x4{o[a][j][e], o[a][j + 1][e], o[a][j + 2][e], o[a][j + 3][e]};
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

template <int HD>
int launch_rows(const Kv4Attn& a, const Kv4RowsPlan& p, float* part, hipStream_t s) {
    const float scale_log2e = 1.4426950408889634f / sqrtf((float)HD);
    float* part_ml = part ? part + (size_t)a.n_tokens * a.n_q * p.parts * HD : nullptr;
    auto kern = p.row_tiles == 1 ? attn_rows_kernel<HD, 1> : attn_rows_kernel<HD, 2>;
    hipLaunchKernelGGL(kern, dim3((a.n_seq * p.parts * p.row_blocks + 7) / 8 * 8 * a.n_kv), dim3(WAVES * 64), 0, s, a.q, a.out, a.k_pool,
                       a.v_pool, a.cu, a.seq_len, a.prefix_len, a.page_table, a.max_pages, a.n_seq, a.n_tokens, a.n_q, a.n_kv, a.n_pool_pages,
                       p.row_blocks, p.parts, p.min_parts, scale_log2e, part, part_ml);
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
// 127 tokens 72, a turn of 900 100, both 3008, in blocks 334).
bool laps_kv4_takes_rows(int n_seq, int n_tokens, int n_q, int n_kv) {
    const long rows = (long)n_tokens * (n_q / n_kv), blocks = (rows + 32L * n_seq - 1) / (32L * n_seq);
    return rows <= 16L * n_seq || blocks * n_seq * n_kv <= 1024;
}

Kv4RowsPlan laps_kv4_rows_plan(int n_seq, int n_tokens, int n_q, int n_kv, int max_pages) {
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
    if (rounds <= 8) return {tiles, (int)blocks, 1, 1};
    const long units = blocks * n_seq * n_kv, places = tiles == 1 ? 768 : 256;
    auto within = [](long n, long most) { return n < most ? (n > 1 ? n : 1) : most; };
    const long min_parts = within(within(places / units, rounds / 2), MAX_PARTS);
    const long parts = within(within((tiles == 1 ? 1536 : 1024) / units, rounds / (tiles == 1 ? 16 : 10)), MAX_PARTS);
    return {tiles, (int)blocks, (int)(parts > min_parts ? parts : min_parts), (int)min_parts};
}

size_t laps_kv4_rows_bytes(const Kv4RowsPlan& p, int n_tokens, int n_q, int hd) {
    return p.parts > 1 ? (size_t)n_tokens * n_q * p.parts * (hd + 2) * sizeof(float) : 0;
}

int laps_launch_kv4_rows(const Kv4Attn& a, const Kv4RowsPlan& p, float* partial, hipStream_t s) {
    return a.hd == 128 ? launch_rows<128>(a, p, partial, s) : launch_rows<64>(a, p, partial, s);
}
