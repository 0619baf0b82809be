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
// Four waves of a workgroup take every fourth pair of pages and add up in LDS.  Few sequences over long keys: a sequence's keys go out
// in parts of equal length to workgroups of their own, and a second kernel adds those, in order.
#include "kv4.h"

#include <climits>
#include <type_traits>

namespace {

constexpr int WAVES = 4;
constexpr int STEP = 2 * LAPS_PAGE;   // keys a wave takes at a time
constexpr int MAX_PARTS = 64;
constexpr float RESCALE_SLACK = 8.f;  // log2; see below

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

// Parts of a sequence's keys: of equal length, at least one step a wave each.
__device__ __forceinline__ int part_steps(int kv_len, int parts, int* used) {
    const int steps = (kv_len + STEP - 1) / STEP, rounds = (steps + WAVES - 1) / WAVES;
    const int n = rounds < parts ? rounds : parts, each = (rounds + n - 1) / n;
    *used = (rounds + each - 1) / each;
    return each * WAVES;
}

// One step's codes and scales as they come from the pools.
template <int HD>
struct Piece {
    unsigned k[2][HD / 32], ks[2];   // [page]: HD / 4 codes of key i, their group's scale byte
    u32x4 v[2];                      // eight codes (HD 64: four of them used) of keys 4g .. 4g + 3
    unsigned vs[2];                  // those keys' scale bytes
};

template <int HD>
__global__ __launch_bounds__(WAVES * 64) void attn_rows_kernel(
    const bf16_t* __restrict__ q, bf16_t* __restrict__ out, const byte_t* __restrict__ k_pool, const byte_t* __restrict__ v_pool,
    const int* __restrict__ cu, const int* __restrict__ seq_len, const int* __restrict__ prefix_len,
    const int* __restrict__ page_table, int max_pages, int n_tokens, int n_q, int n_kv, int n_pool_pages, int row_blocks, int parts,
    float scale_log2e, float* __restrict__ part_o, float* __restrict__ part_ml) {
    constexpr int KS = HD / 32;        // matrix instructions of a page's scores
    constexpr int DL = HD / 16;        // head_dim indices of a lane of V, and of the result's 16 rows each
    constexpr int BLOCK = kv4_block(HD), CODES = kv4_codes(HD);
    __shared__ __align__(16) float red_o[WAVES][16][HD + 4];
    __shared__ float red_ml[WAVES][2][16];

    const int G = n_q / n_kv, kvh = blockIdx.x % n_kv, rest = blockIdx.x / n_kv, rb0 = rest % row_blocks, seq = rest / row_blocks, part = blockIdx.y;
    SeqRange r;
    if (!seq_range(seq, cu, seq_len, prefix_len, n_tokens, max_pages, &r)) return;
    const int n_rows = r.L * G, kv_len = r.H + r.L;
    int used;
    const int each = part_steps(kv_len, parts, &used);
    if (part >= used) return;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), i = lane & 15, g = lane >> 4;
    const int need = (kv_len + LAPS_PAGE - 1) / LAPS_PAGE, n_pages = need < max_pages ? need : max_pages;
    const int* pt = page_table + (size_t)seq * max_pages;
    const int v_chunk = HD == 128 ? i : i >> 1, v_group = i / (KV4_GROUP / DL), o_group = g * 4 * DL / KV4_GROUP;

    for (int rb = rb0; rb * 16 < n_rows; rb += row_blocks) {
        const int row = rb * 16 + i, rc = row < n_rows ? row : n_rows - 1, tq = rc / G;
        const int limit = r.H + tq;                                            // last key this lane's row sees
        const int last_row = rb * 16 + 15 < n_rows ? rb * 16 + 15 : n_rows - 1;
        const int vis_min = r.H + rb * 16 / G, kv_end = r.H + last_row / G + 1;  // seen by every row, by the last row
        bf16x8 qf[KS];
        {
            const u32x4* qp = reinterpret_cast<const u32x4*>(q + (size_t)(r.rs + tq) * n_q * HD + (size_t)(kvh * G + rc - tq * G) * HD);
#pragma unroll
            for (int kk = 0; kk < KS; ++kk) qf[kk] = __builtin_bit_cast(bf16x8, qp[g * KS + kk]);
        }
        f32x4 o[DL];
#pragma unroll
        for (int j = 0; j < DL; ++j) o[j] = f32x4{0.f, 0.f, 0.f, 0.f};
        float m_run = -INFINITY, l_run = 0.f;   // reference in log2 units (the same in the four lanes of a row), this lane's sum
        int nan_key = INT_MAX;                  // first key with a NaN group in this lane's V_group, where not every row sees it

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
        };
        auto load = [&](int n, Piece<HD>& x) {
            if ((n & 31) == 0) fetch_ids(n);
#pragma unroll
            for (int p = 0; p < 2; ++p) {
                const int page = __builtin_amdgcn_readlane(ids, 2 * (n & 31) + p);
                const size_t at = ((size_t)page * n_kv + kvh) * BLOCK;
                const byte_t *kb = k_pool + at, *vb = v_pool + at;
                if constexpr (HD == 128) {
                    const u32x4 w = reinterpret_cast<const u32x4*>(kb)[i * 4 + g];
#pragma unroll
                    for (int kk = 0; kk < 4; ++kk) x.k[p][kk] = w[kk];
                    x.ks[p] = kb[CODES + i * 4 + g];
                } else {
                    const u32x2 w = reinterpret_cast<const u32x2*>(kb)[i * 4 + g];
                    x.k[p][0] = w.x;
                    x.k[p][1] = w.y;
                    x.ks[p] = kb[CODES + i * 2 + (g >> 1)];
                }
                x.v[p] = reinterpret_cast<const u32x4*>(vb)[v_chunk * 4 + g];
                x.vs[p] = reinterpret_cast<const unsigned*>(vb + CODES)[v_group * 4 + g];
            }
        };
        auto compute = [&](int n, Piece<HD>& x) {
            const int key0 = (s_begin + n * WAVES) * STEP;
            f32x4 s[2];
#pragma unroll
            for (int p = 0; p < 2; ++p) {
                const float ks = kv4_scale<0>(x.ks[p]);
                s[p] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int kk = 0; kk < KS; ++kk)
                    s[p] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kv4_eight(x.k[p][kk], ks)), qf[kk], s[p], 0, 0, 0);
            }
            if (key0 + STEP - 1 > vis_min) {   // some row does not see all of these keys
#pragma unroll
                for (int p = 0; p < 2; ++p) {
                    const int k4 = key0 + p * LAPS_PAGE + 4 * g;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        if (k4 + e > limit) s[p][e] = -INFINITY;   // whatever it was, NaN included
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
            float mx = fmaxf(fmaxf(fmaxf(s[0].x, s[0].y), fmaxf(s[0].z, s[0].w)), fmaxf(fmaxf(s[1].x, s[1].y), fmaxf(s[1].z, s[1].w))) * scale_log2e;
            // The reference that the exponentials subtract follows the row's maximum only when that has grown by more than
            // RESCALE_SLACK (weights stay below 2^RESCALE_SLACK; the quotient does not depend on it): the exchange between a row's four
            // lanes and the rescale of O are rare.
            if (__builtin_amdgcn_ballot_w64(mx > m_run + RESCALE_SLACK) != 0) {
                mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
                mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
                const float m_new = fmaxf(m_run, mx);
                const float alpha = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m_run - m_new);
                l_run *= alpha;
#pragma unroll
                for (int j = 0; j < DL; ++j) o[j] *= alpha;
                m_run = m_new;
            }
            const float m_sub = m_run == -INFINITY ? 0.f : m_run;   // a row that has seen no key yet
            bf16x8 pf;
#pragma unroll
            for (int p = 0; p < 2; ++p)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float w = __builtin_amdgcn_exp2f(__builtin_fmaf(s[p][e], scale_log2e, -m_sub));
                    l_run += w;
                    pf[4 * p + e] = (__bf16)w;
                }
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
                o[2 * b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, lo), pf, o[2 * b], 0, 0, 0);
                o[2 * b + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, hi), pf, o[2 * b + 1], 0, 0, 0);
            };
            pair_of_keys(std::integral_constant<int, 0>{});
            pair_of_keys(std::integral_constant<int, 1>{});
            if constexpr (HD == 128) {
                pair_of_keys(std::integral_constant<int, 2>{});
                pair_of_keys(std::integral_constant<int, 3>{});
            }
        };
        // the next step is on its way while this one is worked on; two buffers in turn
        Piece<HD> a, b;
        if (n_steps > 0) load(0, a);
        for (int n = 0; n < n_steps; n += 2) {
            if (n + 1 < n_steps) load(n + 1, b);
            compute(n, a);
            if (n + 1 >= n_steps) break;
            if (n + 2 < n_steps) load(n + 2, a);
            compute(n + 1, b);
        }

        // ---- NaN groups of keys that not every row sees
        nan_key = min(nan_key, __shfl_xor(nan_key, 16, 64));
        nan_key = min(nan_key, __shfl_xor(nan_key, 32, 64));
        if (__shfl(nan_key, o_group * (KV4_GROUP / DL), 64) <= limit) {
#pragma unroll
            for (int j = 0; j < DL; ++j) o[j] += __builtin_nanf("");
        }
        // ---- the four waves' results: lane (i, g) holds row i, head_dim indices 4 DL g + DL e + j
        l_run += __shfl_xor(l_run, 16, 64);
        l_run += __shfl_xor(l_run, 32, 64);
        __syncthreads();   // the row block before is read
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int j = 0; j < DL; j += 4)
                *reinterpret_cast<f32x4*>(&red_o[wave][i][(4 * g + e) * DL + j]) = f32x4{o[j][e], o[j + 1][e], o[j + 2][e], o[j + 3][e]};
        if (g == 0) {
            red_ml[wave][0][i] = m_run;
            red_ml[wave][1][i] = l_run;
        }
        __syncthreads();
        constexpr int PER = 16 * HD / (WAVES * 64);   // values a thread finishes
        const int fr = tid / (HD / PER), fd = tid % (HD / PER) * PER, frow = rb * 16 + fr;
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

// Adds the parts of a sequence's keys: out = sum_p 2^(m_p - M) O_p / sum_p 2^(m_p - M) l_p, M = max_p m_p, each of 8 groups of
// HD / 4 lanes a run of the parts, the groups in order.  A workgroup takes one query head of one sequence, a row after the other.
template <int HD>
__global__ __launch_bounds__(8 * HD / 4) void attn_rows_merge_kernel(bf16_t* __restrict__ out, const float* __restrict__ part_o,
                                                                     const float* __restrict__ part_ml, const int* __restrict__ cu,
                                                                     const int* __restrict__ seq_len,
                                                                     const int* __restrict__ prefix_len, int max_pages,
                                                                     int n_tokens, int n_q, int parts) {
    constexpr int LANES = HD / 4, GROUPS = 8;
    __shared__ float weight[MAX_PARTS], sum[MAX_PARTS];
    __shared__ f32x4 red[GROUPS][LANES];
    const int head = blockIdx.x % n_q, seq = blockIdx.x / n_q, tid = threadIdx.x, c = tid % LANES, grp = tid / LANES;
    SeqRange r;
    if (!seq_range(seq, cu, seq_len, prefix_len, n_tokens, max_pages, &r)) return;
    int used;
    part_steps(r.H + r.L, parts, &used);
    if (used == 1) return;   // written by the attention kernel
    for (int t = blockIdx.y; t < r.L; t += gridDim.y) {
        const size_t at = ((size_t)(r.rs + t) * n_q + head) * parts;
        if (tid < 64) {   // parts <= 64: one a lane
            const float m = tid < used ? part_ml[(at + tid) * 2] : -INFINITY, l = tid < used ? part_ml[(at + tid) * 2 + 1] : 0.f;
            float m_all = m;
#pragma unroll
            for (int k = 32; k > 0; k >>= 1) m_all = fmaxf(m_all, __shfl_xor(m_all, k, 64));
            const float f = __builtin_amdgcn_exp2f(m - (m_all == -INFINITY ? 0.f : m_all));
            weight[tid] = f;
            sum[tid] = f * l;
        }
        __syncthreads();
        f32x4 acc = {0.f, 0.f, 0.f, 0.f};
        const int run = (used + GROUPS - 1) / GROUPS, p1 = (grp + 1) * run < used ? (grp + 1) * run : used;
#pragma unroll 8
        for (int p = grp * run; p < p1; ++p) acc += weight[p] * reinterpret_cast<const f32x4*>(part_o + (at + p) * HD)[c];
        red[grp][c] = acc;
        __syncthreads();
        if (grp == 0) {
            float l = 0.f;
            for (int p = 0; p < used; ++p) l += sum[p];
#pragma unroll
            for (int k = 1; k < GROUPS; ++k) acc += red[k][c];
            const float inv = 1.f / l;
            u32x2 w;
            w.x = pack_bf16x2(acc.x * inv, acc.y * inv);
            w.y = pack_bf16x2(acc.z * inv, acc.w * inv);
            *reinterpret_cast<u32x2*>(out + ((size_t)(r.rs + t) * n_q + head) * HD + 4 * c) = w;
        }
        __syncthreads();
    }
}

template <int HD>
int launch_rows(const Kv4Attn& a, const Kv4RowsPlan& p, float* part, hipStream_t s) {
    const float scale_log2e = 1.4426950408889634f / sqrtf((float)HD);
    float* part_ml = part ? part + (size_t)a.n_tokens * a.n_q * p.parts * HD : nullptr;
    hipLaunchKernelGGL(attn_rows_kernel<HD>, dim3(a.n_kv * p.row_blocks * a.n_seq, p.parts), dim3(WAVES * 64), 0, s, a.q, a.out, a.k_pool,
                       a.v_pool, a.cu, a.seq_len, a.prefix_len, a.page_table, a.max_pages, a.n_tokens, a.n_q, a.n_kv, a.n_pool_pages,
                       p.row_blocks, p.parts, scale_log2e, part, part_ml);
    LAPS_LAUNCH_CHECK();
    if (p.parts > 1) {
        const int rows = (a.n_tokens + a.n_seq - 1) / a.n_seq;
        hipLaunchKernelGGL(attn_rows_merge_kernel<HD>, dim3(a.n_q * a.n_seq, rows < 64 ? rows : 64), dim3(8 * HD / 4), 0, s, a.out, part, part_ml,
                           a.cu, a.seq_len, a.prefix_len, a.max_pages, a.n_tokens, a.n_q, p.parts);
        LAPS_LAUNCH_CHECK();
    }
    return LAPS_OK;
}

}  // namespace

// Blocks of 128 rows read and unpack the keys once for all of them, but pay for 128 whatever they hold, and for their work-item
// table.  This kernel against blocks, graph replays, us: 32B, 16 sequences over 2048 keys, 4 / 6 / 8 / 16 tokens each 29 / 32 / 43 / 63
// and 36 / 37 / 42 / 42; one over 4000 keys, 1 / 8 / 16 tokens 9.6 / 16.4 / 22.7 and 16.8 / 17.6 / 18.5.
bool laps_kv4_takes_rows(int n_seq, int n_tokens, int n_q, int n_kv) {
    return (long)n_tokens * (n_q / n_kv) <= 32L * n_seq;
}

Kv4RowsPlan laps_kv4_rows_plan(int n_seq, int n_tokens, int n_q, int n_kv, int max_pages) {
    const long rows = (long)n_tokens * (n_q / n_kv);
    long blocks = (rows + 16L * n_seq - 1) / (16L * n_seq);
    const long most = (1L << 20) / ((long)n_seq * n_kv);   // a grid of a million workgroups at most; they walk the blocks that are left
    blocks = blocks < most ? blocks : (most > 1 ? most : 1);
    const long rounds = ((long)max_pages * LAPS_PAGE + STEP * WAVES - 1) / (STEP * WAVES);   // of the longest sequence the table holds
    long parts = (2048 + blocks * n_seq * n_kv - 1) / (blocks * n_seq * n_kv);
    parts = parts < rounds ? parts : rounds;
    parts = parts < MAX_PARTS ? parts : MAX_PARTS;
    return {(int)blocks, (int)(parts < 1 ? 1 : parts)};
}

size_t laps_kv4_rows_bytes(const Kv4RowsPlan& p, int n_tokens, int n_q, int hd) {
    return p.parts > 1 ? (size_t)n_tokens * n_q * p.parts * (hd + 2) * sizeof(float) : 0;
}

int laps_launch_kv4_rows(const Kv4Attn& a, const Kv4RowsPlan& p, float* partial, hipStream_t s) {
    return a.hd == 128 ? launch_rows<128>(a, p, partial, s) : launch_rows<64>(a, p, partial, s);
}
