// Token-major bf16 K/V <-> the 4-bit pools.
//
// A group of 32 values x along head_dim becomes a power of two 2^e and 32 four-bit floats x / 2^e; the way back is one product
// that is exact in bf16.  Nothing but the two copies has to move: 2 * 2 * (1 + 17/64) bytes a value pair, no arithmetic to speak of.
//
// One workgroup per (page of a sequence, kv head), 2 * head_dim threads, each eight values of K and eight of V.  K lies
// [token][head_dim] on both sides, so consecutive threads take consecutive chunks and a group is four neighbouring lanes.  V's
// codes lie [head_dim / 8][16 tokens][8 values] (what a lane of the attention reads is four tokens of the same eight head_dim
// indices).  What is written goes out in whole lines: on the way in thread t takes token t % 16 of chunk t / 16 (the pool side in
// order, the token side in 64-byte pieces, a group four lanes 16 apart), on the way out V is assigned as K is and the pool's dwords
// are picked up from all over their kilobyte.  No LDS, no barrier.
//
// Token-major rows that the L2 caches do not hold stream past them.  37 k tokens of 8 heads x 128 (193 MB), cold: written 39.3 us, rows
// read past the caches 35.3 (5.5 TB/s; a large copy 5.1); read back with V as on the way in 43.7, as K 39.3, and rows written past the
// caches 30.8 (6.3 TB/s).  A few hundred tokens: the time of a launch, all ways.
#include "kv4.h"

#include <type_traits>

namespace {

// Work items as in the mover of the bf16 pools: the first item of sequence s is cu[s] / 16 + 2 s (a run of n tokens touches at most
// n / 16 + 2 pages), items that no page needs return at once.
template <int HD, bool SCATTER, bool STREAM>
__global__ __launch_bounds__(2 * HD) void kv4_move_kernel(const int* __restrict__ cu, const int* __restrict__ start_pos,
                                                          const int* __restrict__ page_table, u32x4* __restrict__ k_tok,
                                                          u32x4* __restrict__ v_tok, unsigned char* __restrict__ k_pool,
                                                          unsigned char* __restrict__ v_pool, int n_seq, int n_tokens,
                                                          int max_pages, int n_kv, int n_pool_pages) {
    constexpr int CPR = HD / 8, GROUPS = HD / KV4_GROUP, CODES = kv4_codes(HD);
    const int item = blockIdx.x, head = blockIdx.y, tid = threadIdx.x;
    auto first_item = [&](int s) { return cu[s] / LAPS_PAGE + 2 * s; };
    int lo = 0, hi = n_seq;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (first_item(mid) <= item) lo = mid; else hi = mid;
    }
    // whatever the arrays hold: tokens stay in [0, n_tokens), pages in the table, page ids in the pool
    const int c0 = cu[lo], c1 = cu[lo + 1], t1 = c1 < n_tokens ? c1 : n_tokens;
    if (c0 < 0 || c0 >= t1 || item < first_item(lo)) return;
    const long shift = (long)start_pos[lo] - c0;                       // position of a token = its index + shift
    const long page_index = ((c0 + shift) >> 4) + (item - first_item(lo));
    const long a = page_index * LAPS_PAGE - shift;                     // token at offset 0 of the page, if the sequence has it
    if (a >= t1 || page_index < 0 || page_index >= max_pages) return;
    const int off0 = a < c0 ? (int)(c0 - a) : 0, off1 = t1 - a < LAPS_PAGE ? (int)(t1 - a) : LAPS_PAGE;
    const int page = page_table[(size_t)lo * max_pages + page_index];
    if (page < 0 || page >= n_pool_pages) return;                      // unset table entry, or not a page of the pool
    const size_t block = ((size_t)page * n_kv + head) * kv4_block(HD);
    unsigned char *kb = k_pool + block, *vb = v_pool + block;
    const int k_off = tid / CPR, k_c = tid % CPR, v_off = SCATTER ? tid % LAPS_PAGE : k_off, v_c = SCATTER ? tid / LAPS_PAGE : k_c;
    const bool k_mine = k_off >= off0 && k_off < off1, v_mine = v_off >= off0 && v_off < off1;
    const size_t k_at = ((size_t)(a + k_off) * n_kv + head) * CPR + k_c, v_at = ((size_t)(a + v_off) * n_kv + head) * CPR + v_c;
    unsigned char *k_scale = kb + CODES + k_off * GROUPS + k_c / 4, *v_scale = vb + CODES + (v_c / 4) * LAPS_PAGE + v_off;
    auto take = [](const u32x4* from) { return STREAM ? __builtin_nontemporal_load(from) : *from; };
    auto put = [](u32x4 x, u32x4* to) {
        if (STREAM) __builtin_nontemporal_store(x, to);
        else *to = x;
    };
    if (SCATTER) {
        u32x4 k = {0u, 0u, 0u, 0u}, v = {0u, 0u, 0u, 0u};
        if (k_mine) k = take(k_tok + k_at);
        if (v_mine) v = take(v_tok + v_at);
        // the lanes of a group are all `mine` or none
        unsigned ka = kv4_amax(k), va = kv4_amax(v);
#pragma unroll
        for (int i = 1; i < 4; i <<= 1) {
            const unsigned ko = __shfl_xor(ka, i, 64), vo = __shfl_xor(va, 16 * i, 64);
            ka = ko > ka ? ko : ka;
            va = vo > va ? vo : va;
        }
        const int ks = kv4_scale_byte(ka), vs = kv4_scale_byte(va);
        if (k_mine) {
            reinterpret_cast<unsigned*>(kb)[tid] = kv4_codes_of(k, ks);
            if (k_c % 4 == 0) *k_scale = (unsigned char)ks;
        }
        if (v_mine) {
            reinterpret_cast<unsigned*>(vb)[tid] = kv4_codes_of(v, vs);
            if (v_c % 4 == 0) *v_scale = (unsigned char)vs;
        }
    } else {
        const unsigned kc = reinterpret_cast<const unsigned*>(kb)[tid], vc = reinterpret_cast<const unsigned*>(vb)[v_c * LAPS_PAGE + v_off];
        const float ks = kv4_scale<0>(*k_scale), vs = kv4_scale<0>(*v_scale);
        if (k_mine) put(kv4_eight(kc, ks), k_tok + k_at);
        if (v_mine) put(kv4_eight(vc, vs), v_tok + v_at);
    }
}

}  // namespace

int laps_launch_kv4_move(bool scatter, int n_seq, int n_tokens, const int* cu, const int* start_pos, const int* page_table,
                         int max_pages, void* k_tok, void* v_tok, void* k_pool, void* v_pool, int n_kv, int hd, int n_pool_pages,
                         hipStream_t s) {
    if (n_tokens == 0) return LAPS_OK;
    const dim3 grid(n_tokens / LAPS_PAGE + 2 * n_seq, n_kv);
    const bool stream = (size_t)n_tokens * n_kv * hd * 2 * sizeof(bf16_t) > ((size_t)32 << 20);   // eight L2 caches of 4 MiB
    auto pick = [&](auto HD) {
        constexpr int D = decltype(HD)::value;
        return scatter ? (stream ? kv4_move_kernel<D, true, true> : kv4_move_kernel<D, true, false>)
                       : (stream ? kv4_move_kernel<D, false, true> : kv4_move_kernel<D, false, false>);
    };
    auto kern = hd == 128 ? pick(std::integral_constant<int, 128>{}) : pick(std::integral_constant<int, 64>{});
    hipLaunchKernelGGL(kern, grid, dim3(2 * hd), 0, s, cu, start_pos, page_table, static_cast<u32x4*>(k_tok),
                       static_cast<u32x4*>(v_tok), static_cast<unsigned char*>(k_pool), static_cast<unsigned char*>(v_pool), n_seq,
                       n_tokens, max_pages, n_kv, n_pool_pages);
    LAPS_LAUNCH_CHECK();
    return LAPS_OK;
}
