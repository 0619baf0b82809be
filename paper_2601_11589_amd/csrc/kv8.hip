// Token-major bf16 K/V <-> the 8-bit pools.
//
// A page's 16 tokens of one kv head share a scale 2^e, K and V apart; a value x becomes the 8-bit float x / 2^e.  Tokens come in runs that
// begin and end inside pages, so a run that begins behind slot 0 finds tokens that are there to stay: the scale becomes the larger of the
// page's and the one that the new tokens need, and where it grew the tokens before are rounded again.  Powers of two make that
// exact but for the values that fall among the smallest floats.  A run that begins at slot 0 owes nothing to what the page held.
// What has to move: 2 * 2 * (1 + 1/2) bytes a value pair, no arithmetic to speak of.  8 heads of 128, 17.7 k tokens: written in 24 us, read back
// in 19 (109 MB each, 4.5 and 5.6 TB/s); 64 tokens behind others 5.7.
//
// One workgroup per (page of a sequence, kv head), 2 * head_dim threads.  Thread t holds eight values of K and of V of token
// t / (head_dim / 8); the block's largest magnitude goes through shuffles and a few words of LDS.  K lies [token][head_dim] on both
// sides.  V lies [head_dim / 4][4 groups of tokens][4][4 tokens] in the pool, four tokens of one head_dim index a dword, as the second
// product of the attention takes them; it is turned over in LDS, and both sides are read and written in whole lines.
#include "fp8.h"

#include <type_traits>

namespace {

// Bytes of LDS for 64 of V's block: the threads of a token write, or read, a byte in each second of these, and with 64 they would meet in two
// banks of the 64.
constexpr int TURN = 72;

template <int HD, bool SCATTER, bool STREAM>
__global__ __launch_bounds__(2 * HD) void kv8_move_kernel(const int* __restrict__ cu, const int* __restrict__ start_pos,
                                                          const int* __restrict__ page_table, u32x4* __restrict__ k_tok,
                                                          u32x4* __restrict__ v_tok, unsigned char* __restrict__ k_pool,
                                                          unsigned char* __restrict__ v_pool, int n_seq, int n_tokens,
                                                          int max_pages, int n_kv, int n_pool_pages) {
    constexpr int CPR = HD / 8, CODES = kv8_codes(HD);
    __shared__ __align__(16) unsigned char turn[CODES / 64 * TURN];
    __shared__ unsigned red[2][LAPS_PAGE];
    // Work items: the first item of sequence s is cu[s] / 16 + 2 s (a run of n tokens touches at most n / 16 + 2 pages), items that no
    // page needs return at once.
    const int item = blockIdx.x, head = blockIdx.y, tid = threadIdx.x;
    auto first_item = [&](int s) { return cu[s] / LAPS_PAGE + 2 * s; };
    // A wave looks at 64 sequences at a time, one a lane.
    int lo = 0;
    for (int hi = n_seq; hi - lo > 1;) {
        const int step = (hi - lo + 63) / 64, at = lo + (tid & 63) * step;
        const int n = __popcll(__builtin_amdgcn_ballot_w64(at < hi && first_item(at < hi ? at : lo) <= item));
        if (n > 1) lo += (n - 1) * step;
        hi = lo + step < hi ? lo + step : hi;
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
    const size_t base = (size_t)page * kv8_page(n_kv, HD);
    unsigned char *kb = k_pool + base + (size_t)head * CODES, *vb = v_pool + base + (size_t)head * CODES;
    unsigned char *ks = k_pool + base + (size_t)n_kv * CODES + head, *vs = v_pool + base + (size_t)n_kv * CODES + head;
    const int t = tid / CPR, c = tid % CPR;
    const bool mine = t >= off0 && t < off1;
    const size_t at = ((size_t)(a + t) * n_kv + head) * CPR + c;
    auto take = [](const u32x4* from) { return STREAM ? __builtin_nontemporal_load(from) : *from; };
    auto put = [](u32x4 x, u32x4* to) {
        if (STREAM) __builtin_nontemporal_store(x, to);
        else *to = x;
    };
    // where V's block is turned over: byte of (head_dim index 8 c + j, token t), and this thread's eight bytes as they lie in the pool
    auto v_place = [&](int j) { return (2 * c + j / 4) * TURN + (t / 4) * 16 + (j % 4) * 4 + t % 4; };
    u32x2* turned = reinterpret_cast<u32x2*>(turn + tid / 8 * TURN + tid % 8 * 8);
    u32x2 *k8 = reinterpret_cast<u32x2*>(kb) + tid, *v8 = reinterpret_cast<u32x2*>(vb) + tid;   // this thread's eight bytes of each block
    if (SCATTER) {
        const bool keeps = off0 > 0;   // the page holds tokens that stay
        u32x4 k = {0u, 0u, 0u, 0u}, v = {0u, 0u, 0u, 0u};
        u32x2 k_old = {0u, 0u}, v_old = {0u, 0u};
        int ks_old = 0, vs_old = 0;
        if (mine) {
            k = take(k_tok + at);
            v = take(v_tok + at);
        }
        if (keeps) {
            k_old = *k8;
            v_old = *v8;
            ks_old = fp8_clamp_byte(*ks);
            vs_old = fp8_clamp_byte(*vs);
        }
        // largest magnitude of the token's head, and of the new tokens whose head is finite
        unsigned ka = bf16_amax(k), va = bf16_amax(v);
        ka = fp8_lanes_max<CPR>(ka);
        va = fp8_lanes_max<CPR>(va);
        const bool k_fine = ka < BF16_INF, v_fine = va < BF16_INF;
        ka = k_fine ? ka : 0u;
        va = v_fine ? va : 0u;
        if (c == 0) {   // a word a token
            red[0][t] = ka;
            red[1][t] = va;
        }
        __syncthreads();
        ka = fp8_lanes_max<16>(red[0][tid & 15]);
        va = fp8_lanes_max<16>(red[1][tid & 15]);
        int kn = fp8_scale_byte(ka), vn = fp8_scale_byte(va);
        if (keeps) {
            kn = ks_old > kn ? ks_old : kn;
            vn = vs_old > vn ? vs_old : vn;
        }
        // the tokens that stay, under the scale that holds now
        auto again = [](u32x2 old, int from, int to) { return from == to ? old : fp8_codes_of(fp8_eight(old.x, old.y, fp8_scale(from)), to); };
        if (mine) *k8 = k_fine ? fp8_codes_of(k, kn) : u32x2{FP8_NAN4, FP8_NAN4};
        else if (!keeps) *k8 = u32x2{0u, 0u};
        else if (kn != ks_old) *k8 = again(k_old, ks_old, kn);
        const u32x2 codes = !mine ? u32x2{0u, 0u} : v_fine ? fp8_codes_of(v, vn) : u32x2{FP8_NAN4, FP8_NAN4};
#pragma unroll
        for (int j = 0; j < 8; ++j) turn[v_place(j)] = (unsigned char)(codes[j / 4] >> (8 * (j % 4)));
        __syncthreads();
        // this thread's dwords are tokens 4 g .. 4 g + 3
        const int g = tid / 2 % 4;
        unsigned fresh = 0;   // bytes of a dword that are new
#pragma unroll
        for (int e = 0; e < 4; ++e) fresh |= 4 * g + e >= off0 && 4 * g + e < off1 ? 255u << (8 * e) : 0u;
        u32x2 out = *turned;
        if (keeps && fresh != ~0u) {
            const u32x2 stay = again(v_old, vs_old, vn);
            out = u32x2{(out.x & fresh) | (stay.x & ~fresh), (out.y & fresh) | (stay.y & ~fresh)};
        }
        if (!keeps || fresh != 0u || vn != vs_old) *v8 = out;
        if (tid == 0) {
            *ks = (unsigned char)kn;
            *vs = (unsigned char)vn;
        }
    } else {
        const u32x2 kc = *k8, vc = *v8;
        const float kf = fp8_scale(*ks), vf = fp8_scale(*vs);
        *turned = vc;
        __syncthreads();
        if (!mine) return;
        put(fp8_eight(kc.x, kc.y, kf), k_tok + at);
        unsigned w[2] = {0u, 0u};
#pragma unroll
        for (int j = 0; j < 8; ++j) w[j / 4] |= (unsigned)turn[v_place(j)] << (8 * (j % 4));
        put(fp8_eight(w[0], w[1], vf), v_tok + at);
    }
}

}  // namespace

int laps_launch_kv8_move(bool scatter, int n_seq, int n_tokens, const int* cu, const int* start_pos, const int* page_table,
                         int max_pages, void* k_tok, void* v_tok, void* k_pool, void* v_pool, int n_kv, int hd, int n_pool_pages,
                         hipStream_t s) {
    if (n_tokens == 0) return LAPS_OK;
    const dim3 grid(n_tokens / LAPS_PAGE + 2 * n_seq, n_kv);
    const bool stream = (size_t)n_tokens * n_kv * hd * 2 * sizeof(bf16_t) > ((size_t)32 << 20);   // eight L2 caches of 4 MiB
    auto pick = [&](auto HD) {
        constexpr int D = decltype(HD)::value;
        return scatter ? (stream ? kv8_move_kernel<D, true, true> : kv8_move_kernel<D, true, false>)
                       : (stream ? kv8_move_kernel<D, false, true> : kv8_move_kernel<D, false, false>);
    };
    auto kern = hd == 128 ? pick(std::integral_constant<int, 128>{}) : pick(std::integral_constant<int, 64>{});
    hipLaunchKernelGGL(kern, grid, dim3(2 * hd), 0, s, cu, start_pos, page_table, static_cast<u32x4*>(k_tok),
                       static_cast<u32x4*>(v_tok), static_cast<unsigned char*>(k_pool), static_cast<unsigned char*>(v_pool), n_seq,
                       n_tokens, max_pages, n_kv, n_pool_pages);
    LAPS_LAUNCH_CHECK();
    return LAPS_OK;
}
