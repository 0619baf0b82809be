// The 4-bit K/V cache: what its kernels share (format: include/laps.h).
#pragma once
#include "laps_internal.h"

typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(4))) __bf16 bf16x4;

constexpr int LAPS_KV4_MAX_PAGES = 1 << 26;       // of a page table's row: positions stay below 2^30
constexpr long LAPS_KV4_MAX_SEQ_HEADS = 1 << 20;   // sequences times query heads of an attention: its grid

constexpr int KV4_GROUP = 32;   // values of one token and kv head under one scale
// Bytes of a page of one kv head: the codes of 16 tokens, then their scales (K [token][group], V [group][token]).
__host__ __device__ constexpr int kv4_codes(int hd) { return LAPS_PAGE * hd / 2; }
__host__ __device__ constexpr int kv4_block(int hd) { return kv4_codes(hd) + LAPS_PAGE * hd / KV4_GROUP; }

// The conversions of this chip take a float's exponent bits as the scale and look at no other bit of it (all 256 exponents with
// set and cleared sign and mantissa bits read the same), so a scale byte only has to be moved to bits 23 to 30.
template <int I>
static __device__ __forceinline__ float kv4_scale(unsigned four) {   // byte I of four
    return __uint_as_float(I == 3 ? four >> 1 : four << (23 - 8 * I));
}
// Codes 2 I and 2 I + 1 of a dword of eight: exact in bf16 (three significant bits, subnormals included); scale byte 255 gives NaN.
template <int I>
static __device__ __forceinline__ unsigned kv4_pair(unsigned codes, float scale) {
    return __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, I));
}
static __device__ __forceinline__ u32x4 kv4_eight(unsigned codes, float scale) {
    return u32x4{kv4_pair<0>(codes, scale), kv4_pair<1>(codes, scale), kv4_pair<2>(codes, scale), kv4_pair<3>(codes, scale)};
}

// Scale byte of a group from the largest magnitude's bf16 bits: exponent e + 127, e the smallest with amax <= 7 * 2^e, that is
// amax's own less 2, or less 1 where its seven mantissa bits are above 1.75's (96).  The ends: 1, since 2^-126 already reaches below
// bf16's subnormals' half steps, and 252, where 6 * 2^e is the last multiple that bf16 holds.  An infinity or a NaN: 255.
static __device__ __forceinline__ int kv4_scale_byte(unsigned amax_bits) {
    const int b = (int)((amax_bits + 31) >> 7) - 2;
    return amax_bits >= 0x7f80u ? 255 : (b < 1 ? 1 : (b > 252 ? 252 : b));
}
// Largest magnitude (bf16 bits) of eight values.
static __device__ __forceinline__ unsigned kv4_amax(u32x4 x) {
    typedef __attribute__((ext_vector_type(2))) unsigned short u16x2;
    auto abs2 = [](unsigned w) { return __builtin_bit_cast(u16x2, w & 0x7fff7fffu); };
    const u16x2 a = __builtin_elementwise_max(abs2(x.x), abs2(x.y)), b = __builtin_elementwise_max(abs2(x.z), abs2(x.w));
    const u16x2 m = __builtin_elementwise_max(a, b);
    return m.x > m.y ? m.x : m.y;
}
// Codes of eight values over 2^(byte - 127), to nearest, ties to even, above 6 to 6 (every bf16 value checked at 40 scales).
static __device__ __forceinline__ unsigned kv4_codes_of(u32x4 x, int byte) {
    const float s = __uint_as_float((unsigned)byte << 23);
    auto two = [](unsigned w) { return __builtin_bit_cast(bf16x2, w); };   // by value: a bit cast of a vector's element takes the first one
    unsigned r = 0;
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, two(x.x), s, 0);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, two(x.y), s, 1);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, two(x.z), s, 2);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, two(x.w), s, 3);
    return byte == 255 ? 0 : r;
}

// scatter / gather: token-major bf16 <-> 4-bit pools
int laps_launch_kv4_move(bool scatter, int n_seq, int n_tokens, const int* cu, const int* start_pos, const int* page_table,
                         int max_pages, void* k_tok, void* v_tok, void* k_pool, void* v_pool, int n_kv, int hd, int n_pool_pages,
                         hipStream_t s);

// attention over 4-bit pools
struct Kv4Attn {
    const bf16_t* q;
    bf16_t* out;
    const unsigned char *k_pool, *v_pool;
    const int *cu, *seq_len, *prefix_len, *page_table;   // seq_len may be NULL
    int n_seq, n_tokens, max_pages, n_pool_pages, n_q, n_kv, hd;
};
// Launch of the kernel for few query rows a sequence.
struct Kv4RowsPlan {
    int row_tiles;    // 16-row tiles of a block
    int row_blocks;   // blocks of rows that workgroups of their own walk, a sequence and kv head
    int parts;        // most parts of a sequence's keys
    int min_parts;    // as many at least, where there are keys for them
};
// Which of the two kernels a launch shape takes: this one, or the blocks of 128 or 256 rows of the bf16 pools' attention.
bool laps_kv4_takes_rows(int n_seq, int n_tokens, int n_q, int n_kv);
Kv4RowsPlan laps_kv4_rows_plan(int n_seq, int n_tokens, int n_q, int n_kv, int max_pages);
size_t laps_kv4_rows_bytes(const Kv4RowsPlan& p, int n_tokens, int n_q, int hd);   // partial results of the parts
int laps_launch_kv4_rows(const Kv4Attn& a, const Kv4RowsPlan& p, float* partial, hipStream_t s);
