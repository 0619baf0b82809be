// 8-bit floats under power-of-two scales: what the 8-bit K/V cache and the products of 8-bit matrices share (formats: include/laps.h).
#pragma once
#include "laps_internal.h"

typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(4))) __bf16 bf16x4;

// A block's values are x = code * 2^(byte - 127), code an 8-bit float with 4 exponent and 3 mantissa bits (largest 448, no infinity, 0x7f
// and 0xff NaN).  Between these bytes every x but 0 is a normal bf16 number: 2^-9 * 2^-116 = 2^-125, 448 * 2^119 = 1.75 * 2^127.
constexpr int FP8_LOWEST = 11, FP8_HIGHEST = 246;
constexpr unsigned FP8_NAN4 = 0x7f7f7f7fu;   // four NaN codes
constexpr unsigned BF16_INF = 0x7f80u;

// Scale byte of a block from its largest finite magnitude's bf16 bits: 127 plus the smallest e with amax <= 448 * 2^e = 1.75 * 2^(e + 8), that
// is amax's own exponent less 8, or less 7 where its seven mantissa bits are above 1.75's (96).
static __device__ __forceinline__ int fp8_scale_byte(unsigned amax_bits) {
    const int b = (int)((amax_bits + 31) >> 7) - 8;
    return b < FP8_LOWEST ? FP8_LOWEST : (b > FP8_HIGHEST ? FP8_HIGHEST : b);
}
static __device__ __forceinline__ int fp8_clamp_byte(int byte) {   // what a pool that nothing was written to may hold
    return byte < FP8_LOWEST ? FP8_LOWEST : (byte > FP8_HIGHEST ? FP8_HIGHEST : byte);
}
static __device__ __forceinline__ float fp8_scale(int byte) { return __uint_as_float((unsigned)byte << 23); }

// Largest magnitude (bf16 bits) of eight values; not finite ones count as what they are, BF16_INF and above.
static __device__ __forceinline__ unsigned bf16_amax(u32x4 x) {
    typedef __attribute__((ext_vector_type(2))) unsigned short u16x2;
    auto abs2 = [](unsigned w) { return __builtin_bit_cast(u16x2, w & 0x7fff7fffu); };
    const u16x2 a = __builtin_elementwise_max(abs2(x.x), abs2(x.y)), b = __builtin_elementwise_max(abs2(x.z), abs2(x.w));
    const u16x2 m = __builtin_elementwise_max(a, b);
    return m.x > m.y ? m.x : m.y;
}

static __device__ __forceinline__ unsigned bf16_amax_finite(u32x4 x) {   // of the finite ones
    unsigned top = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const unsigned w = x[j / 2] >> (16 * (j % 2)) & 0x7fffu;
        top = w < BF16_INF && w > top ? w : top;
    }
    return top;
}

// The largest of the values that N (8 or 16) lanes side by side hold, in each of them: pairs, fours, then halves and rows mirrored.
template <int N>
static __device__ __forceinline__ unsigned fp8_lanes_max(unsigned x) {
    auto most = [](unsigned a, unsigned b) { return a > b ? a : b; };
    x = most(x, (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, 0x0b1, 15, 15, true));   // quad_perm 1 0 3 2
    x = most(x, (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, 0x04e, 15, 15, true));   // quad_perm 2 3 0 1
    x = most(x, (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, 0x141, 15, 15, true));   // row_half_mirror
    if (N == 16) x = most(x, (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, 0x140, 15, 15, true));   // row_mirror
    return x;
}

// Codes of eight bf16 values under 2^(byte - 127): to nearest, ties to the even code, what is not finite to NaN.  The conversion makes
// magnitudes of 464 and more NaN, which a scale below the highest never meets; under that one they are cut to 448 first.
static __device__ __forceinline__ u32x2 fp8_codes_of(u32x4 x, int byte) {
    typedef __attribute__((ext_vector_type(2))) short s16x2;
    if (byte == FP8_HIGHEST) {
        auto cut = [](unsigned m) { return (m & 0x7fffu) > 0x7f60u && (m & 0x7fffu) < BF16_INF ? (m & 0x8000u) | 0x7f60u : m; };
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = cut(x[i] & 0xffffu) | cut(x[i] >> 16) << 16;
    }
    const float s = fp8_scale(byte);
    auto four = [&](unsigned lo, unsigned hi) {
        s16x2 r = {0, 0};
        r = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(r, __builtin_bit_cast(bf16x2, lo), s, false);
        r = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(r, __builtin_bit_cast(bf16x2, hi), s, true);
        return __builtin_bit_cast(unsigned, r);
    };
    return u32x2{four(x.x, x.y), four(x.z, x.w)};
}

// Four codes as bf16, exactly.
static __device__ __forceinline__ u32x2 fp8_four(unsigned codes, float scale) {
    return u32x2{__builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, false)),
                 __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, true))};
}
static __device__ __forceinline__ u32x4 fp8_eight(unsigned lo, unsigned hi, float scale) {
    const u32x2 a = fp8_four(lo, scale), b = fp8_four(hi, scale);
    return u32x4{a.x, a.y, b.x, b.y};
}

// ---- the 8-bit K/V cache.  A page: 16 * hd codes of every kv head, then a scale byte of every kv head.
__host__ __device__ constexpr int kv8_codes(int hd) { return LAPS_PAGE * hd; }
__host__ __device__ constexpr size_t kv8_page(int n_kv, int hd) { return (size_t)n_kv * kv8_codes(hd) + (size_t)(n_kv + 127) / 128 * 128; }
// scatter / gather: token-major bf16 <-> 8-bit pools
int laps_launch_kv8_move(bool scatter, int n_seq, int n_tokens, const int* cu, const int* start_pos, const int* page_table,
                         int max_pages, void* k_tok, void* v_tok, void* k_pool, void* v_pool, int n_kv, int hd, int n_pool_pages,
                         hipStream_t s);

// laps_launch_attention over 8-bit pools.
int laps_launch_attention_kv8(const bf16_t* q, bf16_t* out, const void* k_pool, const void* v_pool, const int* page_table, int max_pages,
                              int n_seq, int n_tokens, const int* tile_start, const int* item_seq, float* partial, size_t partial_bytes,
                              int n_q, int n_kv, int hd, int n_pool_pages, hipStream_t s);

// ---- matrices of 8-bit floats: codes [rows][k rounded up to 128], scale bytes [blocks of 128][rows rounded up to 16]
constexpr int FP8_BLOCK = 128;
constexpr long fp8_columns(long k) { return (k + FP8_BLOCK - 1) / FP8_BLOCK * FP8_BLOCK; }
constexpr long fp8_pitch(long rows) { return (rows + 15) / 16 * 16; }
int laps_launch_fp8_quant(const bf16_t* x, int m, int k, unsigned char* codes, unsigned char* scales, hipStream_t s);
int laps_launch_fp8_dequant(const unsigned char* codes, const unsigned char* scales, int m, int k, bf16_t* x, hipStream_t s);

struct Fp8Plan {
    int cfg;     // tile
    int split;   // K slices
    int per;     // blocks of 128 of a slice
};
Fp8Plan laps_fp8_plan(int m, int n, int k);
void laps_fp8_tile_dims(int cfg, int* bm, int* bn);
// out bf16 [m][n] = a w^T; partial: split * m * n floats if split > 1.  k is a multiple of 128.
int laps_launch_gemm_fp8(const Fp8Plan& p, const unsigned char* a, const unsigned char* a_scales, const unsigned char* w,
                         const unsigned char* w_scales, bf16_t* out, int m, int n, int k, float* partial, hipStream_t s);
// A projection of bf16 rows in one launch, without their codes in memory: whether the plan has one for them, and the launch.
bool laps_fp8_takes_bf16_rows(const Fp8Plan& p, const bf16_t* x, int m, int k);
int laps_launch_linear_fp8_rows(const bf16_t* x, const unsigned char* w, const unsigned char* w_scales, bf16_t* out, int m, int n, int k, hipStream_t s);
