// Product of 8-bit matrices under power-of-two block scales, on gfx950's scaled matrix instructions.
//
//   C[m, n] = sum over blocks b of 2^(ea[m, b] + ew[n, b]) * sum over the block's 128 k of a[m, k] w[n, k]      in float32, rounded to bf16
//
// v_mfma_scale_f32_16x16x128_f8f6f4 takes 128 k of 16 rows of either operand, a whole block, and a scale byte for each row, so the scales
// cost no instruction of their own.
#include <algorithm>

#include "fp8.h"

namespace {

typedef __attribute__((ext_vector_type(8))) int i32x8;

constexpr int CHUNKS = FP8_BLOCK / 16;   // 16-byte chunks of a row of a slab

struct Fp8Args {
    const unsigned char *A, *As, *W, *Ws;   // codes and scale bytes
    long a_pitch, w_pitch;                  // rows of the scales
    int M, N, K, split, per, tiles_m, tiles_n;
    bf16_t* out;
    float* partial;                         // [split][M][N] where split > 1
};

__global__ __launch_bounds__(256, 2) void gemm_fp8_kernel(const Fp8Args g) {
    constexpr int BM = 128, BN = 128;
    __shared__ __align__(16) u32x4 sa[BM * CHUNKS], sw[BN * CHUNKS];
    const int tm = blockIdx.x % g.tiles_m, rest = blockIdx.x / g.tiles_m, tn = rest % g.tiles_n, ks = rest / g.tiles_n;
    const int m0 = tm * BM, n0 = tn * BN, blocks = g.K / FP8_BLOCK;
    const int b0 = ks * g.per, b1 = b0 + g.per < blocks ? b0 + g.per : blocks;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, wm = wave / 2, wn = wave % 2, i = lane & 15, q = lane >> 4;
    f32x4 acc[4][4];
#pragma unroll
    for (int x = 0; x < 4; ++x)
#pragma unroll
        for (int y = 0; y < 4; ++y) acc[x][y] = f32x4{0.f, 0.f, 0.f, 0.f};
    auto row_of = [](int r, int rows) { return (size_t)(r < rows ? r : rows - 1); };   // rows past the last one are not stored
    auto swz = [](int row, int chunk) { return row * CHUNKS + (chunk ^ (row & 7)); };
    for (int b = b0; b < b1; ++b) {
        __syncthreads();
#pragma unroll
        for (int j = 0; j < BM * CHUNKS / 256; ++j) {
            const int row = (tid + 256 * j) / CHUNKS, c = tid % CHUNKS;
            sa[swz(row, c)] = *reinterpret_cast<const u32x4*>(g.A + row_of(m0 + row, g.M) * g.K + (size_t)b * FP8_BLOCK + c * 16);
            sw[swz(row, c)] = *reinterpret_cast<const u32x4*>(g.W + row_of(n0 + row, g.N) * g.K + (size_t)b * FP8_BLOCK + c * 16);
        }
        __syncthreads();
        i32x8 fa[4], fw[4];
        int ea[4], ew[4];
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            // which 32 of the 128 k a lane holds does not matter, as long as both operands agree
            const int ra = wm * 64 + x * 16 + i, rw = wn * 64 + x * 16 + i;
            auto two = [](u32x4 lo, u32x4 hi) {
                return i32x8{(int)lo.x, (int)lo.y, (int)lo.z, (int)lo.w, (int)hi.x, (int)hi.y, (int)hi.z, (int)hi.w};
            };
            fa[x] = two(sa[swz(ra, q)], sa[swz(ra, q + 4)]);
            fw[x] = two(sw[swz(rw, q)], sw[swz(rw, q + 4)]);
            ea[x] = g.As[b * g.a_pitch + row_of(m0 + ra, g.M)];
            ew[x] = g.Ws[b * g.w_pitch + row_of(n0 + rw, g.N)];
        }
#pragma unroll
        for (int x = 0; x < 4; ++x)
#pragma unroll
            for (int y = 0; y < 4; ++y)
                acc[x][y] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fw[y], fa[x], acc[x][y], 0, 0, 0, ew[y], 0, ea[x]);
    }
    // a lane holds columns 4 q .. 4 q + 3 of row i of a sub-tile
#pragma unroll
    for (int x = 0; x < 4; ++x) {
        const int m = m0 + wm * 64 + x * 16 + i;
        if (m >= g.M) continue;
#pragma unroll
        for (int y = 0; y < 4; ++y)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int n = n0 + wn * 64 + y * 16 + 4 * q + e;
                if (n >= g.N) continue;
                if (g.split == 1) g.out[(size_t)m * g.N + n] = f32_to_bf16(acc[x][y][e]);
                else g.partial[((size_t)ks * g.M + m) * g.N + n] = acc[x][y][e];
            }
    }
}

// The slices' sums, in order.
__global__ __launch_bounds__(256) void fp8_sum_kernel(const float* __restrict__ partial, int split, long count, bf16_t* __restrict__ out) {
    const long i = (long)blockIdx.x * 256 + threadIdx.x;
    if (i >= count) return;
    float sum = partial[i];
    for (int s = 1; s < split; ++s) sum += partial[s * count + i];
    out[i] = f32_to_bf16(sum);
}

}  // namespace

void laps_fp8_tile_dims(int cfg, int* bm, int* bn) { *bm = *bn = cfg == 0 ? 128 : 0; }

Fp8Plan laps_fp8_plan(int m, int n, int k) {
    const int blocks = k / FP8_BLOCK;
    const long tiles = ((m + 127L) / 128) * ((n + 127L) / 128);
    long split = std::max(1L, std::min(256 / tiles, (long)blocks / 4));
    const int per = (int)((blocks + split - 1) / split);
    return {0, (blocks + per - 1) / per, per};
}

int laps_launch_gemm_fp8(const Fp8Plan& p, const unsigned char* a, const unsigned char* a_scales, const unsigned char* w,
                         const unsigned char* w_scales, bf16_t* out, int m, int n, int k, float* partial, hipStream_t s) {
    Fp8Args g = {a, a_scales, w, w_scales, fp8_pitch(m), fp8_pitch(n), m, n, k, p.split, p.per, (m + 127) / 128, (n + 127) / 128, out, partial};
    hipLaunchKernelGGL(gemm_fp8_kernel, dim3((unsigned)((long)g.tiles_m * g.tiles_n * p.split)), dim3(256), 0, s, g);
    LAPS_LAUNCH_CHECK();
    if (p.split > 1) {
        const long count = (long)m * n;
        hipLaunchKernelGGL(fp8_sum_kernel, dim3((unsigned)((count + 255) / 256)), dim3(256), 0, s, partial, p.split, count, out);
        LAPS_LAUNCH_CHECK();
    }
    return LAPS_OK;
}
