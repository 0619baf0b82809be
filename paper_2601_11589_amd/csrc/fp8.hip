// bf16 matrices <-> matrices of 8-bit floats with a scale 2^e for each block of 128 along a row.
//
// A block's 128 values are 16 lanes of eight: the largest magnitude is four exchanges inside their row away, then every lane turns its own 16 bytes into
// eight.  Nothing but the copies has to move, 2 + 1 bytes a value.  A workgroup takes 16 rows, so that the scale bytes it writes, which lie
// [block][row], are 16 side by side.
#include "fp8.h"

namespace {

constexpr int ROWS = 16;     // of a workgroup, 16 lanes each
// BLOCKS: two where the loads of small matrices end sooner (96 x 5120 3.3 -> 2.7 us), large ones do not care (1, 2, 4, 8: 37888 x 3584 80.8 to
// 82.3, one 86.9).  STREAM: rows are read past the caches, they are not needed again; where the whole exceeds eight L2 caches of 4 MiB what
// is written goes past them as well.  37888 x 3584, 407 MB, there and back 82.6 / 82.0 -> 76.8 / 78.5 us (5.3 TB/s, a large copy reaches 5.0).
constexpr int BLOCKS = 2;    // of a workgroup: loads on their way at once

// Eight values from column c of a row of k, zeros behind it.  VEC: rows and columns keep to 16 bytes.
template <bool VEC>
__device__ __forceinline__ u32x4 take_eight(const bf16_t* row, long c, int k) {
    u32x4 x = {0u, 0u, 0u, 0u};
    if (VEC) {
        if (c < k) x = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(row + c));
        return x;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j)
        if (c + j < k) x[j / 2] |= (unsigned)row[c + j] << (16 * (j % 2));
    return x;
}

template <bool VEC, bool STREAM>
__global__ __launch_bounds__(ROWS * 16) void fp8_quant_kernel(const bf16_t* __restrict__ x, int m, int k, long columns, long pitch,
                                                              unsigned char* __restrict__ codes, unsigned char* __restrict__ scales) {
    const int l = threadIdx.x % 16;
    const long row = (long)blockIdx.x * ROWS + threadIdx.x / 16;
    const int b0 = blockIdx.y * BLOCKS, n = (int)(columns / FP8_BLOCK);
    if (row >= m) {   // the scales' padding
#pragma unroll
        for (int i = 0; i < BLOCKS; ++i)
            if (l == 0 && b0 + i < n) scales[(b0 + i) * pitch + row] = 127;
        return;
    }
    u32x4 v[BLOCKS];
#pragma unroll
    for (int i = 0; i < BLOCKS; ++i) v[i] = take_eight<VEC>(x + row * k, (long)(b0 + i) * FP8_BLOCK + 8 * l, k);
#pragma unroll
    for (int i = 0; i < BLOCKS; ++i) {
        if (b0 + i >= n) break;
        unsigned top = bf16_amax(v[i]);
        if (top >= BF16_INF) top = bf16_amax_finite(v[i]);
        top = fp8_lanes_max<16>(top);
        const int byte = fp8_scale_byte(top);
        u32x2* to = reinterpret_cast<u32x2*>(codes + row * columns + (long)(b0 + i) * FP8_BLOCK + 8 * l);
        if (STREAM) __builtin_nontemporal_store(fp8_codes_of(v[i], byte), to);
        else *to = fp8_codes_of(v[i], byte);
        if (l == 0) scales[(b0 + i) * pitch + row] = (unsigned char)byte;
    }
}

template <bool VEC, bool STREAM>
__global__ __launch_bounds__(ROWS * 16) void fp8_dequant_kernel(const unsigned char* __restrict__ codes, const unsigned char* __restrict__ scales,
                                                                int m, int k, long columns, long pitch, bf16_t* __restrict__ x) {
    const int l = threadIdx.x % 16;
    const long row = (long)blockIdx.x * ROWS + threadIdx.x / 16;
    const int b0 = blockIdx.y * BLOCKS, n = (int)(columns / FP8_BLOCK);
    if (row >= m) return;
    u32x2 v[BLOCKS];
    int byte[BLOCKS];
#pragma unroll
    for (int i = 0; i < BLOCKS; ++i) {
        const int b = b0 + i < n ? b0 + i : n - 1;
        v[i] = *reinterpret_cast<const u32x2*>(codes + row * columns + (long)b * FP8_BLOCK + 8 * l);
        byte[i] = scales[b * pitch + row];
    }
#pragma unroll
    for (int i = 0; i < BLOCKS; ++i) {
        const long c = (long)(b0 + i) * FP8_BLOCK + 8 * l;
        if (c >= k) break;
        const u32x4 w = fp8_eight(v[i].x, v[i].y, fp8_scale(byte[i]));
        if (VEC) {
            if (STREAM) __builtin_nontemporal_store(w, reinterpret_cast<u32x4*>(x + row * k + c));
            else *reinterpret_cast<u32x4*>(x + row * k + c) = w;
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (c + j < k) x[row * k + c + j] = (bf16_t)(w[j / 2] >> (16 * (j % 2)));
        }
    }
}

dim3 grid_of(int m, int k) {
    const long n = fp8_columns(k) / FP8_BLOCK;
    return dim3((unsigned)((m + (long)ROWS - 1) / ROWS), (unsigned)((n + BLOCKS - 1) / BLOCKS));
}

bool streams(int m, int k) { return (size_t)m * k * 3 > ((size_t)32 << 20); }
auto pick_quant(bool vec, bool stream) {
    return vec ? (stream ? fp8_quant_kernel<true, true> : fp8_quant_kernel<true, false>)
               : (stream ? fp8_quant_kernel<false, true> : fp8_quant_kernel<false, false>);
}
auto pick_dequant(bool vec, bool stream) {
    return vec ? (stream ? fp8_dequant_kernel<true, true> : fp8_dequant_kernel<true, false>)
               : (stream ? fp8_dequant_kernel<false, true> : fp8_dequant_kernel<false, false>);
}

}  // namespace

int laps_launch_fp8_quant(const bf16_t* x, int m, int k, unsigned char* codes, unsigned char* scales, hipStream_t s) {
    const bool vec = k % 8 == 0 && (reinterpret_cast<uintptr_t>(x) & 15) == 0;
    hipLaunchKernelGGL(pick_quant(vec, streams(m, k)), grid_of(m, k), dim3(ROWS * 16), 0, s, x, m, k, fp8_columns(k),
                       fp8_pitch(m), codes, scales);
    LAPS_LAUNCH_CHECK();
    return LAPS_OK;
}

int laps_launch_fp8_dequant(const unsigned char* codes, const unsigned char* scales, int m, int k, bf16_t* x, hipStream_t s) {
    const bool vec = k % 8 == 0 && (reinterpret_cast<uintptr_t>(x) & 15) == 0;
    hipLaunchKernelGGL(pick_dequant(vec, streams(m, k)), grid_of(m, k), dim3(ROWS * 16), 0, s, codes, scales, m, k,
                       fp8_columns(k), fp8_pitch(m), x);
    LAPS_LAUNCH_CHECK();
    return LAPS_OK;
}
