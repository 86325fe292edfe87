// A matrix to MX8 (mx8.h): one read of the values, one write of the bytes, nothing kept; bound by memory (262144 rows of 768 bfloat16
// values 112 us, 610 MB at 5.4 TB/s; 2001 float rows of 416 3.7 us).
#include "mx8.h"

namespace unipool {

namespace {

// A workgroup takes 128 columns of 64 rows: 16 lanes of 8 values to a row's 128, so a block is four neighbouring lanes.  The
// words of scales of its rows are neighbours and leave as one piece.
constexpr int kQRows = 64;                // (4 bytes of scales each: one byte a thread)

template <typename TA, bool WIDE>
__global__ __launch_bounds__(256) void quantize_mx8_kernel(const TA* __restrict__ src, long long rows, int cols, unsigned char* __restrict__ q,
                                                           unsigned char* __restrict__ scale, int steps) {
    __shared__ unsigned char sc[kQRows * 4];
    const long long row0 = (long long)(blockIdx.x / steps) * kQRows;
    const int step = blockIdx.x % steps, c0 = step * kMxStep, lane = threadIdx.x & 15;
    const int col = c0 + lane * 8;
#pragma unroll
    for (int p = 0; p < kQRows / 16; p++) {
        const int r = p * 16 + (threadIdx.x >> 4);
        const bool on = row0 + r < rows && col < cols;
        float v[8];
        if (on) {
            const TA* s = src + (size_t)(row0 + r) * cols + col;
            if constexpr (WIDE) {
                union { uint4 u[sizeof(TA) / 2]; TA e[8]; } w;
#pragma unroll
                for (int i = 0; i < (int)sizeof(TA) / 2; i++) w.u[i] = reinterpret_cast<const uint4*>(s)[i];
#pragma unroll
                for (int i = 0; i < 8; i++) v[i] = to_f32(w.e[i]);
            } else {
#pragma unroll
                for (int i = 0; i < 8; i++) v[i] = to_f32(s[i]);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; i++) v[i] = 0.f;
        }
        float m = v[0];
#pragma unroll
        for (int i = 1; i < 8; i++) m = mx8_max(m, v[i]);
        m = mx8_lanes_max<4>(m);
        const int byte = col < cols ? mx8_scale_byte(m) : kMxBias;
        if (on) {
            const unsigned lo = mx8_pack4(v[0], v[1], v[2], v[3], byte), hi = mx8_pack4(v[4], v[5], v[6], v[7], byte);
            unsigned char* dst = q + (size_t)(row0 + r) * cols + col;
            if constexpr (WIDE) {
                *reinterpret_cast<uint2*>(dst) = make_uint2(lo, hi);
            } else {
#pragma unroll
                for (int i = 0; i < 8; i++) dst[i] = (unsigned char)((i < 4 ? lo : hi) >> (8 * (i & 3)));
            }
        }
        if ((lane & 3) == 0) sc[r * 4 + (lane >> 2)] = (unsigned char)byte;
    }
    __syncthreads();
    const long long left = (rows - row0) * 4;
    if (threadIdx.x < left) scale[((size_t)step * rows + row0) * 4 + threadIdx.x] = sc[threadIdx.x];
}

template <typename TA>
hipError_t run_quantize(const void* src, long long rows, int cols, void* q, void* scale, hipStream_t st) {
    const int steps = cdiv(cols, kMxStep);
    const long long grid = (rows + kQRows - 1) / kQRows * steps;      // below 2^24, checked at the boundary
    // rows are multiples of 32 values, so 16-byte pieces follow from the addresses
    if (((uintptr_t)src & 15) == 0 && ((uintptr_t)q & 7) == 0)
        quantize_mx8_kernel<TA, true><<<(unsigned)grid, 256, 0, st>>>((const TA*)src, rows, cols, (unsigned char*)q, (unsigned char*)scale, steps);
    else
        quantize_mx8_kernel<TA, false><<<(unsigned)grid, 256, 0, st>>>((const TA*)src, rows, cols, (unsigned char*)q, (unsigned char*)scale, steps);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_quantize_mx8(int dtype, const void* src, long long rows, int cols, void* q, void* scale, hipStream_t st) {
    return dtype == UNIPOOL_BF16 ? run_quantize<bf16>(src, rows, cols, q, scale, st) : run_quantize<float>(src, rows, cols, q, scale, st);
}

}  // namespace unipool
