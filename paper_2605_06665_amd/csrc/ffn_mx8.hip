// The pool's experts forward on 8-bit rows with 8-bit weights (MX8, mx8.h):
//   A = X_e W_gate,e^T;  B = X_e W_up,e^T;  H = silu(A) * B, to MX8;  Y = H W_down,e^T, to bfloat16.
//
// The products are v_mfma_scale_f32_16x16x128_f8f6f4 on e4m3 operands: one instruction multiplies 16 weight rows by 16
// activation rows over 128 indices and applies the scale of every block of 32 on the way.  Lane l holds row l % 16 of its
// operand, indices 16 g .. 16 g + 15 and 64 + 16 g .. with g = l / 16 (two 16-byte pieces), and brings the scale byte of block g
// of that row (checked on the device with one-hot operands).  Sums over the instructions are float; inside one the products of
// neighbouring indices are added with the terms kept to 2^-13 of the largest (measured; on Gaussian operands 1.5e-5 of the result,
// against the 1.7e-3 of its rounding to bfloat16).  The 16x16x32 form adds the same way at half the rate.
#include "gemm_common.h"
#include "mx8.h"

namespace unipool {

namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));

struct Mx8Args {
    GemmArgs g;                      // tile list only (tile_meta, n_tiles_n, group_m)
    const unsigned char* x;          // [rows][K], or the tokens when gather is given
    const unsigned char* x_scale;    // [ceil(K / 128)][x_rows][4]
    long long x_rows;
    const int32_t* gather;           // row r is row gather[r] / gather_div of x
    int gather_div;
    const unsigned char* w;          // [E][w_rows][K]
    const unsigned char* w_scale;    // [ceil(K / 128)][E * w_rows][4]
    int w_rows, E;
    int K, N;                        // reduction length; output columns (gate-up: of H)
    unsigned char* h;                // gate-up: H [S][N] and its scales
    unsigned char* h_scale;
    bf16* y;                         // down: [S][N]
    long long S;
};

__device__ __forceinline__ i32x8 two16(const uint4& a, const uint4& b) {
    i32x8 v;
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
    v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
    return v;
}

// Tile of 128 rows by 128 weight rows (gate-up: 64 gate and the 64 up rows they meet), four wavefronts of 64 x 64.
template <bool GATE_UP>
__global__ __launch_bounds__(256) void ffn_mx8_kernel(const Mx8Args a) {
    constexpr int BM = 128, BN = 128, ROWB = 128;
    __shared__ __attribute__((aligned(16))) unsigned char xs[BM * ROWB], ws[BN * ROWB];
    __shared__ unsigned xsc[BM], wsc[BN];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int l16 = lane & 15, lg = lane >> 4, wm = wave & 1, wn = wave >> 1;
    const int nk = cdiv(a.K, kMxStep);
    auto swz = [](int row, int ch) { return row * ROWB + ((ch ^ (row >> 1)) & 7) * 16; };
    TileWalk walk(a.g);
    for (TileRef t = walk.next(a.g); t.valid; t = walk.next(a.g)) {
        const int n0 = t.nt * (GATE_UP ? BN / 2 : BN);
        f32x4 acc[4][4];                                   // [16 rows][16 weight rows]
#pragma unroll
        for (int m = 0; m < 4; m++)
#pragma unroll
            for (int n = 0; n < 4; n++) acc[m][n] = f32x4{0.f, 0.f, 0.f, 0.f};
        auto token = [&](int r) {
            int row = t.row0 + min(r, t.rows - 1);
            return (long long)(a.gather ? a.gather[row] / a.gather_div : row);
        };
        auto weight = [&](int r) {                          // weight row of tile row r
            const int c = GATE_UP ? min(n0 + r % 64, a.N - 1) + (r / 64) * a.N : min(n0 + r, a.N - 1);
            return (long long)t.expert * a.w_rows + c;
        };
        for (int kt = 0; kt < nk; kt++) {
            __syncthreads();
#pragma unroll
            for (int i = 0; i < BM * 8 / 256; i++) {
                const int q = i * 256 + tid, r = q >> 3, ch = q & 7, k = kt * kMxStep + ch * 16;
                uint4 xv = make_uint4(0, 0, 0, 0), wv = xv;
                if (k < a.K) {
                    xv = *reinterpret_cast<const uint4*>(a.x + token(r) * a.K + k);
                    wv = *reinterpret_cast<const uint4*>(a.w + weight(r) * a.K + k);
                }
                *reinterpret_cast<uint4*>(xs + swz(r, ch)) = xv;
                *reinterpret_cast<uint4*>(ws + swz(r, ch)) = wv;
            }
            if (tid < 128) xsc[tid] = *reinterpret_cast<const unsigned*>(a.x_scale + ((long long)kt * a.x_rows + token(tid)) * 4);
            else wsc[tid - 128] = *reinterpret_cast<const unsigned*>(a.w_scale + ((long long)kt * a.E * a.w_rows + weight(tid - 128)) * 4);
            __syncthreads();
            // past the end of K the values are zeros; their scales must not be NaN
            const bool tail = kt * kMxStep + lg * kMxBlock >= a.K;
            i32x8 wf[4];
            int wsb[4];
#pragma unroll
            for (int n = 0; n < 4; n++) {
                const int r = GATE_UP ? (n >> 1) * 64 + wn * 32 + (n & 1) * 16 + l16 : wn * 64 + n * 16 + l16;
                wf[n] = two16(*reinterpret_cast<const uint4*>(ws + swz(r, lg)), *reinterpret_cast<const uint4*>(ws + swz(r, 4 + lg)));
                wsb[n] = tail ? kMxBias : (int)(wsc[r] >> (8 * lg));
            }
#pragma unroll
            for (int m = 0; m < 4; m++) {
                const int r = wm * 64 + m * 16 + l16;
                const i32x8 xf = two16(*reinterpret_cast<const uint4*>(xs + swz(r, lg)), *reinterpret_cast<const uint4*>(xs + swz(r, 4 + lg)));
                const int xsb = tail ? kMxBias : (int)(xsc[r] >> (8 * lg));
#pragma unroll
                for (int n = 0; n < 4; n++)
                    acc[m][n] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wf[n], xf, acc[m][n], 0, 0, 0, wsb[n], 0, xsb);
            }
        }
        // acc[m][n][i] = C[row wm 64 + 16 m + l16][weight row 16 n + 4 lg + i of the wavefront's 64]
#pragma unroll
        for (int m = 0; m < 4; m++) {
            const int r = wm * 64 + m * 16 + l16;
            const bool on = r < t.rows;
            const long long row = t.row0 + r;
            if constexpr (GATE_UP) {
                // the wavefront's 32 columns of H are one block of every row, 8 values in each of four lanes
                float h[8];
                unsigned mag = 0;
#pragma unroll
                for (int n = 0; n < 2; n++)
#pragma unroll
                    for (int i = 0; i < 4; i++) {
                        h[4 * n + i] = silu_f(acc[m][n][i]) * acc[m][2 + n][i];
                        mag = max(mag, mx8_mag(h[4 * n + i]));
                    }
                mag = max(mag, (unsigned)__shfl_xor((int)mag, 16, 64));
                mag = max(mag, (unsigned)__shfl_xor((int)mag, 32, 64));
                const int byte = mx8_scale_byte(mag), c = n0 + wn * 32;
                if (on && c < a.N) {
                    unsigned char* dst = a.h + row * a.N + c + 4 * lg;
                    *reinterpret_cast<unsigned*>(dst) = mx8_pack4(h[0], h[1], h[2], h[3], byte);
                    *reinterpret_cast<unsigned*>(dst + 16) = mx8_pack4(h[4], h[5], h[6], h[7], byte);
                    if (lg == 0) a.h_scale[mx8_scale_at(a.S, row, c / kMxBlock)] = (unsigned char)byte;
                }
            } else {
#pragma unroll
                for (int n = 0; n < 4; n++) {
                    const int c = n0 + wn * 64 + n * 16 + 4 * lg;
                    if (on && c < a.N)
                        *reinterpret_cast<uint2*>(a.y + row * a.N + c) = pack4(acc[m][n][0], acc[m][n][1], acc[m][n][2], acc[m][n][3]);
                }
            }
        }
    }
}

template <bool GATE_UP> hipError_t run_mx8(Mx8Args a, int32_t* meta, hipStream_t st) {
    a.g.tile_meta = meta;
    a.g.group_m = 1;
    a.g.n_tiles_n = cdiv(a.N, GATE_UP ? 64 : 128);
    ffn_mx8_kernel<GATE_UP><<<max(kNumXcd, num_cus() / kNumXcd * kNumXcd) * 4, 256, 0, st>>>(a);
    return hipGetLastError();
}

}  // namespace

hipError_t mx8_ffn_fwd(const unipool_shape& s, const void* x, const void* x_scale, const int32_t* slot_of_row, const int32_t* offsets,
                       const void* wgu, const void* wgu_scale, const void* wd, const void* wd_scale, void* h, void* h_scale, void* y,
                       int32_t* tile_meta, hipStream_t st) {
    hipError_t e = mfma_build_tiles(s, offsets, 128, tile_meta, st);
    if (e != hipSuccess) return e;
    const long long S = (long long)s.T * s.k;
    Mx8Args a = {};
    a.x = (const unsigned char*)x; a.x_scale = (const unsigned char*)x_scale;
    a.x_rows = slot_of_row ? s.T : S;
    a.gather = slot_of_row; a.gather_div = s.k;
    a.w = (const unsigned char*)wgu; a.w_scale = (const unsigned char*)wgu_scale;
    a.w_rows = 2 * s.d_ff; a.E = s.E;
    a.K = s.d_model; a.N = s.d_ff;
    a.h = (unsigned char*)h; a.h_scale = (unsigned char*)h_scale; a.S = S;
    e = run_mx8<true>(a, tile_meta, st);
    if (e != hipSuccess) return e;
    Mx8Args b = {};
    b.x = (const unsigned char*)h; b.x_scale = (const unsigned char*)h_scale;
    b.x_rows = S;
    b.w = (const unsigned char*)wd; b.w_scale = (const unsigned char*)wd_scale;
    b.w_rows = s.d_model; b.E = s.E;
    b.K = s.d_ff; b.N = s.d_model;
    b.y = (bf16*)y; b.S = S;
    return run_mx8<false>(b, tile_meta, st);
}

}  // namespace unipool
