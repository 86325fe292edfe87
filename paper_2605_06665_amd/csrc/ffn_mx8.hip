// The pool's experts forward on 8-bit rows with 8-bit weights (MX8, mx8.h):
//   A = X_e W_gate,e^T;  B = X_e W_up,e^T;  H = silu(A) * B, to MX8;  Y = H W_down,e^T, to bfloat16.
//
// The products are v_mfma_scale_f32_16x16x128_f8f6f4 on e4m3 operands: one instruction multiplies 16 weight rows by 16
// activation rows over 128 indices and applies the scale of every block of 32 on the way.  Lane l holds row l % 16 of its
// operand, indices 16 g .. 16 g + 15 and 64 + 16 g .. with g = l / 16 (two 16-byte pieces), and brings the scale byte of block g
// of that row (checked on the device with one-hot operands).  Sums over the instructions are float; inside one the products of
// neighbouring indices are added with the terms kept to 2^-13 of the largest (measured; on Gaussian operands 1.5e-5 of the result,
// against the 1.7e-3 of its rounding to bfloat16).  The 16x16x32 form adds the same way at half the rate.
#include <algorithm>
#include <cmath>

#include "gemm_common.h"
#include "few_rows.h"
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
    const int32_t* offsets;
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

// 32 columns of H of row `row`, from the sums of gate (a0, a1: 16 columns each) and up (b0, b1): the lanes l16, l16 + 16, .. of a row hold
// 8 values each and agree on the scale of the block.  Every lane takes part; on: the row exists.
__device__ __forceinline__ void store_h(const Mx8Args& a, const f32x4& a0, const f32x4& a1, const f32x4& b0, const f32x4& b1, bool on,
                                        long long row, int col, int lg) {
    float h[8];
    unsigned mag = 0;
#pragma unroll
    for (int i = 0; i < 4; i++) {
        h[i] = silu_f(a0[i]) * b0[i];
        h[4 + i] = silu_f(a1[i]) * b1[i];
    }
#pragma unroll
    for (int i = 0; i < 8; i++) mag = max(mag, mx8_mag(h[i]));
    mag = max(mag, (unsigned)__shfl_xor((int)mag, 16, 64));
    mag = max(mag, (unsigned)__shfl_xor((int)mag, 32, 64));
    const int byte = mx8_scale_byte(mag);
    if (!on) return;
    unsigned char* dst = a.h + row * a.N + col + 4 * lg;
    *reinterpret_cast<unsigned*>(dst) = mx8_pack4(h[0], h[1], h[2], h[3], byte);
    *reinterpret_cast<unsigned*>(dst + 16) = mx8_pack4(h[4], h[5], h[6], h[7], byte);
    if (lg == 0) a.h_scale[mx8_scale_at(a.S, row, col / kMxBlock)] = (unsigned char)byte;
}

// What a reduction whose length is no multiple of 128 reads past its end.  Never written.
__device__ __align__(256) uint32_t g_mx8_zero_page[64];

// 64 lanes x 4 bytes -> LDS[lds_addr + 4 lane]
__device__ __forceinline__ void glds4(const void* gptr, unsigned lds_addr) {
    const unsigned base = __builtin_amdgcn_readfirstlane(lds_addr);
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dword %0, off"
                 :
                 : "v"(gptr), "s"(base)
                 : "memory", "m0");
}

// Tile of BM rows by 256 weight rows (gate-up: 128 gate rows and the 128 up rows they meet), eight wavefronts: wavefront (wm, wn)
// owns 64 weight rows and every second fragment of 16 rows starting at wm.  Fragments without rows are skipped.
//
// A workgroup is persistent and its tiles form one stream of stages of 128 indices: while a stage is multiplied, the next ones land
// in rings of LDS buffers (NSX of rows, NSW of weights and scales), whatever tile they belong to, so a tile starts with its first
// stages in place and its epilogue runs beside the loads of the next.  A wavefront waits for its own loads of the next stage
// and meets the others once per stage; the buffers that the meeting frees are filled by the loads that are spread over the next stage.
template <bool GATE_UP, int BM, int NSX, int NSW> struct Mx8Tile {
    static constexpr int BN = 256, NW = 8, ROWB = kMxStep;
    static constexpr int XBYTES = BM * ROWB, WBYTES = BN * ROWB, SBYTES = (BN + BM) * 4;
    static constexpr int XI = XBYTES / (NW * 1024), WI = WBYTES / (NW * 1024);      // 1 KB loads of a wavefront
    static constexpr int MF = BM / 32;                    // fragments of a wavefront
    static constexpr int WBASE = NSX * XBYTES, SBASE = WBASE + NSW * WBYTES;
    static constexpr int LDS = SBASE + NSW * SBYTES;
    static_assert(LDS <= 160 * 1024 && NSX >= 2 && NSX <= NSW, "the rings fit a compute unit");
    static constexpr int COLS = GATE_UP ? BN / 2 : BN;    // output columns
};

template <bool GATE_UP, int BM, int NSX, int NSW>
__global__ __launch_bounds__(512, 2) void ffn_mx8_kernel(const Mx8Args a) {
    using C = Mx8Tile<GATE_UP, BM, NSX, NSW>;
    constexpr int XI = C::XI, WI = C::WI, MF = C::MF, BN = C::BN;
    extern __shared__ __attribute__((aligned(1024))) char smem[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int l16 = lane & 15, lg = lane >> 4, wm = wave & 1, wn = wave >> 1;
    const unsigned lds0 = lds_addr_of(smem);
    const int nk = (a.K + kMxStep - 1) / kMxStep;
    const char* const zeros = reinterpret_cast<const char*>(g_mx8_zero_page);
    // 16-byte piece ch of a row lies at place ch ^ ((row / 2) & 7) of its 128 bytes, so that 16 rows' pieces lie in different banks
    auto swz = [](int row) { return (row >> 1) & 7; };

    // ---- load cursors: the stages of rows run NSX - 1 ahead of the multiplication, those of weights and scales NSW - 1 -------------
    TileWalk xwalk(a.g), wwalk(a.g);
    bool xon, won;
    int xkt = 0, wkt = 0, xbuf = 0, wbuf = 0;
    const char *xsrc[XI], *wsrc[WI], *ssrc;
    // (loads 8 rows apart differ by whole rows: the piece a lane fetches is the same in all of them)
    const int piece = ((lane & 7) ^ swz(wave * 8 + (lane >> 3))) * 16;
    const long long sstep = wave < 4 ? (long long)a.E * a.w_rows * 4 : a.x_rows * 4;
    auto row_of = [&](const TileRef& t, int r) {
        const int row = t.row0 + min(r, t.rows - 1);
        return (long long)(a.gather ? a.gather[row] / a.gather_div : row);
    };
    auto weight_of = [&](const TileRef& t, int r) {
        const int n0 = t.nt * C::COLS;
        const int c = GATE_UP ? min(n0 + (r & (BN / 2 - 1)), a.N - 1) + (r / (BN / 2)) * a.N : min(n0 + r, a.N - 1);
        return (long long)t.expert * a.w_rows + c;
    };
    auto next_x = [&]() {
        const TileRef t = xwalk.next(a.g);
        xon = t.valid;
        xkt = 0;
        if (!xon) return;
#pragma unroll
        for (int i = 0; i < XI; i++)
            xsrc[i] = reinterpret_cast<const char*>(a.x) + row_of(t, (i * C::NW + wave) * 8 + (lane >> 3)) * a.K + piece;
    };
    auto next_w = [&]() {
        const TileRef t = wwalk.next(a.g);
        won = t.valid;
        wkt = 0;
        if (!won) return;
#pragma unroll
        for (int i = 0; i < WI; i++)
            wsrc[i] = reinterpret_cast<const char*>(a.w) + weight_of(t, (i * C::NW + wave) * 8 + (lane >> 3)) * a.K + piece;
        // scales: one load a wavefront, of 64 weight rows or 64 rows (some of them twice where there are fewer)
        if (wave < 4) ssrc = reinterpret_cast<const char*>(a.w_scale) + weight_of(t, wave * 64 + lane) * 4;
        else ssrc = reinterpret_cast<const char*>(a.x_scale) + row_of(t, (wave - 4) % (BM / 64) * 64 + lane) * 4;
    };
    const unsigned sdst = lds0 + C::SBASE + (wave < 4 ? wave * 256 : BN * 4 + (wave - 4) % (BM / 64) * 256);
    // load i of the cursors' stages: first the rows, then the weights, last the scales
    auto issue = [&](int i) {
        if (i < XI) {
            if (xon) {
                const char* src = xkt * kMxStep + piece < a.K ? xsrc[i < XI ? i : 0] + (size_t)xkt * kMxStep : zeros;
                glds16(src, lds0 + xbuf * C::XBYTES + (i * C::NW + wave) * 1024);
            }
        } else if (i < XI + WI) {
            const int u = i - XI;
            if (won) {
                const char* src = wkt * kMxStep + piece < a.K ? wsrc[u >= 0 && u < WI ? u : 0] + (size_t)wkt * kMxStep : zeros;
                glds16(src, lds0 + C::WBASE + wbuf * C::WBYTES + (u * C::NW + wave) * 1024);
            }
        } else if (won) {
            glds4(ssrc + wkt * sstep, sdst + wbuf * C::SBYTES);
        }
    };
    constexpr int NL = XI + WI + 1;
    auto advance_x = [&]() {
        xbuf = xbuf + 1 == NSX ? 0 : xbuf + 1;
        if (xon && ++xkt == nk) next_x();
    };
    auto advance_w = [&]() {
        wbuf = wbuf + 1 == NSW ? 0 : wbuf + 1;
        if (won && ++wkt == nk) next_w();
    };
    next_x();
    next_w();
    for (int s = 0; s < NSW - 1; s++) {
        if (s < NSX - 1) {
#pragma unroll
            for (int i = 0; i < XI; i++) issue(i);
            advance_x();
        }
#pragma unroll
        for (int i = XI; i < NL; i++) issue(i);
        advance_w();
    }
    wait_vmcnt<0>();
    lds_barrier();

    // ---- the tiles ------------------------------------------------------------------------------------------
    TileWalk walk(a.g);
    int cx = 0, cw = 0;                                    // ring places of the stage that is multiplied
    const int woff = l16 * C::ROWB, p0 = (lg ^ swz(l16)) * 16, p1 = ((4 + lg) ^ swz(l16)) * 16;
    for (TileRef t = walk.next(a.g); t.valid; t = walk.next(a.g)) {
        const int n0 = t.nt * C::COLS;
        const int col = n0 + wn * (GATE_UP ? 32 : 64);     // the wavefront's columns are inside N or outside as a whole
        const int mi = col < a.N ? (((t.rows + 15) >> 4) - wm + 1) >> 1 : 0;
        f32x4 acc[MF][4];
#pragma unroll
        for (int m = 0; m < MF; m++)
#pragma unroll
            for (int n = 0; n < 4; n++) acc[m][n] = f32x4{0.f, 0.f, 0.f, 0.f};
        for (int kt = 0; kt < nk; kt++) {
            const char* xb = smem + cx * C::XBYTES;
            const char* wb = smem + C::WBASE + cw * C::WBYTES;
            const unsigned char* sb = reinterpret_cast<const unsigned char*>(smem) + C::SBASE + cw * C::SBYTES;
            // past the end of K the values are zeros; their scales must not be NaN
            const bool tail = kt * kMxStep + lg * kMxBlock >= a.K;
            i32x8 wf[4];
            int wsb[4];
#pragma unroll
            for (int n = 0; n < 4; n++) {
                const int r = GATE_UP ? (n >> 1) * (BN / 2) + wn * 32 + (n & 1) * 16 : wn * 64 + n * 16;
                const char* p = wb + r * C::ROWB + woff;
                wf[n] = two16(*reinterpret_cast<const uint4*>(p + p0), *reinterpret_cast<const uint4*>(p + p1));
                wsb[n] = sb[(r + l16) * 4 + lg];
            }
#pragma unroll
            for (int n = 0; n < 4; n++) wsb[n] = tail ? kMxBias : wsb[n];
            const bool w_issued = won;
#pragma unroll
            for (int m = 0; m < MF; m++) {
                if (m < mi) {
                    const int r = (2 * m + wm) * 16;
                    const char* p = xb + r * C::ROWB + woff;
                    const i32x8 xf = two16(*reinterpret_cast<const uint4*>(p + p0), *reinterpret_cast<const uint4*>(p + p1));
                    int xsb = sb[(BN + r + l16) * 4 + lg];
                    xsb = tail ? kMxBias : xsb;
#pragma unroll
                    for (int n = 0; n < 4; n++)
                        acc[m][n] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wf[n], xf, acc[m][n], 0, 0, 0, wsb[n], 0, xsb);
                }
#pragma unroll
                for (int i = m * NL / MF; i < (m + 1) * NL / MF; i++) issue(i);
            }
            advance_x();
            advance_w();
            // the loads of the next stage have landed: only what was issued behind them may be outstanding
            if (w_issued) wait_vmcnt<NSX == NSW ? (NSW - 2) * NL : (NSW - 2) * (WI + 1)>();
            else wait_vmcnt<0>();
            lds_barrier();
            cx = cx + 1 == NSX ? 0 : cx + 1;
            cw = cw + 1 == NSW ? 0 : cw + 1;
        }
        // acc[m][n][i] = C[row 16 (2 m + wm) + l16][weight row 16 n + 4 lg + i of the wavefront's 64]
#pragma unroll
        for (int m = 0; m < MF; m++) {
            if (m >= mi) break;
            const int r = (2 * m + wm) * 16 + l16;
            const bool on = r < t.rows;
            const long long row = t.row0 + r;
            if constexpr (GATE_UP) {
                store_h(a, acc[m][0], acc[m][1], acc[m][2], acc[m][3], on, row, col, lg);
            } else {
#pragma unroll
                for (int n = 0; n < 4; n++)
                    if (on)
                        *reinterpret_cast<uint2*>(a.y + row * a.N + col + n * 16 + 4 * lg) =
                            pack4(acc[m][n][0], acc[m][n][1], acc[m][n][2], acc[m][n][3]);
            }
        }
    }
}

template <bool GATE_UP, int BM, int NSX, int NSW> hipError_t run_tile(Mx8Args a, hipStream_t st) {
    using C = Mx8Tile<GATE_UP, BM, NSX, NSW>;
    auto kern = ffn_mx8_kernel<GATE_UP, BM, NSX, NSW>;
    static bool attr_set = false;
    if (!attr_set) {
        hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, C::LDS);
        if (e != hipSuccess) return e;
        attr_set = true;
    }
    a.g.group_m = BM > 128 ? 2 : 1;
    a.g.n_tiles_n = cdiv(a.N, C::COLS);
    kern<<<max(kNumXcd, num_cus() / kNumXcd * kNumXcd), 512, C::LDS, st>>>(a);
    return hipGetLastError();
}

// Rows of a tile: one tile for most experts where that is possible.
int tile_bm(const unipool_shape& s) {
    const double S = (double)s.T * s.k, used = s.E * -std::expm1(-S / s.E), r = S / used;       // rows of an expert that has any
    const double most = r + 2.0 * std::sqrt(r);
    return most <= 64 ? 64 : most <= 128 ? 128 : 192;
}

template <bool GATE_UP> hipError_t run_mx8(const unipool_shape& s, const Mx8Args& a, hipStream_t st) {
    switch (tile_bm(s)) {
        case 64: return run_tile<GATE_UP, 64, 3, 3>(a, st);
        case 128: return run_tile<GATE_UP, 128, 3, 3>(a, st);
        default: return run_tile<GATE_UP, 192, 2, 3>(a, st);
    }
}

// ---------------------------------------------------------------------------------------------
// Few rows per expert (decoding, short prompts): one pass over the weights of the experts that have rows, bound by the bytes that are
// in flight.  A wavefront owns 16 NF weight rows of one expert (gate-up: 32 gate rows and the 32 up rows they meet, which are a whole
// block of H) for all rows of the expert; weights go from memory to registers, whole 128-byte lines at a time (few_rows.h), D
// steps of 128 indices ahead, with no LDS and no barrier.
// ---------------------------------------------------------------------------------------------
template <typename V> __device__ __forceinline__ i32x8 two16(const V& a, const V& b) {
    union { V v[2]; i32x8 i; } u;
    u.v[0] = a;
    u.v[1] = b;
    return u.i;
}

template <bool GATE_UP, int NF, int R, int D>
__device__ __forceinline__ void few_mx8_task(const Mx8Args& a, int e, int c0, int row0, int rows, int lane) {
    static_assert(!GATE_UP || NF == 4, "32 gate and 32 up rows");
    const int l16 = lane & 15, lg = lane >> 4;
    const int chunk = few_chunk(lane);
    const int nk = (a.K + kMxStep - 1) / kMxStep;
    const bool half = a.K % kMxStep != 0;                  // the last step has 64 indices
    // addresses are a wave-uniform base and a 32-bit offset per lane (at most 512 rows, and 16 rows of weights)
    unsigned xo[R], xso[R];
#pragma unroll
    for (int r = 0; r < R; r++) {
        int row = row0 + min(16 * r + l16, rows - 1);
        if (a.gather != nullptr) row = a.gather[row] / a.gather_div;
        xo[r] = (unsigned)row * (unsigned)a.K + 16 * lg;
        xso[r] = (unsigned)row * 4 + lg;
    }
    const unsigned wo = (unsigned)(lane & 7) * (unsigned)a.K + 16 * chunk, wso = l16 * 4 + lg;
    // in a half step the pieces past the end are read from the first half: any finite value will do beside rows of zeros
    const unsigned wo_cut = wo - (chunk >= 4 ? 64 : 0);
    const unsigned char* const we = a.w + ((size_t)e * a.w_rows + c0) * a.K;
    const unsigned char* const wse = a.w_scale + ((size_t)e * a.w_rows + c0) * 4;
    const size_t w_plane = (size_t)a.E * a.w_rows * 4, x_plane = (size_t)a.x_rows * 4;
    u32x4v wq[D][NF][2];
    u32x4v xq[D][R][2];
    int ws[D][NF], xs[D][R];
    f32x4 acc[R][NF];
#pragma unroll
    for (int r = 0; r < R; r++)
#pragma unroll
        for (int f = 0; f < NF; f++) acc[r][f] = f32x4{0.f, 0.f, 0.f, 0.f};
    // wave-uniform addresses of the step that is requested next; past the end it stays the last one, whose values are never used
    const unsigned char *wk = we, *wsk = wse, *xk = a.x, *xsk = a.x_scale;
    int next = 0;
    auto fetch = [&](int u) {
        const bool last = next == nk - 1;
        const bool cut = half && last;
        unsigned o = cut ? wo_cut : wo, so = wso;
        // (known to the compiler as 32-bit offsets right here: widened outside the loop they would be added to every base in vector registers)
        asm volatile("" : "+v"(o), "+v"(so));
#pragma unroll
        for (int f = 0; f < NF; f++) {
            const size_t fr = GATE_UP ? (size_t)(f >> 1) * a.N + 16 * (f & 1) : 16 * f;
#pragma unroll
            for (int h = 0; h < 2; h++)
                wq[u][f][h] = __builtin_nontemporal_load(reinterpret_cast<const u32x4v*>(wk + (fr + h * 8) * a.K + o));
            ws[u][f] = (wsk + fr * 4)[so];
        }
#pragma unroll
        for (int r = 0; r < R; r++) {
            unsigned q = xo[r], p = xso[r];
            asm volatile("" : "+v"(q), "+v"(p));
            xq[u][r][0] = *reinterpret_cast<const u32x4v*>(xk + q);
            xq[u][r][1] = *reinterpret_cast<const u32x4v*>(xk + (cut ? 0 : 64) + q);
            xs[u][r] = xsk[p];
        }
        next += last ? 0 : 1;
        wk += last ? 0 : kMxStep;
        xk += last ? 0 : kMxStep;
        wsk += last ? 0 : w_plane;
        xsk += last ? 0 : x_plane;
    };
    // last: a half step's second half counts as zeros, with scales that are not NaN
    auto multiply = [&](int u, bool last) {
        const bool cut = half && last;
#pragma unroll
        for (int r = 0; r < R; r++) {
            if (cut) xq[u][r][1] = u32x4v{0, 0, 0, 0};
            if (cut && lg >= 2) xs[u][r] = kMxBias;
        }
#pragma unroll
        for (int f = 0; f < NF; f++) {
            bf16x8 first, second;
            few_fragments(wq[u][f][0], wq[u][f][1], first, second);
            const i32x8 w = two16(first, second);
            if (cut && lg >= 2) ws[u][f] = kMxBias;
#pragma unroll
            for (int r = 0; r < R; r++)
                acc[r][f] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w, two16(xq[u][r][0], xq[u][r][1]), acc[r][f], 0, 0, 0,
                                                                            ws[u][f], 0, xs[u][r]);
        }
    };
#pragma unroll
    for (int u = 0; u < D; u++) fetch(u);
    int s = 0;
    for (; s + D < nk; s += D) {
#pragma unroll
        for (int u = 0; u < D; u++) {
            multiply(u, false);
            fetch(u);
            __builtin_amdgcn_sched_barrier(0);
        }
    }
#pragma unroll
    for (int u = 0; u < D; u++)
        if (s + u < nk) multiply(u, s + u == nk - 1);
    // acc[r][f][i] = C[row 16 r + l16][weight row 16 f + 4 lg + i]
#pragma unroll
    for (int r = 0; r < R; r++) {
        const bool on = 16 * r + l16 < rows;
        const long long row = row0 + 16 * r + l16;
        if constexpr (GATE_UP) {
            store_h(a, acc[r][0], acc[r][1], acc[r][2], acc[r][3], on, row, c0, lg);
        } else {
#pragma unroll
            for (int f = 0; f < NF; f++)
                if (on)
                    *reinterpret_cast<uint2*>(a.y + row * a.N + c0 + 16 * f + 4 * lg) =
                        pack4(acc[r][f][0], acc[r][f][1], acc[r][f][2], acc[r][f][3]);
        }
    }
}

// RM: most fragments of 16 rows per pass over an expert's weights; D1, DM: steps in flight with one and with RM of them
template <bool GATE_UP, int NF, int WAVES, int RM, int D1, int DM>
__global__ __launch_bounds__(64 * WAVES, WAVES == 1 ? 1 : GATE_UP ? 2 : 3) void few_mx8_kernel(const Mx8Args a) {
    __shared__ int list_e[kMaxE], list_r0[kMaxE], list_n[kMaxE];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int n_list = few_experts<WAVES>(a.offsets, a.E, list_e, list_r0, list_n);
    constexpr int COLS = GATE_UP ? 32 : 16 * NF;
    const int per_e = a.N / COLS, tasks = n_list * per_e;
    for (int t = blockIdx.x * WAVES + wave; t < tasks; t += gridDim.x * WAVES) {
        const int i = t / per_e, c0 = (t % per_e) * COLS;
        const int e = __builtin_amdgcn_readfirstlane(list_e[i]);
        const int r0 = __builtin_amdgcn_readfirstlane(list_r0[i]);
        const int n = __builtin_amdgcn_readfirstlane(list_n[i]);
        for (int c = 0; c < n; c += 16 * RM) {
            const int rows = min(n - c, 16 * RM);
            if (RM == 1 || rows <= 16) few_mx8_task<GATE_UP, NF, 1, D1>(a, e, c0, r0 + c, rows, lane);
            else few_mx8_task<GATE_UP, NF, RM, DM>(a, e, c0, r0 + c, rows, lane);
        }
    }
}

template <bool GATE_UP> hipError_t run_few_mx8(const unipool_shape& s, const Mx8Args& a, hipStream_t st) {
    constexpr int NF = GATE_UP ? 4 : 1;
    const int S = s.T * s.k, cus = num_cus();
    const int most = std::min(S, s.E) * (a.N / (GATE_UP ? 32 : 16));        // tasks if every row had an expert of its own
    const bool one = s.T <= 16;                            // an expert gets a token at most once
    // At most one wavefront per SIMD: all its registers hold steps in flight.
    if (most <= 4 * cus) {
        constexpr int D1 = GATE_UP ? 6 : 16, DM = GATE_UP ? 5 : 8;
        if (one) few_mx8_kernel<GATE_UP, NF, 1, 1, D1, D1><<<most, 64, 0, st>>>(a);
        else few_mx8_kernel<GATE_UP, NF, 1, 2, D1, DM><<<most, 64, 0, st>>>(a);
        return hipGetLastError();
    }
    constexpr int D1 = GATE_UP ? 3 : 6, DM = GATE_UP ? 2 : 4;
    const int blocks = std::min(cdiv(most, 4), 4 * cus);
    if (one) few_mx8_kernel<GATE_UP, NF, 4, 1, D1, D1><<<blocks, 256, 0, st>>>(a);
    else few_mx8_kernel<GATE_UP, NF, 4, 2, D1, DM><<<blocks, 256, 0, st>>>(a);
    return hipGetLastError();
}

bool few_mx8(const unipool_shape& s) { return s.T <= 16 || (s.T <= 64 && s.T * s.k <= 8 * s.E); }

}  // namespace

hipError_t mx8_ffn_fwd(const unipool_shape& s, const void* x, const void* x_scale, const int32_t* slot_of_row, const int32_t* offsets,
                       const void* wgu, const void* wgu_scale, const void* wd, const void* wd_scale, void* h, void* h_scale, void* y,
                       int32_t* tile_meta, hipStream_t st) {
    const bool few = few_mx8(s);
    hipError_t e = few ? hipSuccess : mfma_build_tiles(s, offsets, tile_bm(s), tile_meta, st);
    if (e != hipSuccess) return e;
    const long long S = (long long)s.T * s.k;
    Mx8Args a = {};
    a.g.tile_meta = tile_meta;
    a.offsets = offsets;
    a.x = (const unsigned char*)x; a.x_scale = (const unsigned char*)x_scale;
    a.x_rows = slot_of_row ? s.T : S;
    a.gather = slot_of_row; a.gather_div = s.k;
    a.w = (const unsigned char*)wgu; a.w_scale = (const unsigned char*)wgu_scale;
    a.w_rows = 2 * s.d_ff; a.E = s.E;
    a.K = s.d_model; a.N = s.d_ff;
    a.h = (unsigned char*)h; a.h_scale = (unsigned char*)h_scale; a.S = S;
    e = few ? run_few_mx8<true>(s, a, st) : run_mx8<true>(s, a, st);
    if (e != hipSuccess) return e;
    Mx8Args b = {};
    b.g.tile_meta = tile_meta;
    b.offsets = offsets;
    b.x = (const unsigned char*)h; b.x_scale = (const unsigned char*)h_scale;
    b.x_rows = S;
    b.w = (const unsigned char*)wd; b.w_scale = (const unsigned char*)wd_scale;
    b.w_rows = s.d_model; b.E = s.E;
    b.K = s.d_ff; b.N = s.d_model;
    b.y = (bf16*)y; b.S = S;
    return few ? run_few_mx8<false>(s, b, st) : run_mx8<false>(s, b, st);
}

}  // namespace unipool
