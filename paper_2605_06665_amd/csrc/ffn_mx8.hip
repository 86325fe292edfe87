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
    GemmArgs g;                      // tile list only (n_tiles_n, group_m)
    const unsigned char* x;          // [rows][K], or the tokens when gather is given
    const unsigned char* x_scale;    // [ceil(K / 128)][x_rows][4]
    long long x_rows;                // of x_scale
    const int32_t* gather;           // row r is row gather[r] / gather_div of x, and of x_scale if scales_too
    bool scales_too;
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

// 32 columns of H of a row, from the sums of gate (a0, a1: 16 columns each) and up (b0, b1): the lanes l16, l16 + 16, .. of a row hold
// 8 values each (columns 4 lg .. and 16 + 4 lg ..) and agree on the scale of the block.  Every lane takes part.
__device__ __forceinline__ int block_of_h(const f32x4& a0, const f32x4& a1, const f32x4& b0, const f32x4& b1, unsigned& lo, unsigned& hi) {
    // silu(a) b step by step for all values, so that no instruction waits for the exponential or the reciprocal in front of it
    float h[8], p[8];
#pragma unroll
    for (int i = 0; i < 8; i++) p[i] = __expf(-(i < 4 ? a0[i] : a1[i - 4]));
#pragma unroll
    for (int i = 0; i < 8; i++) p[i] = __builtin_amdgcn_rcpf(1.0f + p[i]);
#pragma unroll
    for (int i = 0; i < 8; i++) h[i] = (i < 4 ? a0[i] : a1[i - 4]) * p[i] * (i < 4 ? b0[i] : b1[i - 4]);
    float m = h[0];
#pragma unroll
    for (int i = 1; i < 8; i++) m = mx8_max(m, h[i]);
    const auto r16 = __builtin_amdgcn_permlane16_swap(__float_as_uint(m), __float_as_uint(m), false, false);
    m = mx8_max(__uint_as_float(r16[0]), __uint_as_float(r16[1]));
    const auto r32 = __builtin_amdgcn_permlane32_swap(__float_as_uint(m), __float_as_uint(m), false, false);
    m = mx8_max(__uint_as_float(r32[0]), __uint_as_float(r32[1]));
    const int byte = mx8_scale_byte(m);
    lo = mx8_pack4(h[0], h[1], h[2], h[3], byte);
    hi = mx8_pack4(h[4], h[5], h[6], h[7], byte);
    return byte;
}
// The scale of such a block, and behind the last one what fills its word.
__device__ __forceinline__ void store_h_scale(const Mx8Args& a, long long row, int col, int byte) {
    unsigned char* const sc = a.h_scale + mx8_scale_at(a.S, row, col / kMxBlock);
    *sc = (unsigned char)byte;
    if (col + kMxBlock == a.N && a.N % kMxStep != 0) sc[1] = sc[2] = kMxBias;
}
// on: the row exists
__device__ __forceinline__ void store_h(const Mx8Args& a, const f32x4& a0, const f32x4& a1, const f32x4& b0, const f32x4& b1, bool on,
                                        long long row, int col, int lg) {
    unsigned lo, hi;
    const int byte = block_of_h(a0, a1, b0, b1, lo, hi);
    if (!on) return;
    unsigned char* dst = a.h + row * a.N + col + 4 * lg;
    *reinterpret_cast<unsigned*>(dst) = lo;
    *reinterpret_cast<unsigned*>(dst + 16) = hi;
    if (lg == 0) store_h_scale(a, row, col, byte);
}

// v[i] of group lg of 16 lanes -> v[lg] of group i
__device__ __forceinline__ uint4 lane_groups_transposed(unsigned v0, unsigned v1, unsigned v2, unsigned v3) {
    const auto a = __builtin_amdgcn_permlane32_swap(v0, v2, false, false), b = __builtin_amdgcn_permlane32_swap(v1, v3, false, false);
    const auto lo = __builtin_amdgcn_permlane16_swap(a[0], b[0], false, false), hi = __builtin_amdgcn_permlane16_swap(a[1], b[1], false, false);
    return make_uint4(lo[0], lo[1], hi[0], hi[1]);
}

// u and v of four groups of 16 lanes -> u0 u2 v0 v2 and u1 u3 v1 v3
__device__ __forceinline__ void pair_lane_groups(unsigned u, unsigned v, unsigned& even, unsigned& odd) {
    const auto a = __builtin_amdgcn_permlane32_swap(u, v, false, false);
    const auto b = __builtin_amdgcn_permlane16_swap(a[0], a[1], false, false);
    even = b[0];
    odd = b[1];
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

// The tile list.  The rows of an expert are cut into equal tiles of at most BM rows (multiples of 16); with BM > 128 an expert takes an
// even number of places, since the two row tiles of a pair run side by side and share their weights through L2.  Every workgroup
// counts the places for itself (place[e]: those of the experts before e), which takes a fraction of a launch.
__device__ __forceinline__ int row_tiles_of(int rows, int bm) {
    const int n = (rows + bm - 1) / bm;
    return bm > 128 ? (n + 1) & ~1 : n;
}
__device__ __forceinline__ void count_places(const int32_t* offsets, int E, int bm, int* place) {
    constexpr int PER = kMaxE / 64;
    if (threadIdx.x < 64) {
        int n[PER], sum = 0;
#pragma unroll
        for (int i = 0; i < PER; i++) {
            const int e = threadIdx.x * PER + i;
            n[i] = e < E ? offsets[e + 1] - offsets[e] : 0;
        }
#pragma unroll
        for (int i = 0; i < PER; i++) {
            n[i] = row_tiles_of(n[i], bm);
            sum += n[i];
        }
        int upto = sum;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int o = __shfl_up(upto, d, 64);
            if ((int)threadIdx.x >= d) upto += o;
        }
        int at = upto - sum;
#pragma unroll
        for (int i = 0; i < PER; i++) {
            place[threadIdx.x * PER + i] = at;
            at += n[i];
        }
        if (threadIdx.x == 63) place[kMaxE] = at;
    }
    __syncthreads();
}

// The tiles of a workgroup in the order of TileWalk, 64 at a time: lane i holds the tile of round base + i, so the divisions and the
// search of a tile are done once for 64 of them.
struct TileList {
    int next, base;                  // round that comes next; round of lane 0
    int rows, expert, row0, nt;      // per lane; rows: 0 a place without a tile, -1 past the end
};
__device__ __forceinline__ void tiles_at(TileList& l, const Mx8Args& a, const int* place, int bm, int round0, int lane) {
    const GemmArgs& g = a.g;
    const int n_mt = place[kMaxE], G = g.group_m, per_group = G * g.n_tiles_n;
    const int total = ((n_mt + G - 1) / G) * per_group, per_xcd = (total + kNumXcd - 1) / kNumXcd;
    const int xcd = blockIdx.x % kNumXcd, slot = blockIdx.x / kNumXcd, P = gridDim.x / kNumXcd;
    const int round = round0 + lane, lt = xcd * per_xcd + round * P + (slot + round) % P;
    l.next = l.base = round0;
    l.rows = l.expert = l.row0 = l.nt = 0;
    if (lt >= min(total, (xcd + 1) * per_xcd)) {
        l.rows = -1;
        return;
    }
    const int rem = lt % per_group, mt = lt / per_group * G + rem % G;
    if (mt >= n_mt) return;
    int e = 0;                       // the last expert whose first place is not behind mt
#pragma unroll
    for (int step = kMaxE / 2; step > 0; step >>= 1)
        if (place[e + step] <= mt) e += step;
    const int r0 = a.offsets[e], rows = a.offsets[e + 1] - r0;
    const int n = (rows + bm - 1) / bm, per = ((rows + n - 1) / n + 15) / 16 * 16, i = mt - place[e];
    l.expert = e;
    l.row0 = r0 + i * per;
    l.rows = max(0, min(per, rows - i * per));
    l.nt = rem / G;
}
__device__ __forceinline__ TileRef next_tile(TileList& l, const Mx8Args& a, const int* place, int bm, int lane) {
    TileRef t = {0, 0, 0, 0, 0, -1};
    for (;;) {
        if (l.next - l.base == 64) tiles_at(l, a, place, bm, l.next, lane);
        const int i = l.next - l.base;
        const int rows = __builtin_amdgcn_readlane(l.rows, i);
        if (rows < 0) return t;
        l.next++;
        if (rows == 0) continue;
        t.valid = 1;
        t.rows = rows;
        t.expert = __builtin_amdgcn_readlane(l.expert, i);
        t.row0 = __builtin_amdgcn_readlane(l.row0, i);
        t.nt = __builtin_amdgcn_readlane(l.nt, i);
        return t;
    }
}

// Tile of BM rows by BN = 256 weight rows (gate-up: 128 gate rows and the 128 up rows they meet), eight wavefronts: wavefront (wm, wn)
// owns 64 weight rows and every second fragment of 16 rows starting at wm.  Fragments without rows are multiplied like the others: the tile's time
// is that of its loads, and one straight body keeps the accumulators where they are (a body per number of fragments, as alternatives of one
// switch, had the compiler move and spill them).
//
// A workgroup is persistent and its tiles form one stream of stages of 128 indices, whatever tile they belong to: rings of LDS buffers
// (NSX of rows, NSW of weights and scales) are filled ahead across tiles, so a tile starts with its first stages in place and its
// epilogue runs beside the loads of the next.
// A stage has two parts.  In the first the wavefront multiplies all but its last two fragments, fetching the rows' fragments two ahead, while
// the loads of weights go out that fill the buffer the stage before has released.  Then the wavefronts meet: everyone's loads of the next stage have landed and nobody reads
// this one any more.  The second part multiplies the last two fragments from registers, and while it does the weights' fragments are replaced
// by the next stage's, the next stage's first rows are fetched, and the loads of rows go out into the buffer that has become free.
//
// 192 experts of 1536 x 4096, 32768 tokens, k = 2 (341 rows an expert, 192 x 256): gate-up 1050 us, down 490; 1.6 PFLOP/s, matrix pipes
// busy half of the time.  What bounds it is delivery into LDS, of which two stages are in flight: without the loads 0.65 of the time,
// without the products 0.81, with all weights from L2 0.88, all rows from L2 0.96; 128 rows instead of 192 1.16.  The epilogue
// (SwiGLU, scales, stores) takes 0.11.
// 90 experts of 832 x 1472, 1501 tokens, hot (96 x 128): 66 and 37 us, 340 MB of weights at 3.3 TB/s; 512 experts of 1024 x 704, 48 tokens, k = 8
// (64 x 128): 74 and 44 us, 5.1 TB/s.
template <bool GATE_UP, int BM, int BNN, int NSX, int NSW> struct Mx8Tile {
    static constexpr int BN = BNN, NW = BN / 32, ROWB = kMxStep;
    static constexpr int XBYTES = BM * ROWB, WBYTES = BN * ROWB, SBYTES = (BN + (BM + 63) / 64 * 64) * 4;
    static constexpr int XI = XBYTES / (NW * 1024), WI = WBYTES / (NW * 1024);      // 1 KB loads of a wavefront
    static constexpr int MF = BM / 32;                    // fragments of a wavefront
    static constexpr int WBASE = NSX * XBYTES, SBASE = WBASE + NSW * WBYTES, GBASE = SBASE + NSW * SBYTES;
    static constexpr int GROWS = (BM + 63) / 64 * 64;     // looked-up rows of a tile
    static constexpr int PBASE = GBASE + 2 * GROWS * 4;
    static constexpr int LDS = PBASE + (kMaxE + 1) * 4;
    static constexpr int WG = NW == 8 ? 1 : 2;            // workgroups of a compute unit
    static_assert(WG * LDS <= 160 * 1024 && NSX >= 2 && NSW == 3 && NSX <= NSW, "the rings fit a compute unit");
    static_assert(XBYTES % (NW * 1024) == 0 && (NW == 8 || NW == 4), "whole loads");
    // scales: the words of 64 rows a load, by wavefronts 0 ..; the weights' by the last ones, all of them in one load where a row group has 256
    static constexpr int XS = (BM + 63) / 64, WS = NW == 8 ? 1 : 2;
    static_assert(XS + WS <= NW, "one load of scales a wavefront");
    static constexpr int COLS = GATE_UP ? BN / 2 : BN;    // output columns
};

template <bool GATE_UP, int BM, int BN_, int NSX, int NSW>
__global__ __launch_bounds__(2 * BN_, 2) void ffn_mx8_kernel(const Mx8Args a) {
    using C = Mx8Tile<GATE_UP, BM, BN_, NSX, NSW>;
    constexpr int XI = C::XI, WI = C::WI, MF = C::MF, BN = C::BN;
    extern __shared__ __attribute__((aligned(1024))) char smem[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int l16 = lane & 15, lg = lane >> 4, wm = wave & 1, wn = wave >> 1;
    const bool x_scales = wave < C::XS, w_scales = wave >= C::NW - C::WS;
    const unsigned lds0 = lds_addr_of(smem);
    const int nk = (a.K + kMxStep - 1) / kMxStep;
    const bool half = a.K % kMxStep != 0;                  // the last stage of a tile has 64 indices
    // 16-byte piece ch of a row lies at place ch ^ ((row / 2) & 7) of its 128 bytes, so that 16 rows' pieces lie in different banks
    auto swz = [](int row) { return (row >> 1) & 7; };

    // ---- load cursors ---------------------------------------------------------------------------------------
    int* const place = reinterpret_cast<int*>(smem + C::PBASE);
    count_places(a.offsets, a.E, BM, place);
    TileList xlist, wlist;
    tiles_at(xlist, a, place, BM, 0, lane);
    wlist = xlist;
    TileList clist = xlist;
    bool xon, won;
    int xkt = 0, wkt = 0, xtile = -1, wtile = -1;
    unsigned xdst = 0, wdst = 0, sdst = 0;                 // ring places, in bytes
    const char *xsrc[XI], *wbase, *ssrc;
    constexpr int WV = GATE_UP ? WI / 2 : WI;              // gate and up rows of a lane lie at the same offsets from their first rows
    unsigned woff[WV];
    // (loads 64 rows apart have the same piece in a lane)
    auto piece_of = [&](int ln) { return ((ln & 7) ^ swz(wave * 8 + (ln >> 3))) * 16; };
    const bool upper = piece_of(lane) >= 64;               // absent from a stage of 64 indices: zeros
    const char* const zeros = reinterpret_cast<const char*>(g_mx8_zero_page);
    long long xinc = kMxStep, winc = kMxStep, sinc = w_scales ? (long long)a.E * a.w_rows * 4 : a.x_rows * 4;      // from stage to stage
    // Rows of a gathered tile are looked up while the tile before is loaded: their numbers pass through LDS (two tiles' worth), since a wait
    // for a load to a register would wait for every stage in flight.  They are there two stages later: tiles of one or two are too short.
    const bool by_lds = a.gather != nullptr && nk >= 3;
    bool prologue = true;
    auto row_of = [&](const TileRef& t, int r, int tile) {
        const int row = t.row0 + min(r, t.rows - 1);
        if (a.gather == nullptr) return (long long)row;
        const int slot = by_lds && !prologue ? *reinterpret_cast<const int*>(smem + C::GBASE + ((tile & 1) * C::GROWS + min(r, t.rows - 1)) * 4)
                                             : a.gather[row];
        return (long long)(slot / a.gather_div);
    };
    auto weight_of = [&](const TileRef& t, int r, int n) {         // the first of n neighbours, all inside the matrix
        const int n0 = t.nt * C::COLS;
        const int c = GATE_UP ? min(n0 + (r & (BN / 2 - 1)), a.N - n) + (r / (BN / 2)) * a.N : min(n0 + r, a.N - n);
        return (long long)t.expert * a.w_rows + c;
    };
    // (in what follows the lane number is made opaque, or what depends on it alone would be kept in registers across the stages)
    auto next_x = [&]() {
        int ln = lane;
        asm volatile("" : "+v"(ln));
        const TileRef t = next_tile(xlist, a, place, BM, ln);
        xon = t.valid;
        xkt = 0;
        xtile++;
        if (!xon) {                                        // past the last tile the loads go on, from the page of zeros
            xinc = 0;
#pragma unroll
            for (int i = 0; i < XI; i++) xsrc[i] = zeros;
            return;
        }
        const int r = wave * 8 + (ln >> 3), at = piece_of(ln);
#pragma unroll
        for (int i = 0; i < XI; i++) xsrc[i] = reinterpret_cast<const char*>(a.x) + row_of(t, i * C::NW * 8 + r, xtile) * a.K + at;
    };
    TileRef wnext = next_tile(wlist, a, place, BM, lane);
    if (!wnext.valid) return;                              // no tile for this workgroup
    auto next_w = [&]() {
        int ln = lane;
        asm volatile("" : "+v"(ln));
        const TileRef t = wnext;
        won = t.valid;
        wkt = 0;
        wtile++;
        if (!won) {
            winc = sinc = 0;
            wbase -= kMxStep;
            ssrc = zeros;                                  // (the weights' loads repeat the last stage)
            wkt = nk - 1;
            return;
        }
        const int r = wave * 8 + (ln >> 3), at = piece_of(ln);
#pragma unroll
        for (int i = 0; i < WV; i++) woff[i] = (unsigned)min(i * C::NW * 8 + r, a.N - 1 - t.nt * C::COLS) * (unsigned)a.K + at;
        wbase = reinterpret_cast<const char*>(a.w) + ((long long)t.expert * a.w_rows + t.nt * C::COLS) * a.K;
        if (x_scales) ssrc = reinterpret_cast<const char*>(a.x_scale) + (a.scales_too ? row_of(t, wave * 64 + ln, wtile) : (long long)t.row0 + min(wave * 64 + ln, t.rows - 1)) * 4;
        else if (w_scales) ssrc = reinterpret_cast<const char*>(a.w_scale) + (C::WS == 1 ? weight_of(t, ln * 4, 4) : weight_of(t, (wave - C::NW + C::WS) * 64 + ln, 1)) * 4;
        wnext = next_tile(wlist, a, place, BM, ln);
        if (by_lds && wnext.valid && wave < C::XS)
            glds4(a.gather + wnext.row0 + min(wave * 64 + ln, wnext.rows - 1), lds0 + C::GBASE + (((wtile + 1) & 1) * C::GROWS + wave * 64) * 4);
    };
    const unsigned sbase = lds0 + C::SBASE + (x_scales ? BN * 4 + wave * 256 : (wave - C::NW + C::WS) * 256);
    auto issue_x = [&](int i) {
        const char* src = half && xkt == nk - 1 && upper ? zeros : xsrc[i];
        glds16(src, lds0 + xdst + (i * C::NW + wave) * 1024);
        xsrc[i] += xinc;
    };
    const long long up = (long long)a.N * a.K;             // from a gate row to its up row
    auto issue_w = [&](int i) {                            // i == WI: the scales
        if (i < WI) {
            // (in a stage of 64 indices the absent pieces are those of the first half again: they meet zeros)
            const unsigned at = woff[i % WV] - (half && wkt == nk - 1 && upper ? 64 : 0);
            glds16_s(wbase + (i / WV) * up, at, lds0 + C::WBASE + wdst + (i * C::NW + wave) * 1024);
        } else {
            if (x_scales || (w_scales && C::WS > 1)) glds4(ssrc, sbase + sdst);
            else if (w_scales) glds16(ssrc, sbase + sdst);
            ssrc += sinc;
            wbase += winc;
        }
    };
    auto advance_x = [&]() {
        xdst = xdst + C::XBYTES == NSX * C::XBYTES ? 0 : xdst + C::XBYTES;
        if (xon && ++xkt == nk) next_x();
    };
    auto advance_w = [&]() {
        wdst = wdst + C::WBYTES == NSW * C::WBYTES ? 0 : wdst + C::WBYTES;
        sdst = sdst + C::SBYTES == NSW * C::SBYTES ? 0 : sdst + C::SBYTES;
        if (won && ++wkt == nk) next_w();
    };
    next_x();
    next_w();
#pragma unroll
    for (int s = 0; s < NSX; s++) {
#pragma unroll
        for (int i = 0; i < XI; i++) issue_x(i);
        advance_x();
    }
#pragma unroll
    for (int s = 0; s < NSW - 1; s++) {
#pragma unroll
        for (int i = 0; i <= WI; i++) issue_w(i);
        advance_w();
    }
    prologue = false;
    wait_vmcnt<0>();
    lds_barrier();

    // ---- fragments --------------------------------------------------------------------------------------------
    // ring places of the stage that is multiplied; lane addresses: a base per ring, the fragment in the instruction's offset
    unsigned xo = 0, wo = 0, so = 0;
    const int p0 = (lg ^ swz(l16)) * 16, p1 = ((4 + lg) ^ swz(l16)) * 16;
    const unsigned lx = (wm * 16 + l16) * C::ROWB, lsx = C::SBASE + (BN + wm * 16 + l16) * 4 + lg;
    const unsigned lw = C::WBASE + (wn * (GATE_UP ? 32 : 64) + l16) * C::ROWB, lsw = C::SBASE + (wn * (GATE_UP ? 32 : 64) + l16) * 4 + lg;
    i32x8 wf[4], xf[3];                                    // fragment m of the rows in registers m mod 3
    int wsb[4], xsb[3];
    auto load_w = [&](int n, unsigned w_at, unsigned s_at) {
        constexpr int kHalf = GATE_UP ? BN / 2 : 32;
        const int r = (n >> 1) * kHalf + (n & 1) * 16;
        wf[n] = two16(*reinterpret_cast<const uint4*>(smem + lw + p0 + w_at + r * C::ROWB), *reinterpret_cast<const uint4*>(smem + lw + p1 + w_at + r * C::ROWB));
        wsb[n] = *reinterpret_cast<const unsigned char*>(smem + lsw + s_at + r * 4);
    };
    auto load_x = [&](int b, int m, unsigned x_at, unsigned s_at) {      // fragment m into registers b
        xf[b] = two16(*reinterpret_cast<const uint4*>(smem + lx + p0 + x_at + m * 32 * C::ROWB),
                      *reinterpret_cast<const uint4*>(smem + lx + p1 + x_at + m * 32 * C::ROWB));
        xsb[b] = *reinterpret_cast<const unsigned char*>(smem + lsx + s_at + m * 32 * 4);
    };
    const bool upper_half = lg >= 2;
#pragma unroll
    for (int n = 0; n < 4; n++) load_w(n, 0, 0);
    load_x(0, 0, 0, 0);
    load_x(1, 1, 0, 0);

    // ---- a stage ------------------------------------------------------------------------------------------
    f32x4 acc[MF][4];
    auto stage = [&](int kt) {
        constexpr int H = 2, M1 = MF - H;                   // fragments of the second and of the first part
        const bool tail = half && kt == nk - 1 && upper_half;
        auto mfma = [&](int m, int n) {
            const int b = m % 3;
            // past the end of K the values are zeros; their scales must not be NaN
            if (m == 0) wsb[n] = tail ? kMxBias : wsb[n];
            if (n == 0) xsb[b] = tail ? kMxBias : xsb[b];
            acc[m][n] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wf[n], xf[b], acc[m][n], 0, 0, 0, wsb[n], 0, xsb[b]);
        };
        // Products stay where they are written: moved behind the meeting or the change of tiles they would keep the fragments of two stages in
        // registers.
        auto keep = [&](int m0, int m1) {
#pragma unroll
            for (int m = m0; m < m1; m++)
#pragma unroll
                for (int n = 0; n < 4; n++) asm volatile("" : "+v"(acc[m][n]));
        };
        // first part
        constexpr int SL = 4 * M1;
        if constexpr (SL == 0) {
#pragma unroll
            for (int u = 0; u <= WI; u++) issue_w(u);
        }
#pragma unroll
        for (int sl = 0; sl < SL; sl++) {
            const int m = sl >> 2, n = sl & 3;
            mfma(m, n);
            if (n == 0) load_x((m + 2) % 3, m + 2, xo, so);
#pragma unroll
            for (int u = 0; u <= WI; u++)
                if (u * SL / (WI + 1) == sl) issue_w(u);
            __builtin_amdgcn_sched_barrier(0);
        }
        keep(0, M1);
        // the loads of the next stage have landed: only what was issued behind them may be outstanding
        constexpr int kBehind = NSX == NSW ? XI + WI : WI;
        if (x_scales || w_scales) wait_vmcnt<kBehind + 1>();
        else wait_vmcnt<kBehind>();
        lds_barrier();
        xo = xo + C::XBYTES == NSX * C::XBYTES ? 0 : xo + C::XBYTES;
        wo = wo + C::WBYTES == NSW * C::WBYTES ? 0 : wo + C::WBYTES;
        so = so + C::SBYTES == NSW * C::SBYTES ? 0 : so + C::SBYTES;
        // second part; registers 0 and 1 take the next stage's rows at once if the last two fragments are not in them
        auto free_early = [](int b) { return b != M1 % 3 && b != (M1 + 1) % 3; };
#pragma unroll
        for (int n = 0; n < 4; n++) {
#pragma unroll
            for (int j = 0; j < H; j++) {
                mfma(M1 + j, n);
                if (n * H + j < XI) issue_x(n * H + j < XI ? n * H + j : 0);
                __builtin_amdgcn_sched_barrier(0);
            }
            load_w(n, wo, so);
            if (n < 2 && free_early(n)) load_x(n, n, xo, so);
            __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int n = 0; n < 2; n++)
            if (!free_early(n)) load_x(n, n, xo, so);
        keep(M1, MF);
    };
    // ---- the tiles ------------------------------------------------------------------------------------------
    for (;;) {
        int ln = lane;
        asm volatile("" : "+v"(ln));
        const TileRef t = next_tile(clist, a, place, BM, ln);
        if (!t.valid) break;
        const int col = t.nt * C::COLS + wn * (GATE_UP ? 32 : 64);       // the wavefront's columns are inside N or outside as a whole
        const int mi = col < a.N ? (((t.rows + 15) >> 4) - wm + 1) >> 1 : 0;
#pragma unroll
        for (int m = 0; m < MF; m++)
#pragma unroll
            for (int n = 0; n < 4; n++) acc[m][n] = f32x4{0.f, 0.f, 0.f, 0.f};
        for (int kt = 0; kt < nk; kt++) {
            stage(kt);
            advance_w();
            advance_x();
        }
        // acc[m][n][i] = C[row 16 (2 m + wm) + l16][weight row 16 n + 4 lg + i of the wavefront's 64]
        asm volatile("" : "+v"(ln));
        const int r16 = ln & 15, rg = ln >> 4;
        if constexpr (GATE_UP) {
            // two fragments at a time: their rows of 32 bytes leave in pieces of 16 a lane, half as many stores and requests as in words
#pragma unroll
            for (int m = 0; m < MF; m += 2) {
                if (m >= mi) break;
                unsigned p[4];
                const int byte0 = block_of_h(acc[m][0], acc[m][1], acc[m][2], acc[m][3], p[0], p[1]);
                int byte1 = 0;
                p[2] = p[3] = 0;
                const int m1 = m + 1 < MF ? m + 1 : m;
                if (m + 1 < mi) byte1 = block_of_h(acc[m1][0], acc[m1][1], acc[m1][2], acc[m1][3], p[2], p[3]);
                const uint4 piece = lane_groups_transposed(p[0], p[1], p[2], p[3]);
                const int r = (2 * m + (rg & 2) + wm) * 16 + r16;
                const long long row = t.row0 + r;
                if (r < t.rows && (m + 1 < mi || rg < 2)) {
                    *reinterpret_cast<uint4*>(a.h + row * a.N + col + (rg & 1) * 16) = piece;
                    if ((rg & 1) == 0) store_h_scale(a, row, col, rg == 0 ? byte0 : byte1);
                }
            }
        } else {
#pragma unroll
            for (int m = 0; m < MF; m++) {
                if (m >= mi) break;
                const int r = (2 * m + wm) * 16 + r16;
                // 64 bytes of a row a store
#pragma unroll
                for (int n = 0; n < 4; n += 2) {
                    const uint2 u = pack4(acc[m][n][0], acc[m][n][1], acc[m][n][2], acc[m][n][3]);
                    const uint2 v = pack4(acc[m][n + 1][0], acc[m][n + 1][1], acc[m][n + 1][2], acc[m][n + 1][3]);
                    uint4 piece;
                    pair_lane_groups(u.x, v.x, piece.x, piece.z);
                    pair_lane_groups(u.y, v.y, piece.y, piece.w);
                    if (r < t.rows) *reinterpret_cast<uint4*>(a.y + (long long)(t.row0 + r) * a.N + col + n * 16 + 8 * rg) = piece;
                }
            }
        }
    }
    wait_vmcnt<0>();                                       // no load may land in LDS that is someone else's by then
}

// Scales of the gathered rows in group order: a tile's then lie in a few lines, where those of tokens are a line each, fetched
// again for every tile of columns.  Rows outside the offsets have no token: their entries of gather may hold anything and are not read.
__global__ __launch_bounds__(256) void gather_scales_kernel(const unsigned* __restrict__ in, long long T, const int32_t* __restrict__ gather, int gather_div,
                                                            const int32_t* __restrict__ offsets, int E, unsigned* __restrict__ out, long long S, int words) {
    const long long r = (long long)blockIdx.x * 256 + threadIdx.x;
    if (r >= S || r < offsets[0] || r >= offsets[E]) return;
    const int t = gather[r] / gather_div;
#pragma unroll 4
    for (int w = 0; w < words; w++) out[w * S + r] = in[w * T + t];
}

template <bool GATE_UP, int BM, int BN, int NSX, int NSW> hipError_t run_tile(Mx8Args a, hipStream_t st) {
    using C = Mx8Tile<GATE_UP, BM, BN, NSX, NSW>;
    auto kern = ffn_mx8_kernel<GATE_UP, BM, BN, NSX, NSW>;
    static bool attr_set = false;
    if (!attr_set) {
        hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, C::LDS);
        if (e != hipSuccess) return e;
        attr_set = true;
    }
    a.g.group_m = BM > 128 ? 2 : 1;
    a.g.n_tiles_n = cdiv(a.N, C::COLS);
    kern<<<max(kNumXcd, num_cus() / kNumXcd * kNumXcd) * C::WG, 64 * C::NW, C::LDS, st>>>(a);
    return hipGetLastError();
}

// Which form a call takes, from the rows r of an expert that has any (as if the picks were independent) and from how many rounds its
// gate-up tiles of 128 rows by 256 weight rows are on the card's compute units.  All of the call, us, three sets of weights in turn:
//   few: up to 64 tokens, with few tasks (64 experts of 768 x 2048, k = 2, 1 token: few 14.5, tiles of 64 x 128 21.8, 4 tokens 18.6 / 23.4; but 5
//     tokens of 90 experts of 832 x 1472, k = 3 25.0 / 25.0, 40 tokens 77 / 68), or where the reductions are long (192 experts of 1536 x
//     4096, k = 2, 4 tokens 41 / 52, 64 tokens 342 / 358; up to three rows an expert also the 64 experts, 16 tokens 38 / 41, 32 tokens
//     50 / 53, but 16 experts of 768 x 2048, 64 tokens, k = 1 29.4 / 27.2);
//   128 weight rows, two workgroups to a compute unit, while there are less than 16 rounds of the wide ones, or 4 with more than 96
//     rows (64 x 128 / 96 x 128 / 64 x 256 / 128 x 256: 90 experts, 50 rows, hot 108 / 106 / 115 / 112; 16 experts of 768 x 2048, 37 rows 28.0 /
//     29.2 / 31.3 / 35.4, 187 rows 49 / 44 / 50 / 46);
//   256 weight rows beyond (192 experts of 1536 x 4096, 11 rows 716 / 729 / 653 / 691, 42 rows 759 / 760 / 712 / 734, 85 rows 1087 / 906 / 1007 / 789);
//   192 rows where experts take several tiles of 128 (the 192 experts, 125 rows: 128 x 256 939, 192 x 256 869; 512 of 1024 x 704, 256 rows 582 / 567).
// The pools named here are all that was measured; between their widths (few rows: 832 to 1536 in the shorter dimension) the lines are drawn, not found.
enum Mx8Form { MX8_FEW, MX8_64x128, MX8_96x128, MX8_64x256, MX8_128x256, MX8_192x256 };
Mx8Form mx8_form(const unipool_shape& s) {
    const double S = (double)s.T * s.k, used = s.E * -std::expm1(-S / s.E), r = S / used, most = r + 2.0 * std::sqrt(r);
    const int cus = num_cus();
    if (s.T <= 16 || (s.T <= 64 && S <= 8.0 * s.E)) {
        const double tasks = std::min(S, (double)s.E) * (s.d_ff / 32);
        const int least = std::min(s.d_model, s.d_ff);
        if (tasks <= 2.0 * cus || least >= 1536 || (least >= 768 && s.d_ff >= 2048 && S <= 3.0 * s.E)) return MX8_FEW;
    }
    const double rounds = used * std::ceil((r + std::sqrt(r)) / 128) * cdiv(s.d_ff, 128) / cus;
    if (r > 96) return rounds < 4 ? MX8_96x128 : most <= 128 ? MX8_128x256 : MX8_192x256;
    if (rounds < 16) return most <= 64 ? MX8_64x128 : MX8_96x128;
    return most <= 32 ? MX8_64x256 : MX8_128x256;
}

template <bool GATE_UP> hipError_t run_mx8(Mx8Form form, const Mx8Args& a, hipStream_t st) {
    switch (form) {
        case MX8_64x128: return run_tile<GATE_UP, 64, 128, 3, 3>(a, st);
        case MX8_96x128: return run_tile<GATE_UP, 96, 128, 2, 3>(a, st);
        case MX8_64x256: return run_tile<GATE_UP, 64, 256, 3, 3>(a, st);
        case MX8_128x256: return run_tile<GATE_UP, 128, 256, 3, 3>(a, st);
        default: return run_tile<GATE_UP, 192, 256, 2, 3>(a, st);
    }
}

// ---------------------------------------------------------------------------------------------
// Few rows per expert (decoding, short prompts): one pass over the weights of the experts that have rows, bound by the bytes that are
// in flight.  A wavefront owns 16 NF weight rows of one expert (gate-up: 32 gate rows and the 32 up rows they meet, which are a whole
// block of H) for all rows of the expert; weights go from memory to registers, whole 128-byte lines at a time (few_rows.h), D
// steps of 128 indices ahead, with no LDS and no barrier.  192 experts of 1536 x 4096, 4 tokens: 20.1 us for 104 MB (5.2 TB/s), 13.4 us
// for 52 MB (at the rate of a large copy 20.5 and 10.3; the weights lie in the last-level cache here, else 40.4 for both).
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
    int row[R];
#pragma unroll
    for (int r = 0; r < R; r++) {
        row[r] = row0 + min(16 * r + l16, rows - 1);
        if (a.gather != nullptr) row[r] = a.gather[row[r]];
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
    int next_w = 0, next_x = 0;
    auto fetch_w = [&](int u) {
        const bool last = next_w == nk - 1;
        unsigned o = half && last ? wo_cut : wo, so = wso;
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
        next_w += last ? 0 : 1;
        wk += last ? 0 : kMxStep;
        wsk += last ? 0 : w_plane;
    };
    auto fetch_x = [&](int u) {
        const bool last = next_x == nk - 1;
#pragma unroll
        for (int r = 0; r < R; r++) {
            unsigned q = xo[r], p = xso[r];
            asm volatile("" : "+v"(q), "+v"(p));
            xq[u][r][0] = *reinterpret_cast<const u32x4v*>(xk + q);
            xq[u][r][1] = *reinterpret_cast<const u32x4v*>(xk + (half && last ? 0 : 64) + q);
            xs[u][r] = xsk[p];
        }
        next_x += last ? 0 : 1;
        xk += last ? 0 : kMxStep;
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
    // the weights first: which rows meet them is still being looked up
#pragma unroll
    for (int u = 0; u < D; u++) fetch_w(u);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int r = 0; r < R; r++) {
        if (a.gather != nullptr) row[r] /= a.gather_div;
        xo[r] = (unsigned)row[r] * (unsigned)a.K + 16 * lg;
        xso[r] = (unsigned)row[r] * 4 + lg;
    }
#pragma unroll
    for (int u = 0; u < D; u++) fetch_x(u);
    int s = 0;
    for (; s + D < nk; s += D) {
#pragma unroll
        for (int u = 0; u < D; u++) {
            multiply(u, false);
            fetch_w(u);
            fetch_x(u);
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
    // At most one wavefront per SIMD.  More steps in flight than these would fit its registers, but every step is code of its own that has to
    // come from memory too (6 and 16 steps: 192 experts of 1536 x 4096, k = 2, 1 token 22.6 us instead of 19.9, 4 tokens 44.0 instead of 40.4; 32
    // of 512 x 512, 8 tokens 17.5 instead of 14.4; 4 and 12 steps: 21.8, 42.7, 15.1; 3 and 4: 21.2, 40.3, 13.1).
    if (most <= 4 * cus) {
        constexpr int D1 = GATE_UP ? 3 : 8, DM = GATE_UP ? 2 : 4;
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

}  // namespace

int mx8_ffn_form(const unipool_shape& s) {
    constexpr int kForms[] = {0, 64128, 96128, 64256, 128256, 192256};
    return kForms[mx8_form(s)];
}

hipError_t mx8_ffn_fwd(const unipool_shape& s, const void* x, const void* x_scale, const int32_t* slot_of_row, const int32_t* offsets,
                       const void* wgu, const void* wgu_scale, const void* wd, const void* wd_scale, void* h, void* h_scale, void* y,
                       void* scratch, size_t scratch_bytes, hipStream_t st) {
    const Mx8Form form = mx8_form(s);
    const bool few = form == MX8_FEW;
    const long long S = (long long)s.T * s.k;
    // A launch for the scales of gathered rows (7 us) where every one would be fetched for 32 tiles of columns or more, 3 million words and
    // over in all (192 experts of 1536 x 4096, k = 2, 4001 tokens 734 -> 726 us, 8192 787 -> 773, 32768 1570 -> 1548; but 64 experts of
    // 768 x 2048, k = 8, 16384 tokens, 16 tiles of columns, 809 / 809, and 512 of 1024 x 704, k = 8, 16384 tokens 568 / 576).
    const int words = cdiv(s.d_model, kMxStep), tiles = cdiv(s.d_ff, 128);
    const bool scales_first = slot_of_row && !few && tiles >= 32 && (double)S * words * tiles >= 3e6 && (size_t)S * words * 4 <= scratch_bytes;
    if (scales_first)
        gather_scales_kernel<<<(unsigned)((S + 255) / 256), 256, 0, st>>>((const unsigned*)x_scale, s.T, slot_of_row, s.k, offsets, s.E,
                                                                          (unsigned*)scratch, S, words);
    Mx8Args a = {};
    a.offsets = offsets;
    a.x = (const unsigned char*)x; a.x_scale = (const unsigned char*)(scales_first ? scratch : x_scale);
    a.scales_too = slot_of_row && !scales_first;
    a.x_rows = a.scales_too ? s.T : S;
    a.gather = slot_of_row; a.gather_div = s.k;
    a.w = (const unsigned char*)wgu; a.w_scale = (const unsigned char*)wgu_scale;
    a.w_rows = 2 * s.d_ff; a.E = s.E;
    a.K = s.d_model; a.N = s.d_ff;
    a.h = (unsigned char*)h; a.h_scale = (unsigned char*)h_scale; a.S = S;
    hipError_t e = few ? run_few_mx8<true>(s, a, st) : run_mx8<true>(form, a, st);
    if (e != hipSuccess) return e;
    Mx8Args b = {};
    b.offsets = offsets;
    b.x = (const unsigned char*)h; b.x_scale = (const unsigned char*)h_scale;
    b.x_rows = S;
    b.w = (const unsigned char*)wd; b.w_scale = (const unsigned char*)wd_scale;
    b.w_rows = s.d_model; b.E = s.E;
    b.K = s.d_ff; b.N = s.d_model;
    b.y = (bf16*)y; b.S = S;
    return few ? run_few_mx8<false>(s, b, st) : run_mx8<false>(form, b, st);
}

}  // namespace unipool
