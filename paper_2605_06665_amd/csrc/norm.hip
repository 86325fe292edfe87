// Root-mean-square norm of the rows in front of a layer, with the residual's addition, and its backward pass.
//
//   h = x + r;  s = 1 / sqrt(mean(h^2) + eps);  y = h s w
//   g = w dy;   dx = s g - h s^3 mean(g h) + dh;   dw = sum over the rows of dy h s
// (h s is of order one and is formed first: s^3 alone would pass the largest float where rows are of order 1e-13 and eps is 0)
//
// Both passes are bound by memory: a row is read once, held in registers as it came, and every output leaves from there.  A
// value takes a handful of operations, all in float; h is rounded only where it is stored, and y, in 16 or in 8 bits, is made
// from the unrounded sum.  32768 rows of 1536 in bfloat16: forward 73 us (403 MB, 5.5 TB/s), backward 84 us (4.8 TB/s) and 4.8 us
// for the sum of d_weight; 4001 rows with 16-bit and 8-bit output 10.6 us (55 MB); 1001 float rows of 252 3.1, 4.3 and 2.2 us.
#include <algorithm>
#include <initializer_list>

#include "mx8.h"

namespace unipool {

namespace {

// N neighbouring values as they lie in memory
template <typename TA, int N> struct Pack { typedef __attribute__((ext_vector_type(N * sizeof(TA) / 4))) unsigned type; };
template <> struct Pack<float, 1> { typedef float type; };
template <> struct Pack<bf16, 1> { typedef bf16 type; };

template <typename TA, int N> __device__ __forceinline__ void unpack(const typename Pack<TA, N>::type& p, float (&v)[N]) {
    union { typename Pack<TA, N>::type p; TA e[N]; } u;
    u.p = p;
#pragma unroll
    for (int i = 0; i < N; i++) v[i] = to_f32(u.e[i]);
}
template <typename TA, int N> __device__ __forceinline__ typename Pack<TA, N>::type pack(const float (&v)[N]) {
    union { typename Pack<TA, N>::type p; TA e[N]; } u;
#pragma unroll
    for (int i = 0; i < N; i++) u.e[i] = from_f32<TA>(v[i]);
    return u.p;
}

// Sum over the W wavefronts that share a row, the same bits in all of them.  red: W floats of LDS that nobody reads any more.
template <int W> __device__ __forceinline__ float row_sum(float v, float* red) {
    v = wave_sum(v);
    if constexpr (W > 1) {
        const int wave = threadIdx.x >> 6;
        if ((threadIdx.x & 63) == 0) red[wave] = v;
        __syncthreads();
        v = 0.f;
#pragma unroll
        for (int w = 0; w < W; w++) v += red[w];
    }
    return v;
}

// 8-bit outputs of one chunk of N values: the LPB lanes that hold a block agree on its scale.
template <int N>
__device__ __forceinline__ void store_mx8(const float (&y)[N], bool on, size_t rows, size_t row, int d, int col, unsigned char* q,
                                          unsigned char* scale) {
    constexpr int LPB = kMxBlock / N;
    float m = y[0];
#pragma unroll
    for (int i = 1; i < N; i++) m = mx8_max(m, y[i]);
    m = mx8_lanes_max<LPB>(m);
    if (!on) return;
    const int byte = mx8_scale_byte(m);
    unsigned char* dst = q + row * d + col;
    if constexpr (N == 8) {
        uint2 w;
        w.x = mx8_pack4(y[0], y[1], y[2], y[3], byte);
        w.y = mx8_pack4(y[4], y[5], y[6], y[7], byte);
        *reinterpret_cast<uint2*>(dst) = w;
    } else if constexpr (N == 4) {
        *reinterpret_cast<unsigned*>(dst) = mx8_pack4(y[0], y[1], y[2], y[3], byte);
    } else {
        dst[0] = mx8_pack1(y[0], byte);
    }
    if ((threadIdx.x & (LPB - 1)) == 0) scale[mx8_scale_at(rows, row, col / kMxBlock)] = (unsigned char)byte;
}

struct NormArgs {
    const void *x, *residual, *weight;
    void *h, *y;
    unsigned char *q, *scale;
    int T, d;
    float eps;
    int row0;                 // first row of the launch
};

// W wavefronts share a row and hold it in R chunks of N values a lane.  h and y may lie in the place of x or of the residual: a lane has
// read all of its chunks before it writes the first, and no lane reads another's.
template <typename TA, int N, int W, int R>
__global__ __launch_bounds__(W == 1 ? 256 : 64 * W) void rmsnorm_kernel(const NormArgs a) {
    typedef typename Pack<TA, N>::type P;
    constexpr int kRows = W == 1 ? 4 : 1;                  // rows of a workgroup
    __shared__ float red[W];
    const int lane = W == 1 ? threadIdx.x & 63 : threadIdx.x;
    const size_t row = a.row0 + (size_t)blockIdx.x * kRows + (W == 1 ? threadIdx.x >> 6 : 0);
    if (row >= (size_t)a.T) return;
    const int d = a.d;
    const size_t o = row * d;
    const TA* x = (const TA*)a.x + o;
    const TA* r = a.residual ? (const TA*)a.residual + o : nullptr;
    const TA* w = (const TA*)a.weight;
    TA* h = a.h ? (TA*)a.h + o : nullptr;
    TA* y = a.y ? (TA*)a.y + o : nullptr;
    constexpr int STEP = 64 * W * N;
    float v[R][N];
    P wp[R];                                               // requested with the row, or a second latency would follow the sum
    float ss = 0.f;
#pragma unroll
    for (int i = 0; i < R; i++) wp[i] = i * STEP + lane * N < d ? *reinterpret_cast<const P*>(w + i * STEP + lane * N) : P{};
    auto fetch = [&](int col, float (&s)[N]) {
#pragma unroll
        for (int i = 0; i < N; i++) s[i] = 0.f;
        if (col < d) {
            unpack<TA, N>(*reinterpret_cast<const P*>(x + col), s);
            if (r != nullptr) {
                float t[N];
                unpack<TA, N>(*reinterpret_cast<const P*>(r + col), t);
#pragma unroll
                for (int i = 0; i < N; i++) s[i] += t[i];
            }
        }
    };
    auto finish = [&](int col, const float (&s)[N], const P& wv, float rs) {
        const bool on = col < d;
        float out[N];
        unpack<TA, N>(wv, out);
        if (on && h != nullptr) *reinterpret_cast<P*>(h + col) = pack<TA, N>(s);
#pragma unroll
        for (int i = 0; i < N; i++) out[i] = on ? s[i] * rs * out[i] : 0.f;
        if (on && y != nullptr) *reinterpret_cast<P*>(y + col) = pack<TA, N>(out);
        if (a.q != nullptr) store_mx8<N>(out, on, a.T, row, d, col, a.q, a.scale);
    };
#pragma unroll
    for (int i = 0; i < R; i++) fetch(i * STEP + lane * N, v[i]);
#pragma unroll
    for (int i = 0; i < R; i++)
#pragma unroll
        for (int j = 0; j < N; j++) ss += v[i][j] * v[i][j];
    ss = row_sum<W>(ss, red);
    const float rs = 1.0f / sqrtf(ss / (float)d + a.eps);
#pragma unroll
    for (int i = 0; i < R; i++) finish(i * STEP + lane * N, v[i], wp[i], rs);
    if (a.q != nullptr) {
        const int b = d / kMxBlock + lane;                  // blocks that fill the last word of scales
        if (b < cdiv(d, kMxStep) * 4) a.scale[mx8_scale_at(a.T, row, b)] = kMxBias;
    }
}

struct NormBwdArgs {
    const void *h, *weight, *dy, *dh;
    void* dx;
    float* part;              // [workgroups][d] partial sums of d_weight
    int T, d;
    float eps;
};

// As above; W == 1: eight rows a workgroup, since fewer partial sums of d_weight are written and read again (32768 rows of 1536: four
// 89 us, eight 84).  A workgroup takes the rows blockIdx.x, blockIdx.x + gridDim.x, ... and holds its share of d_weight in
// registers.
constexpr int kBwdRows = 8;
template <typename TA, int N, int W, int R>
__global__ __launch_bounds__(W == 1 ? 64 * kBwdRows : 64 * W) void rmsnorm_bwd_kernel(const NormBwdArgs a) {
    typedef typename Pack<TA, N>::type P;
    constexpr int kRows = W == 1 ? kBwdRows : 1;
    constexpr int STEP = 64 * W * N;
    __shared__ float red[2][W];
    __shared__ float sums[W == 1 ? STEP * R : 1];
    const int lane = W == 1 ? threadIdx.x & 63 : threadIdx.x;
    const int wave = W == 1 ? threadIdx.x >> 6 : 0;
    const int d = a.d;
    const TA* w = (const TA*)a.weight;
    float dw[R][N];
    P wp[R];
#pragma unroll
    for (int i = 0; i < R; i++) {
        const int c = i * STEP + lane * N;
        wp[i] = c < d ? *reinterpret_cast<const P*>(w + c) : P{};
#pragma unroll
        for (int j = 0; j < N; j++) dw[i][j] = 0.f;
    }
    for (size_t row = (size_t)blockIdx.x * kRows + wave; row < (size_t)a.T; row += (size_t)gridDim.x * kRows) {
        const size_t o = row * d;
        P hp[R], gp[R], ep[R];
#pragma unroll
        for (int i = 0; i < R; i++) {
            const int c = i * STEP + lane * N;
            const bool on = c < d;
            hp[i] = on ? *reinterpret_cast<const P*>((const TA*)a.h + o + c) : P{};
            gp[i] = on ? *reinterpret_cast<const P*>((const TA*)a.dy + o + c) : P{};
            if (a.dh != nullptr) ep[i] = on ? *reinterpret_cast<const P*>((const TA*)a.dh + o + c) : P{};
        }
        float ss = 0.f, sg = 0.f;
#pragma unroll
        for (int i = 0; i < R; i++) {
            float h[N], g[N], q[N];
            unpack<TA, N>(hp[i], h);
            unpack<TA, N>(gp[i], g);
            unpack<TA, N>(wp[i], q);
#pragma unroll
            for (int j = 0; j < N; j++) {
                ss += h[j] * h[j];
                sg += (q[j] * g[j]) * h[j];
            }
        }
        if constexpr (W > 1) __syncthreads();               // the sums of the row before have been read
        ss = row_sum<W>(ss, red[0]);
        sg = row_sum<W>(sg, red[1]);
        const float rs = 1.0f / sqrtf(ss / (float)d + a.eps);
        const float back = rs * (rs * (sg / (float)d));
#pragma unroll
        for (int i = 0; i < R; i++) {
            const int c = i * STEP + lane * N;
            float h[N], g[N], q[N], e[N];
            // (1024 threads have 128 registers each, so there a row is unpacked again: kept as floats from the sums on it would pass them; 4096
            // rows of 16384 in bfloat16, forward and backward, 263 us with the spills, 225)
            if constexpr (W == 16 && sizeof(P) == 16) asm volatile("" : "+v"(hp[i]), "+v"(gp[i]), "+v"(wp[i]));
            unpack<TA, N>(hp[i], h);
            unpack<TA, N>(gp[i], g);
            unpack<TA, N>(wp[i], q);
            if (a.dh != nullptr) unpack<TA, N>(ep[i], e);
#pragma unroll
            for (int j = 0; j < N; j++) {
                const float hs = h[j] * rs;
                float v = rs * (q[j] * g[j]) - hs * back;
                if (a.dh != nullptr) v += e[j];
                dw[i][j] += g[j] * hs;
                q[j] = v;
            }
            if (c < d) *reinterpret_cast<P*>((TA*)a.dx + o + c) = pack<TA, N>(q);
        }
    }
    float* part = a.part + (size_t)blockIdx.x * d;
    if constexpr (W == 1) {
        // the wavefronts one after the other, so that the sum has one order
        for (int v = 0; v < kBwdRows; v++) {
            if (wave == v) {
#pragma unroll
                for (int i = 0; i < R; i++)
#pragma unroll
                    for (int j = 0; j < N; j++) {
                        float* p = &sums[i * STEP + j * 64 + lane];
                        *p = v == 0 ? dw[i][j] : *p + dw[i][j];
                    }
            }
            __syncthreads();
        }
        for (int c = threadIdx.x; c < d; c += 64 * kBwdRows) part[c] = sums[c / STEP * STEP + (c % N) * 64 + c % STEP / N];
    } else {
#pragma unroll
        for (int i = 0; i < R; i++)
#pragma unroll
            for (int j = 0; j < N; j++) {
                const int c = i * STEP + lane * N + j;
                if (c < d) part[c] = dw[i][j];
            }
    }
}

// d_weight from the partial sums of the workgroups: a workgroup of 1024 threads adds up 64 columns, 16 threads to a column, their
// shares in a fixed order.
__global__ __launch_bounds__(1024) void rmsnorm_dweight_kernel(const float* __restrict__ part, int nparts, int d, float* __restrict__ d_weight) {
    __shared__ float red[16][64];
    const int lane = threadIdx.x & 63, g = threadIdx.x >> 6;
    const int c = blockIdx.x * 64 + lane, cc = min(c, d - 1);
    float v = 0.f;
    for (int p = g; p < nparts; p += 8 * 16) {
        float q[8];
#pragma unroll
        for (int u = 0; u < 8; u++) q[u] = part[(size_t)min(p + u * 16, nparts - 1) * d + cc];
#pragma unroll
        for (int u = 0; u < 8; u++)
            if (p + u * 16 < nparts) v += q[u];
    }
    red[g][lane] = v;
    __syncthreads();
    if (g == 0 && c < d) {
        for (int i = 1; i < 16; i++) v += red[i][lane];
        d_weight[c] = v;
    }
}

template <int V> using Int = std::integral_constant<int, V>;
// 16-byte chunks of bfloat16, of float, and single values (addresses or widths that are no multiple of a chunk).  A row belongs to one
// wavefront as long as its chunks fit the registers, then to four, then to sixteen (forward and backward: 32768 rows of 1536 in
// bfloat16 by one 161 us, by four 180; 8192 rows of 4096 by one 241, by two 118, by four 99; 8192 float rows of 2048 107, 103, 90).
template <class F> void with_form_8(int d, F f) {
    if (d <= 512) f(Int<8>{}, Int<1>{}, Int<1>{});
    else if (d <= 1024) f(Int<8>{}, Int<1>{}, Int<2>{});
    else if (d <= 1536) f(Int<8>{}, Int<1>{}, Int<3>{});
    else if (d <= 2048) f(Int<8>{}, Int<1>{}, Int<4>{});
    else if (d <= 4096) f(Int<8>{}, Int<4>{}, Int<2>{});
    else if (d <= 8192) f(Int<8>{}, Int<4>{}, Int<4>{});
    else f(Int<8>{}, Int<16>{}, Int<2>{});
}
template <class F> void with_form_4(int d, F f) {
    if (d <= 256) f(Int<4>{}, Int<1>{}, Int<1>{});
    else if (d <= 512) f(Int<4>{}, Int<1>{}, Int<2>{});
    else if (d <= 1024) f(Int<4>{}, Int<1>{}, Int<4>{});
    else if (d <= 2048) f(Int<4>{}, Int<4>{}, Int<2>{});
    else if (d <= 4096) f(Int<4>{}, Int<4>{}, Int<4>{});
    else f(Int<4>{}, Int<16>{}, Int<4>{});
}
template <class F> void with_form_1(int d, F f) {
    if (d <= 256) f(Int<1>{}, Int<1>{}, Int<4>{});
    else if (d <= 1024) f(Int<1>{}, Int<4>{}, Int<4>{});
    else if (d <= 4096) f(Int<1>{}, Int<16>{}, Int<4>{});
    else f(Int<1>{}, Int<16>{}, Int<16>{});
}
static_assert(kNormMaxD == 16384, "the longest forms above hold it");
template <typename TA, class F> void with_norm_form(int d, bool wide, F f) {
    if (!wide) with_form_1(d, f);
    else if constexpr (sizeof(TA) == 2) with_form_8(d, f);
    else with_form_4(d, f);
}

bool aligned16(std::initializer_list<const void*> ps) {
    for (const void* p : ps)
        if (((uintptr_t)p & 15) != 0) return false;
    return true;
}

template <typename TA>
hipError_t run_norm(NormArgs a, hipStream_t st) {
    constexpr int n = 16 / sizeof(TA), kRowsPerLaunch = 1 << 21;      // a launch has less than 2^32 threads, and a row up to 1024
    const int T = a.T;
    const bool wide = a.d % n == 0 && aligned16({a.x, a.residual, a.weight, a.h, a.y}) && ((uintptr_t)a.q & 7) == 0;
    with_norm_form<TA>(a.d, wide, [&](auto nn, auto w, auto r) {
        for (long long row0 = 0; row0 < T; row0 += kRowsPerLaunch) {
            const int rows = (int)std::min<long long>(T - row0, kRowsPerLaunch);
            a.row0 = (int)row0;
            rmsnorm_kernel<TA, nn(), w(), r()><<<w() == 1 ? cdiv(rows, 4) : rows, w() == 1 ? 256 : 64 * w(), 0, st>>>(a);
        }
    });
    return hipGetLastError();
}

template <typename TA>
hipError_t run_norm_bwd(NormBwdArgs a, float* d_weight, float* part, hipStream_t st) {
    constexpr int n = 16 / sizeof(TA);
    const bool wide = a.d % n == 0 && aligned16({a.h, a.weight, a.dy, a.dh, a.dx});
    int grid = 1;
    with_norm_form<TA>(a.d, wide, [&](auto nn, auto w, auto r) {
        grid = std::min(kNormParts, w() == 1 ? (a.T - 1) / kBwdRows + 1 : a.T);      // (T + 7 may pass 2^31)
        a.part = grid == 1 ? d_weight : part;
        rmsnorm_bwd_kernel<TA, nn(), w(), r()><<<grid, w() == 1 ? 64 * kBwdRows : 64 * w(), 0, st>>>(a);
    });
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || grid == 1) return e;
    rmsnorm_dweight_kernel<<<cdiv(a.d, 64), 1024, 0, st>>>(part, grid, a.d, d_weight);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_rmsnorm(const unipool_shape& s, const void* x, const void* residual, const void* weight, float eps, void* h,
                          void* y, void* y_q, void* y_scale, hipStream_t st) {
    const NormArgs a = {x, residual, weight, h, y, (unsigned char*)y_q, (unsigned char*)y_scale, s.T, s.d_model, eps, 0};
    return s.dtype == UNIPOOL_BF16 ? run_norm<bf16>(a, st) : run_norm<float>(a, st);
}

hipError_t launch_rmsnorm_bwd(const unipool_shape& s, const void* h, const void* weight, const void* dy, const void* dh, float eps,
                              void* dx, float* d_weight, float* part, hipStream_t st) {
    const NormBwdArgs a = {h, weight, dy, dh, dx, nullptr, s.T, s.d_model, eps};
    return s.dtype == UNIPOOL_BF16 ? run_norm_bwd<bf16>(a, d_weight, part, st) : run_norm_bwd<float>(a, d_weight, part, st);
}

}  // namespace unipool
