// Balance loss of one layer over the sequences of a batch, with the gradient of its logits and its sigma.
//
// Sequence b holds the tokens [o_b, o_{b+1}), T_b of them; n_{b,i} of its picks went to expert i.  With
//   f_{b,i} = E n_{b,i} / (k T_b),   P_{b,i} = mean over the sequence of the score s_{t,i},
//   loss = alpha / B' sum_b sum_i f_{b,i} P_{b,i}        (B': sequences that have tokens; f is constant for differentiation)
// the gradient of a score is coef_{b,i} = alpha f_{b,i} / (B' T_b), the same for all tokens of a sequence, and the loss is the sum of
// <coef, s_t> over the tokens.  coef follows from the picks alone, so the picks are counted first and ONE pass over the logits
// then gives loss and gradient.  The score is linear in sigma: d loss / d sigma = loss / sigma (softmax: 0).
//
// Bound by memory and by what a token costs in instructions and latency: 4 bytes in and 4 out per logit.  16384 tokens of 512
// experts, k = 8, 37 sequences, softmax: counts 4.9 us, loss and gradient 19 to 20 us (67 MB, 3.4 TB/s;
// without the gradient's stores 4.8 us less, without the sum over the workgroups 2 less, without the search for the sequence 1 less).
// A sequence is counted in parts by the average length, as lengths are known on the device only: one that is much longer than the others
// keeps few workgroups busy while the rest of the card waits (131072 tokens of 512 experts, k = 8: 33 even sequences 125 us, 32 of
// 32 tokens beside a long one 355, the long one alone 130).
#include <algorithm>

#include "gemm_common.h"
#include "route_select.h"
#include "kernels.h"

namespace unipool {

namespace {

constexpr int kTokensPerPart = 4096;      // tokens that one workgroup counts where the sequences are as long as their average or shorter
constexpr int kCountThreads = 512;
constexpr int kLossThreads = 1024;
constexpr int kLossTokens = 64;           // tokens of a workgroup, a multiple of that from kLossBlocks workgroups on
constexpr int kLossBlocks = 512;
constexpr int kOneTokens = 256, kOneCounts = 8192;      // what a single workgroup does by itself

struct SeqArgs {
    const int32_t* offsets;               // [n_seq + 1]
    const float* logits;
    const int32_t* topk_idx;
    int32_t* counts;                      // [n_seq][E]
    int32_t* part;                        // [parts][n_seq][E] where sequences are counted in parts
    int32_t* state;                       // [0] sequences with tokens, [1] workgroups that have added their share
    float* loss_part;
    float *loss, *d_logits, *d_sigma;
    int T, E, k, n_seq, parts;
    float alpha, sigma, c, eps;
    int softmax, tok_per_block;
};

// Bounds of a sequence, inside [0, T] whatever the offsets say.
__device__ __forceinline__ void seq_range(const SeqArgs& a, int b, int& t0, int& t1) {
    t0 = min(max(a.offsets[b], 0), a.T);
    t1 = min(max(a.offsets[b + 1], t0), a.T);
}

// Picks per expert of part blockIdx.y of sequence blockIdx.x.  A thread requests eight picks at a time.
__global__ __launch_bounds__(kCountThreads) void seq_count_kernel(const SeqArgs a) {
    __shared__ int hist[kMaxE];
    __shared__ int used[kCountThreads / 64];
    const int b = blockIdx.x, p = blockIdx.y;
    for (int i = threadIdx.x; i < a.E; i += kCountThreads) hist[i] = 0;
    int t0, t1;
    seq_range(a, b, t0, t1);
    const int per = (int)(((long long)(t1 - t0) + a.parts - 1) / a.parts);
    const long long s0 = (long long)min(t0 + (long long)p * per, (long long)t1) * a.k, s1 = (long long)min(t0 + (long long)(p + 1) * per, (long long)t1) * a.k;
    __syncthreads();
    for (long long s = s0 + threadIdx.x; s < s1; s += 8 * kCountThreads) {
        int e[8];
#pragma unroll
        for (int u = 0; u < 8; u++) e[u] = s + u * kCountThreads < s1 ? a.topk_idx[s + u * kCountThreads] : -1;
#pragma unroll
        for (int u = 0; u < 8; u++)
            if (e[u] >= 0 && e[u] < a.E) atomicAdd(&hist[e[u]], 1);
    }
    __syncthreads();
    int32_t* out = (a.parts > 1 ? a.part + (size_t)p * a.n_seq * a.E : a.counts) + (size_t)b * a.E;
    for (int i = threadIdx.x; i < a.E; i += kCountThreads) out[i] = hist[i];
    if (b == 0 && p == 0) {
        int n = 0;
        for (int i = threadIdx.x; i < a.n_seq; i += kCountThreads) {
            int r0, r1;
            seq_range(a, i, r0, r1);
            n += r1 > r0;
        }
        n = wave_sum_i(n);
        if ((threadIdx.x & 63) == 0) used[threadIdx.x >> 6] = n;
        __syncthreads();
        if (threadIdx.x == 0) {
            int all = 0;
            for (int w = 0; w < kCountThreads / 64; w++) all += used[w];
            a.state[0] = all;
            a.state[1] = 0;
        }
    }
}

__global__ __launch_bounds__(256) void seq_count_sum_kernel(const SeqArgs a) {
    const size_t n = (size_t)a.n_seq * a.E, i = (size_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= n) return;
    int v = 0;
    for (int p = 0; p < a.parts; p++) v += a.part[p * n + i];
    a.counts[i] = v;
}

// The sequence that holds token t, or else the next one that ends behind it: the first b with offsets[b + 1] > t, n_seq if there is
// none.  By a wavefront, 64 places at a time.
__device__ __forceinline__ int find_sequence(const SeqArgs& a, int t, int lane) {
    int lo = 0, hi = a.n_seq;                         // the answer lies in [lo, hi]
    while (lo < hi) {
        const int step = (hi - lo + 63) >> 6;
        const int at = lo + (lane + 1) * step - 1;    // last place of the lane's part
        const unsigned long long over = __ballot(at >= hi || a.offsets[min(at, hi - 1) + 1] > t);
        const int first = over ? __builtin_ctzll(over) : 64;
        const int from = lo + first * step;
        if (from >= hi) return hi;                     // every part that there is ends at or before t
        hi = min(hi, from + step - 1);                 // (its last place is an answer)
        lo = from;
    }
    return lo;
}

// GS lanes to a token, VPL logits to a lane: lane s holds logits s + GS i, or with V4 groups of four neighbours.  The logits of the
// next round of tokens are requested before this one's are worked on, and the first ones before the sequence is looked up.
// ONE: a single workgroup counts the picks too, in LDS, and needs no other's share.
template <int GS, int VPL, bool V4, bool ONE>
__global__ __launch_bounds__(kLossThreads) void seq_loss_kernel(const SeqArgs a) {
    constexpr int TPW = 64 / GS;
    __shared__ float red[kLossThreads / 64];
    __shared__ int last, used_one;
    __shared__ int hist[ONE ? kOneCounts : 1];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int grp = lane / GS, sl = lane % GS;
    const int E = a.E;
    const auto add = [](float x, float y) { return x + y; };
    const auto fmx = [](float x, float y) { return fmaxf(x, y); };
    auto index = [&](int i) { return V4 ? (i / 4) * GS * 4 + sl * 4 + i % 4 : sl + GS * i; };
    const int per_wave = a.tok_per_block / (kLossThreads / 64);
    const long long block0 = (long long)blockIdx.x * a.tok_per_block;
    const int t0 = (int)min(block0 + wave * per_wave, (long long)a.T), end = (int)min((long long)t0 + per_wave, (long long)a.T);
    const float none = a.softmax ? -INFINITY : 0.f;          // past the pool: adds nothing to any sum
    float zn[VPL];
    auto fetch = [&](int t) {
        const float* zr = a.logits + (size_t)min(t, a.T - 1) * E;
        if constexpr (V4) {
#pragma unroll
            for (int i = 0; i < VPL; i += 4) {
                const f32x4 v = index(i) < E ? *reinterpret_cast<const f32x4*>(zr + index(i)) : f32x4{none, none, none, none};
#pragma unroll
                for (int j = 0; j < 4; j++) zn[i + j] = v[j];
            }
        } else {
#pragma unroll
            for (int i = 0; i < VPL; i++) zn[i] = index(i) < E ? zr[index(i)] : none;
        }
    };
    float sum = 0.f;
    int b = 0, s0 = 0, s1 = 0;
    if (t0 < end) {
        fetch(t0 + grp);
        b = find_sequence(a, t0, lane);
        if (b < a.n_seq) seq_range(a, b, s0, s1);
    }
    const int n_counts = a.n_seq * E;
    if constexpr (ONE) {
        for (int i = threadIdx.x; i < n_counts; i += kLossThreads) hist[i] = 0;
        if (threadIdx.x == 0) used_one = 0;
        __syncthreads();
        for (int i = wave; i < a.n_seq; i += kLossThreads / 64) {          // a wavefront to a sequence
            int r0, r1;
            seq_range(a, i, r0, r1);
            if (lane == 0 && r1 > r0) atomicAdd(&used_one, 1);
            for (int s = r0 * a.k + lane; s < r1 * a.k; s += 64) {
                const int e = a.topk_idx[s];
                if (e >= 0 && e < E) atomicAdd(&hist[i * E + e], 1);
            }
        }
        __syncthreads();
        for (int i = threadIdx.x; i < n_counts; i += kLossThreads) a.counts[i] = hist[i];
    }
    const int* const counts = ONE ? hist : a.counts;
    const float used = (float)(ONE ? used_one : a.state[0]);
    int have = -1;                                   // the sequence whose coefficients are held
    float coef[VPL];
#pragma unroll
    for (int i = 0; i < VPL; i++) coef[i] = 0.f;
    for (int tw = t0; tw < end; tw += TPW) {
        const int t = tw + grp;
        const bool live = t < end;
        if (b < a.n_seq && s1 <= t) {                // mostly the next one; behind many empty ones it is looked for
            b++;
            if (b < a.n_seq) seq_range(a, b, s0, s1);
            if (b < a.n_seq && s1 <= t) {
                int hi = a.n_seq;
                for (b++; b < hi;) {
                    const int mid = b + (hi - b) / 2;
                    if (a.offsets[mid + 1] > t) hi = mid;
                    else b = mid + 1;
                }
                if (b < a.n_seq) seq_range(a, b, s0, s1);
            }
        }
        const bool in = live && b < a.n_seq && t >= s0;
        if (in && have != b) {
            have = b;
            const float len = (float)(s1 - s0);
            const float w = a.alpha * (float)E / ((float)a.k * len * len * used);
#pragma unroll
            for (int i = 0; i < VPL; i++) coef[i] = index(i) < E ? w * (float)counts[(size_t)b * E + index(i)] : 0.f;
        }
        float z[VPL], dz[VPL];
#pragma unroll
        for (int i = 0; i < VPL; i++) z[i] = zn[i];
        if (tw + TPW < end) fetch(tw + TPW + grp);
        float part = 0.f;
        if (a.softmax) {
            float zmax = z[0];
#pragma unroll
            for (int i = 1; i < VPL; i++) zmax = fmaxf(zmax, z[i]);
            zmax = group_reduce_f<GS>(zmax, fmx);
            float se = 0.f;
#pragma unroll
            for (int i = 0; i < VPL; i++) {
                z[i] = __expf(z[i] - zmax);           // off by 2^-23 of the exponent, so of small probabilities only
                se += z[i];
            }
            se = group_reduce_f<GS>(se, add);
            const float inv = 1.0f / se;
#pragma unroll
            for (int i = 0; i < VPL; i++) {
                z[i] *= inv;
                dz[i] = coef[i] * z[i];
                part += dz[i];
            }
            part = group_reduce_f<GS>(part, add);
#pragma unroll
            for (int i = 0; i < VPL; i++) dz[i] -= z[i] * part;
        } else {
            float ss = 0.f;
#pragma unroll
            for (int i = 0; i < VPL; i++) ss += z[i] * z[i];
            ss = group_reduce_f<GS>(ss, add);
            const float n = sqrtf(ss), inv = 1.0f / (n + a.eps), sc = a.sigma * a.c;
            float dot = 0.f;
#pragma unroll
            for (int i = 0; i < VPL; i++) {
                dz[i] = z[i] * inv > 0.f ? coef[i] * sc : 0.f;
                dot += dz[i] * z[i];
            }
            dot = group_reduce_f<GS>(dot, add);
            part = n > 0.f ? dot * inv : 0.f;                          // <coef, s>; a token without a direction has none (eps may be 0)
            const float back = n > 0.f ? dot * inv * inv / n : 0.f;
#pragma unroll
            for (int i = 0; i < VPL; i++) dz[i] = n > 0.f ? dz[i] * inv - z[i] * back : 0.f;
        }
        if (in && sl == 0) sum += part;
        if (live && a.d_logits != nullptr) {
            float* o = a.d_logits + (size_t)t * E;
            if constexpr (V4) {
#pragma unroll
                for (int i = 0; i < VPL; i += 4)
                    if (index(i) < E)
                        *reinterpret_cast<f32x4*>(o + index(i)) = in ? f32x4{dz[i], dz[i + 1], dz[i + 2], dz[i + 3]} : f32x4{0.f, 0.f, 0.f, 0.f};
            } else {
#pragma unroll
                for (int i = 0; i < VPL; i++)
                    if (index(i) < E) o[index(i)] = in ? dz[i] : 0.f;
            }
        }
    }
    // The workgroup's share in a fixed order; the last workgroup to hand its share in adds all of them up, in a fixed order too.  (The
    // barriers do not wait for the gradients on their way to memory.)
    sum = wave_sum(sum);
    if (lane == 0) red[wave] = sum;
    lds_barrier();
    if (threadIdx.x == 0) {
        float v = 0.f;
        for (int w = 0; w < kLossThreads / 64; w++) v += red[w];
        if constexpr (ONE) {
            a.loss[0] = v;
            if (a.d_sigma != nullptr) a.d_sigma[0] = a.softmax ? 0.f : v / a.sigma;
            return;
        }
        // The exchange returns when the share has reached memory, where all XCDs see it; only then is the arrival counted.  An
        // arrival with release order instead would write the whole L2 back, once per workgroup (16384 tokens of 512 experts: 53 us).
        const float old = __hip_atomic_exchange(&a.loss_part[blockIdx.x], v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        int one = 1;
        asm volatile("" : "+v"(one) : "v"(old) : "memory");
        last = __hip_atomic_fetch_add(&a.state[1], one, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (int)gridDim.x - 1;
    }
    if constexpr (ONE) return;
    lds_barrier();
    if (!last) return;
    float v = 0.f;
    for (int i = threadIdx.x; i < (int)gridDim.x; i += kLossThreads)
        v += __hip_atomic_load(&a.loss_part[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    v = wave_sum(v);
    if (lane == 0) red[wave] = v;                    // (thread 0 has read the shares that were there)
    lds_barrier();
    if (threadIdx.x == 0) {
        v = 0.f;
        for (int w = 0; w < kLossThreads / 64; w++) v += red[w];
        a.loss[0] = v;
        if (a.d_sigma != nullptr) a.d_sigma[0] = a.softmax ? 0.f : v / a.sigma;
    }
}

}  // namespace

hipError_t launch_seq_balance_loss(const unipool_shape& s, int n_seq, const int32_t* seq_offsets, float alpha, const float* logits,
                                   const int32_t* topk_idx, int32_t* counts, float* loss, float* d_logits, float* d_sigma,
                                   int32_t* cnt_part, float* loss_part, int32_t* state, hipStream_t st) {
    SeqArgs a = {};
    a.offsets = seq_offsets; a.logits = logits; a.topk_idx = topk_idx; a.counts = counts; a.part = cnt_part; a.state = state;
    a.loss_part = loss_part; a.loss = loss; a.d_logits = d_logits; a.d_sigma = d_sigma;
    a.T = s.T; a.E = s.E; a.k = s.k; a.n_seq = n_seq;
    // In 64 bits: T, n_seq kTokensPerPart and a workgroup's tokens are each below 2^31, their sums are not.
    // (parts n_seq <= T / kTokensPerPart + n_seq <= 2 T / kTokensPerPart: fits the area of the partial counts, T / 64 rows)
    const auto pieces = [](long long n, long long of) { return (n + of - 1) / of; };
    const long long per_part = (long long)n_seq * kTokensPerPart;
    a.parts = per_part <= s.T ? (int)std::min(pieces(s.T, per_part), 1024LL) : 1;
    a.alpha = alpha; a.sigma = s.sigma; a.c = s.c; a.eps = s.eps;
    a.softmax = s.router == UNIPOOL_ROUTER_SOFTMAX;
    a.tok_per_block = (int)(kLossTokens * pieces(pieces(s.T, kLossTokens), kLossBlocks));      // (a word per 64 tokens at most in loss_part)
    // A few tokens go in one launch instead of two (128 tokens, 8 experts 8.1 -> 5.2 us on the device)
    const bool one = s.T <= kOneTokens && (long long)n_seq * s.E <= kOneCounts;
    if (one) {
        a.tok_per_block = kLossTokens * cdiv(s.T, kLossTokens);
    } else {
        seq_count_kernel<<<dim3(n_seq, a.parts), kCountThreads, 0, st>>>(a);
        if (a.parts > 1) seq_count_sum_kernel<<<(unsigned)(((size_t)n_seq * s.E + 255) / 256), 256, 0, st>>>(a);
    }
    const bool v4 = s.E % 4 == 0 && (((uintptr_t)logits | (uintptr_t)d_logits) & 15) == 0;
    const int grid = (int)pieces(s.T, a.tok_per_block);
    auto run = [&](auto gs, auto vpl) {
        if (one && v4) seq_loss_kernel<gs(), vpl(), true, true><<<1, kLossThreads, 0, st>>>(a);
        else if (one) seq_loss_kernel<gs(), vpl(), false, true><<<1, kLossThreads, 0, st>>>(a);
        else if (v4) seq_loss_kernel<gs(), vpl(), true, false><<<grid, kLossThreads, 0, st>>>(a);
        else seq_loss_kernel<gs(), vpl(), false, false><<<grid, kLossThreads, 0, st>>>(a);
    };
    using std::integral_constant;
    if (s.E <= 64) run(integral_constant<int, 16>{}, integral_constant<int, 4>{});
    else if (s.E <= 128) run(integral_constant<int, 16>{}, integral_constant<int, 8>{});
    else if (s.E <= 256) run(integral_constant<int, 16>{}, integral_constant<int, 16>{});
    else run(integral_constant<int, 32>{}, integral_constant<int, 16>{});
    return hipGetLastError();
}

}  // namespace unipool
