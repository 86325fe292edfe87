// Balance loss of one layer over the sequences of a batch, with the gradient of its logits and its sigma.
//
// Sequence b holds the tokens [o_b, o_{b+1}), T_b of them; n_{b,i} of its picks went to expert i.  With
//   f_{b,i} = E n_{b,i} / (k T_b),   P_{b,i} = mean over the sequence of the score s_{t,i},
//   loss = alpha / B' sum_b sum_i f_{b,i} P_{b,i}        (B': sequences that have tokens; f is constant for differentiation)
// the gradient of a score is coef_{b,i} = alpha f_{b,i} / (B' T_b), the same for all tokens of a sequence, and the loss is the sum of
// <coef, s_t> over the tokens.  coef follows from the picks alone, so the picks are counted first and ONE pass over the logits
// then gives loss and gradient.  The score is linear in sigma: d loss / d sigma = loss / sigma (softmax: 0).
//
// Bound by memory: 4 bytes in and 4 out per logit, in the lane layout of the router's backward pass.
#include <algorithm>

#include "route_select.h"
#include "kernels.h"

namespace unipool {

namespace {

constexpr int kTokensPerPart = 4096;      // tokens of a sequence that one workgroup counts

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

// Picks per expert of part blockIdx.y of sequence blockIdx.x.
__global__ __launch_bounds__(256) void seq_count_kernel(const SeqArgs a) {
    __shared__ int hist[kMaxE];
    __shared__ int used[4];
    const int b = blockIdx.x, p = blockIdx.y;
    for (int i = threadIdx.x; i < a.E; i += 256) hist[i] = 0;
    int t0, t1;
    seq_range(a, b, t0, t1);
    const int per = (int)(((long long)(t1 - t0) + a.parts - 1) / a.parts);
    const long long s0 = (long long)min(t0 + (long long)p * per, (long long)t1) * a.k, s1 = (long long)min(t0 + (long long)(p + 1) * per, (long long)t1) * a.k;
    __syncthreads();
    for (long long s = s0 + threadIdx.x; s < s1; s += 256) {
        const int e = a.topk_idx[s];
        if (e >= 0 && e < a.E) atomicAdd(&hist[e], 1);
    }
    __syncthreads();
    int32_t* out = (a.parts > 1 ? a.part + (size_t)p * a.n_seq * a.E : a.counts) + (size_t)b * a.E;
    for (int i = threadIdx.x; i < a.E; i += 256) out[i] = hist[i];
    if (b == 0 && p == 0) {
        int n = 0;
        for (int i = threadIdx.x; i < a.n_seq; i += 256) {
            int r0, r1;
            seq_range(a, i, r0, r1);
            n += r1 > r0;
        }
        n = wave_sum_i(n);
        if ((threadIdx.x & 63) == 0) used[threadIdx.x >> 6] = n;
        __syncthreads();
        if (threadIdx.x == 0) {
            a.state[0] = used[0] + used[1] + used[2] + used[3];
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

// GS lanes to a token, VPL logits to a lane: lane s holds logits s + GS i, or with V4 groups of four neighbours.
template <int GS, int VPL, bool V4>
__global__ __launch_bounds__(256) void seq_loss_kernel(const SeqArgs a) {
    constexpr int TPW = 64 / GS;
    __shared__ float red[256];
    __shared__ int last;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int grp = lane / GS, sl = lane % GS;
    const int E = a.E;
    const auto add = [](float x, float y) { return x + y; };
    const auto fmx = [](float x, float y) { return fmaxf(x, y); };
    auto index = [&](int i) { return V4 ? (i / 4) * GS * 4 + sl * 4 + i % 4 : sl + GS * i; };
    const int per_wave = a.tok_per_block / 4;
    const int t_first = blockIdx.x * a.tok_per_block + wave * per_wave + grp;
    const int end = min(a.T, blockIdx.x * a.tok_per_block + (wave + 1) * per_wave);
    // the sequence that holds a token, or the next one: the first whose end lies behind it
    int b = 0, s0 = 0, s1 = 0;
    {
        int hi = a.n_seq;
        while (b < hi) {
            const int mid = (b + hi) >> 1;
            if (a.offsets[mid + 1] > t_first) hi = mid;
            else b = mid + 1;
        }
        if (b < a.n_seq) seq_range(a, b, s0, s1);
    }
    int have = -1;                                   // the sequence whose coefficients are held
    float coef[VPL];
#pragma unroll
    for (int i = 0; i < VPL; i++) coef[i] = 0.f;
    float sum = 0.f;
    for (int t = t_first; t - grp < end; t += TPW) {                  // the groups of a wavefront stay together
        const bool live = t < end;
        const int tc = min(t, a.T - 1);
        while (b < a.n_seq && s1 <= t) {
            b++;
            if (b < a.n_seq) seq_range(a, b, s0, s1);
        }
        const bool in = live && b < a.n_seq && t >= s0;
        if (in && have != b) {
            have = b;
            const float len = (float)(s1 - s0);
            const float w = a.alpha * (float)E / ((float)a.k * len * len * (float)a.state[0]);
#pragma unroll
            for (int i = 0; i < VPL; i++) coef[i] = index(i) < E ? w * (float)a.counts[(size_t)b * E + index(i)] : 0.f;
        }
        const float* zr = a.logits + (size_t)tc * E;
        float z[VPL], dz[VPL];
        if constexpr (V4) {
#pragma unroll
            for (int i = 0; i < VPL; i += 4) {
                const f32x4 v = index(i) < E ? *reinterpret_cast<const f32x4*>(zr + index(i)) : f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int j = 0; j < 4; j++) z[i + j] = v[j];
            }
        } else {
#pragma unroll
            for (int i = 0; i < VPL; i++) z[i] = index(i) < E ? zr[index(i)] : 0.f;
        }
        float part = 0.f;
        if (a.softmax) {
            float zmax = -INFINITY;
#pragma unroll
            for (int i = 0; i < VPL; i++)
                if (index(i) < E) zmax = fmaxf(zmax, z[i]);
            zmax = group_reduce_f<GS>(zmax, fmx);
            float se = 0.f;
#pragma unroll
            for (int i = 0; i < VPL; i++) {
                z[i] = index(i) < E ? expf(z[i] - zmax) : 0.f;
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
            part = dot * inv;                                          // <coef, s>
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
    // the workgroup's share in a fixed order; the last workgroup to hand its share in adds all of them up, in index order
    sum = wave_sum(sum);
    if (lane == 0) red[wave] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        const float v = ((red[0] + red[1]) + red[2]) + red[3];
        __hip_atomic_store(&a.loss_part[blockIdx.x], v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        last = __hip_atomic_fetch_add(&a.state[1], 1, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) == (int)gridDim.x - 1;
    }
    __syncthreads();
    if (!last) return;
    float v = 0.f;
    for (int i = threadIdx.x; i < (int)gridDim.x; i += 256)
        v += __hip_atomic_load(&a.loss_part[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    red[threadIdx.x] = v;
    __syncthreads();
    for (int s = 128; s > 0; s >>= 1) {
        if (threadIdx.x < s) red[threadIdx.x] += red[threadIdx.x + s];
        __syncthreads();
    }
    if (threadIdx.x == 0) {
        a.loss[0] = red[0];
        if (a.d_sigma != nullptr) a.d_sigma[0] = a.softmax ? 0.f : red[0] / a.sigma;
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
    // (parts n_seq <= T / kTokensPerPart + n_seq <= 2 T / kTokensPerPart: fits the area of the partial counts, T / 64 rows)
    a.parts = (long long)n_seq * kTokensPerPart <= s.T ? std::min(cdiv(s.T, n_seq * kTokensPerPart), 1024) : 1;
    a.alpha = alpha; a.sigma = s.sigma; a.c = s.c; a.eps = s.eps;
    a.softmax = s.router == UNIPOOL_ROUTER_SOFTMAX;
    a.tok_per_block = std::max(dz_tokens_per_block(s), 16);
    seq_count_kernel<<<dim3(n_seq, a.parts), 256, 0, st>>>(a);
    if (a.parts > 1) seq_count_sum_kernel<<<(unsigned)(((size_t)n_seq * s.E + 255) / 256), 256, 0, st>>>(a);
    const bool v4 = s.E % 4 == 0 && (((uintptr_t)logits | (uintptr_t)d_logits) & 15) == 0;
    const int grid = cdiv(s.T, a.tok_per_block);
    auto run = [&](auto gs, auto vpl) {
        if (v4) seq_loss_kernel<gs(), vpl(), true><<<grid, 256, 0, st>>>(a);
        else seq_loss_kernel<gs(), vpl(), false><<<grid, 256, 0, st>>>(a);
    };
    using std::integral_constant;
    if (s.E <= 64) run(integral_constant<int, 16>{}, integral_constant<int, 4>{});
    else if (s.E <= 128) run(integral_constant<int, 16>{}, integral_constant<int, 8>{});
    else if (s.E <= 256) run(integral_constant<int, 16>{}, integral_constant<int, 16>{});
    else run(integral_constant<int, 32>{}, integral_constant<int, 16>{});
    return hipGetLastError();
}

}  // namespace unipool
