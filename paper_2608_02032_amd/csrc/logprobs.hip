// logprobs.hip -- log probabilities of given tokens over a vocabulary, with
// the entropy and the best alternatives, and their gradient.  For a row l of V
// logits, in one pass with the running maximum m:
//   s = sum exp(l_j - m),  c = sum exp(l_j - m) (l_j - m),
//   logprob = (l_t - m) - log s,  entropy = log s - c / s.
// The pieces m and log s stay apart: their sum rounds at the size of m, their
// difference from a logit does not.  Backward, with p_j = exp(l_j - m - log s):
//   dl_j = p_j (dlse - dlogprob - dentropy (log p_j + entropy)) + [j = t] dlogprob.
// A logit of -infinity has p = 0 and takes no part; a row of nothing else has
// no distribution (m = log s = -infinity, entropy 0, p = 0).
#include "dart_common.hpp"
#include "dart_internal.hpp"

namespace dart {
namespace {

constexpr float kLowest = -3.402823466e+38f;
constexpr float kFar = -1e30f;  // stands for a logit's distance of -infinity where exp is 0

// Statistics of part of a row: maximum (at least kLowest), sum, weighted sum.
struct Stat {
    float m, s, c;
};
__device__ __forceinline__ Stat stat_none() { return Stat{kLowest, 0.f, 0.f}; }
__device__ __forceinline__ void stat_add(Stat& a, float l) {
    if (l > a.m) {
        const float d = fmaxf(a.m - l, kFar), f = __expf(d);
        a.c = f * (a.c + a.s * d);
        a.s *= f;
        a.m = l;
    }
    const float d = l - a.m, e = __expf(d);
    a.s += e;
    a.c += e * fmaxf(d, kFar);  // (the maximum drops a NaN, e keeps it)
}
__device__ __forceinline__ Stat stat_join(const Stat& a, const Stat& b) {
    const float m = fmaxf(a.m, b.m);
    const float da = fmaxf(a.m - m, kFar), db = fmaxf(b.m - m, kFar);
    const float fa = __expf(da), fb = __expf(db);
    return Stat{m, fa * a.s + fb * b.s, fa * (a.c + a.s * da) + fb * (b.c + b.s * db)};
}

// Order of the alternatives: by value (a NaN above all, -0 as 0), then by the
// lowest index; as one integer, larger first.
__device__ __forceinline__ uint64_t order_key(float v, uint32_t index) {
    const float z = v + 0.f;
    uint32_t u = __builtin_bit_cast(uint32_t, z);
    u = z != z ? 0xFFFFFFFFu : (u >> 31 ? ~u : u | 0x80000000u);
    return (uint64_t)u << 32 | (uint32_t)~index;
}
__device__ __forceinline__ uint64_t shfl_xor64(uint64_t v, int mask) {
    return (uint64_t)__shfl_xor((unsigned long long)v, mask, 64);
}

// What a row's gradient needs: dl_j = p_j (f + h log p_j) + [j = t] a.
struct RowGrad {
    float m, ls, f, h, a;
    int64_t t;
    bool zero;
};
__device__ __forceinline__ RowGrad row_grad(int64_t r, const int64_t* targets, int64_t ignore, int64_t V,
                                            float m, float ls, float ent, const float* dlogprob,
                                            const float* dentropy, const float* dlse) {
    RowGrad g;
    g.t = targets ? targets[r] : ignore;
    g.a = targets && dlogprob && g.t != ignore ? dlogprob[r] : 0.f;
    if (targets && g.t != ignore && (g.t < 0 || g.t >= V)) g.a = __builtin_nanf("");
    const float dh = dentropy ? dentropy[r] : 0.f;
    g.f = (dlse ? dlse[r] : 0.f) - g.a - (dentropy ? dh * ent : 0.f);
    g.h = -dh;
    const bool none = m == -INFINITY;  // nothing but -infinity
    g.m = none ? 0.f : m;
    g.ls = none ? 0.f : ls;
    g.zero = g.a == 0.f && g.f == 0.f && g.h == 0.f;
    return g;
}
__device__ __forceinline__ float grad_of(const RowGrad& g, float l, int64_t j) {
    const float q = (l - g.m) - g.ls, p = __expf(q);
    // (p is 0 in fp32 long before -200)
    return p * (g.f + g.h * fmaxf(q, -200.f)) + (j == g.t ? g.a : 0.f);
}

// One block per row: a pass for the statistics, one for every alternative.
template <typename T>
__global__ __launch_bounds__(256) void k_token_logprobs(LogprobArgs a) {
    __shared__ Stat s_st[4];
    __shared__ uint64_t s_key[4];
    const int64_t r = flat_block();
    if (r >= a.rows) return;
    const T* row = (const T*)a.logits + r * a.stride;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    Stat st = stat_none();
    for (int64_t j = threadIdx.x; j < a.vocab; j += 256) stat_add(st, to_f(row[j]));
    for (int o = 32; o >= 1; o >>= 1)
        st = stat_join(st, Stat{__shfl_xor(st.m, o, 64), __shfl_xor(st.s, o, 64), __shfl_xor(st.c, o, 64)});
    if (lane == 0) s_st[wave] = st;
    __syncthreads();
    st = stat_join(stat_join(s_st[0], s_st[1]), stat_join(s_st[2], s_st[3]));
    const bool none = st.s == 0.f;  // nothing but -infinity
    const float ls = none ? -INFINITY : logf(st.s), m = none ? 0.f : st.m, lz = none ? 0.f : ls;
    if (threadIdx.x == 0) {
        if (a.row_max) a.row_max[r] = none ? -INFINITY : st.m;
        if (a.log_sum) a.log_sum[r] = ls;
        if (a.entropy) a.entropy[r] = none ? 0.f : ls - st.c / st.s;
        if (a.logprob) {
            const int64_t t = a.targets[r];
            a.logprob[r] = t == a.ignore_index ? 0.f : t < 0 || t >= a.vocab ? __builtin_nanf("") : (to_f(row[t]) - m) - lz;
        }
    }
    uint64_t last = ~0ull;
    for (int k = 0; k < a.top_k; ++k) {
        uint64_t best = 0;
        for (int64_t j = threadIdx.x; j < a.vocab; j += 256) {
            const uint64_t key = order_key(to_f(row[j]), (uint32_t)j);
            if (key > best && (k == 0 || key < last)) best = key;
        }
        for (int o = 32; o >= 1; o >>= 1) {
            const uint64_t v = shfl_xor64(best, o);
            best = v > best ? v : best;
        }
        __syncthreads();
        if (lane == 0) s_key[wave] = best;
        __syncthreads();
        for (int i = 0; i < 4; ++i) best = s_key[i] > best ? s_key[i] : best;
        last = best;
        if (threadIdx.x == 0) {
            const uint32_t j = ~(uint32_t)best;
            a.top_ids[r * a.top_k + k] = j;
            a.top_logprobs[r * a.top_k + k] = (to_f(row[j]) - m) - lz;
        }
    }
}

template <typename T, typename GT>
__global__ __launch_bounds__(256) void k_token_logprobs_bwd(LogprobArgs a, LogprobGrad g) {
    const int64_t r = flat_block();
    if (r >= a.rows) return;
    const T* row = (const T*)a.logits + r * a.stride;
    GT* out = (GT*)g.dlogits + r * g.stride;
    const RowGrad rg = row_grad(r, a.targets, a.ignore_index, a.vocab, a.row_max[r], a.log_sum[r],
                                g.dentropy ? a.entropy[r] : 0.f, g.dlogprob, g.dentropy, g.dlse);
    for (int64_t j = threadIdx.x; j < a.vocab; j += 256)
        out[j] = from_f<GT>(rg.zero ? 0.f : grad_of(rg, to_f(row[j]), j));
}

}  // namespace

size_t token_logprobs_workspace_bytes(int64_t, int64_t, int, int) { return 0; }

hipError_t launch_token_logprobs(const LogprobArgs& a, const LogprobGrad* grad, void*, hipStream_t st) {
    if (a.rows == 0) return hipSuccess;
    prof_begin("k_token_logprobs", st);
    if (a.dtype == 1) k_token_logprobs<bf16><<<flat_grid(a.rows, 256), 256, 0, st>>>(a);
    else k_token_logprobs<float><<<flat_grid(a.rows, 256), 256, 0, st>>>(a);
    prof_end(st);
    return grad ? launch_token_logprobs_bwd(a, *grad, st) : hipGetLastError();
}

hipError_t launch_token_logprobs_bwd(const LogprobArgs& a, const LogprobGrad& g, hipStream_t st) {
    if (a.rows == 0) return hipSuccess;
    const dim3 grid = flat_grid(a.rows, 256);
    prof_begin("k_token_logprobs_bwd", st);
    if (a.dtype == 0) k_token_logprobs_bwd<float, float><<<grid, 256, 0, st>>>(a, g);
    else if (g.dtype == 0) k_token_logprobs_bwd<bf16, float><<<grid, 256, 0, st>>>(a, g);
    else k_token_logprobs_bwd<bf16, bf16><<<grid, 256, 0, st>>>(a, g);
    prof_end(st);
    return hipGetLastError();
}

}  // namespace dart
