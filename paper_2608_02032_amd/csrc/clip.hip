// clip.hip -- the global norm of many gradient tensors and their clipping:
//   n = scale sqrt(sum over all tensors of sum g^2),
//   c = min(1, max_norm / (n + 1e-6)),   out = g scale c.
// The squares are formed and summed in 64 bits: the square of no float
// overflows or underflows there, and sums over 10^9 elements keep their digits.
// The order is fixed (no atomics).
#include "dart_common.hpp"
#include "dart_internal.hpp"

namespace dart {
namespace {

// One tensor of the list, and the first of the chunks of kChunk elements that
// the list is cut into.
struct Entry {
    const void* g;
    void* out;
    int64_t numel;
    int32_t first;
    int16_t dtype, out_dtype;
};
constexpr int64_t kChunk = 8192;
constexpr int kInline = 120;       // entries in a launch's arguments (4 KiB)
constexpr int kMaxBlocks = 2048;   // of the norm: partial sums to add

struct Batch {
    Entry e[kInline];
};

__global__ void k_clip_table(Batch b, int n, Entry* table) {
    for (int i = threadIdx.x; i < n; i += blockDim.x) table[i] = b.e[i];
}

// The entry that chunk c belongs to: the last whose first chunk is at most c.
__device__ __forceinline__ int find_entry(const Entry* tab, int n, int64_t c) {
    int lo = 0, hi = n - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) / 2;
        if (tab[mid].first <= c) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}

__device__ __forceinline__ double block_sum64(double v, double* s_red) {
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) v += __shfl_xor(v, o, 64);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) s_red[threadIdx.x >> 6] = v;
    __syncthreads();
    double s = 0;
    for (int i = 0; i < (int)(blockDim.x >> 6); ++i) s += s_red[i];
    return s;
}

__global__ __launch_bounds__(256) void k_grad_norm(const Entry* tab, int n, int64_t chunks, double* part) {
    __shared__ double s_red[4];
    double acc = 0;
    for (int64_t c = blockIdx.x; c < chunks; c += gridDim.x) {
        const Entry e = tab[find_entry(tab, n, c)];
        const int64_t i0 = (c - e.first) * kChunk, i1 = i0 + kChunk < e.numel ? i0 + kChunk : e.numel;
        for (int64_t i = i0 + threadIdx.x; i < i1; i += 256) {
            const double v = e.dtype == 1 ? (double)to_f(((const bf16*)e.g)[i]) : (double)((const float*)e.g)[i];
            acc += v * v;
        }
    }
    acc = block_sum64(acc, s_red);
    if (threadIdx.x == 0) part[blockIdx.x] = acc;
}

// Every block adds the partial sums in the same order; the first one writes the norm.
__global__ __launch_bounds__(256) void k_clip(const Entry* tab, int n, int64_t chunks, const double* part,
                                              int nparts, float max_norm, float scale, float* norm) {
    __shared__ double s_red[4];
    double acc = 0;
    for (int i = threadIdx.x; i < nparts; i += 256) acc += part[i];
    const double total = fabs((double)scale) * sqrt(block_sum64(acc, s_red));
    if (blockIdx.x == 0 && threadIdx.x == 0) norm[0] = (float)total;
    const double coef = (double)max_norm / (total + 1e-6);
    const float f = (float)(scale * (coef >= 1.0 ? 1.0 : coef));  // (a NaN stays)
    for (int64_t c = blockIdx.x; c < chunks; c += gridDim.x) {
        const Entry e = tab[find_entry(tab, n, c)];
        if (f == 1.f && e.out == e.g) continue;
        const int64_t i0 = (c - e.first) * kChunk, i1 = i0 + kChunk < e.numel ? i0 + kChunk : e.numel;
        for (int64_t i = i0 + threadIdx.x; i < i1; i += 256) {
            const float v = f * (e.dtype == 1 ? to_f(((const bf16*)e.g)[i]) : ((const float*)e.g)[i]);
            if (e.out_dtype == 1) ((bf16*)e.out)[i] = (bf16)v;
            else ((float*)e.out)[i] = v;
        }
    }
}

size_t table_bytes(int64_t n) { return align256(sizeof(Entry) * (size_t)(n > 0 ? n : 1)); }

}  // namespace

size_t grad_norm_workspace_bytes(int64_t n) { return table_bytes(n) + sizeof(double) * kMaxBlocks; }

hipError_t launch_clip_grad_norm(int64_t n, const void* const* grads, void* const* outs,
                                 const int64_t* numels, const int32_t* dtypes,
                                 const int32_t* out_dtypes, float max_norm, float scale, float* norm,
                                 void* ws, hipStream_t st) {
    Entry* table = reinterpret_cast<Entry*>(ws);
    double* part = reinterpret_cast<double*>((char*)ws + table_bytes(n));
    int64_t chunks = 0;
    int entries = 0;
    Batch b;
    for (int64_t i = 0; i < n; ++i) {
        if (numels[i] == 0) continue;
        Entry& e = b.e[entries % kInline];
        e.g = grads[i];
        e.out = outs ? outs[i] : nullptr;
        e.numel = numels[i];
        e.first = (int32_t)chunks;
        e.dtype = (int16_t)dtypes[i];
        e.out_dtype = (int16_t)(outs ? out_dtypes[i] : dtypes[i]);
        chunks += (numels[i] + kChunk - 1) / kChunk;
        if (++entries % kInline == 0) {
            prof_begin("k_clip_table", st);
            k_clip_table<<<1, 128, 0, st>>>(b, kInline, table + entries - kInline);
            prof_end(st);
        }
    }
    if (const int rest = entries % kInline) {
        prof_begin("k_clip_table", st);
        k_clip_table<<<1, 128, 0, st>>>(b, rest, table + entries - rest);
        prof_end(st);
    }
    const int blocks = (int)(chunks < kMaxBlocks ? chunks : kMaxBlocks);
    if (blocks > 0) {
        prof_begin("k_grad_norm", st);
        k_grad_norm<<<blocks, 256, 0, st>>>(table, entries, chunks, part);
        prof_end(st);
    }
    prof_begin("k_clip", st);
    k_clip<<<outs && blocks > 0 ? blocks : 1, 256, 0, st>>>(table, entries, outs ? chunks : 0, part, blocks, max_norm, scale, norm);
    prof_end(st);
    return hipGetLastError();
}

}  // namespace dart
