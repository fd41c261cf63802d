// clip.hip -- the global norm of many gradient tensors and their clipping:
//   n = scale sqrt(sum over all tensors of sum g^2),
//   c = min(1, max_norm / (n + 1e-6)) (1 without a limit),   out = g scale c.
// The squares are formed and summed in 64 bits: the square of no float
// overflows or underflows there, and sums over 10^9 elements keep their digits.
// The order is fixed (no atomics).
//
// Bound by HBM: every gradient is read for the norm and, as the factor needs
// them all, again for the clipping.  Two launches: partial sums of a grid that
// fills the card once, each workgroup walking a stretch of the list; then the
// same stretches backwards, the last read first (what the 256 MB cache in front
// of the HBM still holds), every workgroup adding the partial sums by itself.
// A list of up to 120 tensors travels in the launches' arguments.  Two tensors of
// 38.6 M float: the norm 51 us (6.0 TB/s), with the clipping into others 187 us (4.9
// TB/s); chunks of 4096 elements, half as much in flight, 65 and 190.
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
constexpr int kChunk = 8192;
constexpr int kThreads = 256;
constexpr int kInline = 120;      // entries in a launch's arguments (4 KiB)
constexpr int kPerCu = 4;        // workgroups of the grid

struct Batch {
    Entry e[kInline];
};

__global__ void k_clip_table(const Batch b, int n, Entry* table) {
    for (int i = threadIdx.x; i < n; i += blockDim.x) table[i] = b.e[i];
}

// The entry that chunk c belongs to: the last whose first chunk is at most c.
__device__ __forceinline__ int find_entry(const Entry* tab, int n, int64_t c) {
    int at = -1;
    for (int i = 0; i < n; i += kThreads) {
        const int j = i + (int)threadIdx.x;
        at += __syncthreads_count(j < n && tab[j < n ? j : 0].first <= c);
    }
    return at;
}

__device__ __forceinline__ double block_sum64(double v, double* s_red) {
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) v += __shfl_xor(v, o, 64);
    if ((threadIdx.x & 63) == 0) s_red[threadIdx.x >> 6] = v;
    __syncthreads();
    return s_red[0] + s_red[1] + s_red[2] + s_red[3];
}

__device__ __forceinline__ float bits_f(uint32_t u) { return __builtin_bit_cast(float, u); }

// N elements of T at any alignment of one, N sizeof(T) = 8 or 16 bytes.
template <int WORDS> struct Words;
template <> struct Words<4> { typedef unsigned int type __attribute__((ext_vector_type(4))); typedef type mem __attribute__((aligned(2))); };
template <> struct Words<2> { typedef unsigned int type __attribute__((ext_vector_type(2))); typedef type mem __attribute__((aligned(2))); };
template <typename T, int N> struct Pack {
    using W = Words<N * (int)sizeof(T) / 4>;
    using type = typename W::type;
    static __device__ __forceinline__ type load(const T* p) { return *reinterpret_cast<const typename W::mem*>(p); }
    static __device__ __forceinline__ type load_last(const T* p) { return __builtin_nontemporal_load(reinterpret_cast<const typename W::mem*>(p)); }
    static __device__ __forceinline__ void unpack(type r, float (&v)[N]) {
#pragma unroll
        for (int i = 0; i < N * (int)sizeof(T) / 4; ++i) {
            if constexpr (sizeof(T) == 2) {
                v[2 * i] = bits_f(r[i] << 16);
                v[2 * i + 1] = bits_f(r[i] & 0xFFFF0000u);
            } else {
                v[i] = bits_f(r[i]);
            }
        }
    }
};
template <int N>
__device__ __forceinline__ void store_n(bf16* p, const float (&v)[N]) {
    typedef bf16 vec __attribute__((ext_vector_type(N)));
    typedef vec mem __attribute__((aligned(2)));
    vec r;
#pragma unroll
    for (int i = 0; i < N; ++i) r[i] = (bf16)v[i];
    *reinterpret_cast<mem*>(p) = r;
}
template <int N>
__device__ __forceinline__ void store_n(float* p, const float (&v)[N]) {
    typedef f32x4 mem __attribute__((aligned(4)));
#pragma unroll
    for (int i = 0; i < N; i += 4) *reinterpret_cast<mem*>(p + i) = f32x4{v[i], v[i + 1], v[i + 2], v[i + 3]};
}

// Elements [i0, i0 + n) of a tensor, n <= kChunk: whole vectors, U of them in
// flight, then single elements.
template <typename T>
__device__ __forceinline__ void chunk_squares(const T* g, int n, double& acc) {
    constexpr int N = 16 / sizeof(T), U = kChunk / (kThreads * N);
    const int whole = n / N;
    typename Pack<T, N>::type r[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int v = threadIdx.x + u * kThreads;
        r[u] = {};
        if (v < whole) r[u] = Pack<T, N>::load(g + v * N);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        float f[N];
        Pack<T, N>::unpack(r[u], f);
#pragma unroll
        for (int i = 0; i < N; ++i) acc += (double)f[i] * (double)f[i];
    }
    const int at = whole * N + threadIdx.x;
    if (at < n) {
        const double d = (double)to_f(g[at]);
        acc += d * d;
    }
}
template <typename T, typename O>
__device__ __forceinline__ void chunk_scale(const T* g, O* out, int n, float f) {
    // (16 bytes of the wider type: a wave's stores cover whole lines)
    constexpr int N = 16 / (sizeof(T) > sizeof(O) ? sizeof(T) : sizeof(O)), U = kChunk / (kThreads * N);
    const int whole = n / N;
    typename Pack<T, N>::type r[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int v = threadIdx.x + u * kThreads;
        if (v < whole) r[u] = Pack<T, N>::load_last(g + v * N);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int v = threadIdx.x + u * kThreads;
        if (v < whole) {
            float x[N];
            Pack<T, N>::unpack(r[u], x);
#pragma unroll
            for (int i = 0; i < N; ++i) x[i] *= f;
            store_n(out + v * N, x);
        }
    }
    const int at = whole * N + threadIdx.x;
    if (at < n) out[at] = from_f<O>(to_f(g[at]) * f);
}

// Chunk c of entry e: its first element and how many it has.
__device__ __forceinline__ int chunk_of(const Entry& e, int64_t c, int64_t& i0) {
    i0 = (c - e.first) * kChunk;
    return (int)(e.numel - i0 < kChunk ? e.numel - i0 : kChunk);
}

template <bool INLINE>
__global__ __launch_bounds__(kThreads) void k_grad_norm(const Batch b, const Entry* table, int n, int64_t chunks, double* part) {
    __shared__ double s_red[4];
    const Entry* tab = INLINE ? b.e : table;
    const int64_t c0 = chunks * blockIdx.x / gridDim.x, c1 = chunks * (blockIdx.x + 1) / gridDim.x;
    int at = find_entry(tab, n, c0);
    double acc = 0;
    Entry e = tab[at];
    int64_t last = e.first + (e.numel + kChunk - 1) / kChunk;  // one past its chunks
    for (int64_t c = c0; c < c1; ++c) {
        if (c == last) {
            e = tab[++at];
            last = e.first + (e.numel + kChunk - 1) / kChunk;
        }
        int64_t i0;
        const int m = chunk_of(e, c, i0);
        if (e.dtype == 1) chunk_squares((const bf16*)e.g + i0, m, acc);
        else chunk_squares((const float*)e.g + i0, m, acc);
    }
    acc = block_sum64(acc, s_red);
    if (threadIdx.x == 0) part[blockIdx.x] = acc;
}

// Every block adds the partial sums in the same order; the first one writes the norm.
template <bool INLINE>
__global__ __launch_bounds__(kThreads) void k_clip(const Batch b, const Entry* table, int n, int64_t chunks, const double* part,
                                                   int nparts, float max_norm, float scale, float* norm) {
    __shared__ double s_red[4];
    const Entry* tab = INLINE ? b.e : table;
    double acc = 0;
    for (int i = threadIdx.x; i < nparts; i += kThreads) acc += part[i];
    const double total = fabs((double)scale) * sqrt(block_sum64(acc, s_red));
    if (blockIdx.x == 0 && threadIdx.x == 0) norm[0] = (float)total;
    // (no limit, no clipping: an infinite norm would make inf / inf of it)
    const double coef = max_norm == INFINITY && total == total ? 1.0 : (double)max_norm / (total + 1e-6);
    const float f = (float)(scale * (coef >= 1.0 ? 1.0 : coef));  // (a NaN stays)
    const int64_t c0 = chunks * blockIdx.x / gridDim.x, c1 = chunks * (blockIdx.x + 1) / gridDim.x;
    if (c0 == c1) return;
    int at = find_entry(tab, n, c1 - 1);
    Entry e = tab[at];
    for (int64_t c = c1 - 1; c >= c0; --c) {
        if (c < e.first) e = tab[--at];
        if (f == 1.f && e.out == e.g) {  // nothing changes
            c = e.first;
            continue;
        }
        int64_t i0;
        const int m = chunk_of(e, c, i0);
        if (e.dtype == 1) {
            if (e.out_dtype == 1) chunk_scale((const bf16*)e.g + i0, (bf16*)e.out + i0, m, f);
            else chunk_scale((const bf16*)e.g + i0, (float*)e.out + i0, m, f);
        } else {
            if (e.out_dtype == 1) chunk_scale((const float*)e.g + i0, (bf16*)e.out + i0, m, f);
            else chunk_scale((const float*)e.g + i0, (float*)e.out + i0, m, f);
        }
    }
}

size_t table_bytes(int64_t n) { return align256(sizeof(Entry) * (size_t)(n > kInline ? n : 0)); }
int64_t max_blocks() { return (int64_t)device_cu_count() * kPerCu; }

}  // namespace

size_t grad_norm_workspace_bytes(int64_t n) { return table_bytes(n) + sizeof(double) * max_blocks(); }

hipError_t launch_clip_grad_norm(int64_t n, const void* const* grads, void* const* outs,
                                 const int64_t* numels, const int32_t* dtypes,
                                 const int32_t* out_dtypes, float max_norm, float scale, float* norm,
                                 void* ws, hipStream_t st) {
    Entry* table = reinterpret_cast<Entry*>(ws);
    double* part = reinterpret_cast<double*>((char*)ws + table_bytes(n));
    const bool in_args = n <= kInline;
    int64_t chunks = 0;
    int entries = 0;
    Batch b = {};
    const auto write_table = [&](int count) {
        prof_begin("k_clip_table", st);
        k_clip_table<<<1, 128, 0, st>>>(b, count, table + entries - count);
        prof_end(st);
    };
    for (int64_t i = 0; i < n; ++i) {
        if (numels[i] == 0) continue;
        b.e[entries % kInline] = Entry{grads[i], outs ? outs[i] : nullptr, numels[i], (int32_t)chunks,
                                       (int16_t)dtypes[i], (int16_t)(outs ? out_dtypes[i] : dtypes[i])};
        chunks += (numels[i] + kChunk - 1) / kChunk;
        if (++entries % kInline == 0 && !in_args) write_table(kInline);
    }
    if (!in_args && entries % kInline) write_table(entries % kInline);
    const int blocks = (int)(chunks < max_blocks() ? chunks : max_blocks());
    if (blocks > 0) {
        prof_begin("k_grad_norm", st);
        if (in_args) k_grad_norm<true><<<blocks, kThreads, 0, st>>>(b, nullptr, entries, chunks, part);
        else k_grad_norm<false><<<blocks, kThreads, 0, st>>>(Batch{}, table, entries, chunks, part);
        prof_end(st);
    }
    const int clip_blocks = outs && blocks > 0 ? blocks : 1;
    prof_begin("k_clip", st);
    if (in_args) k_clip<true><<<clip_blocks, kThreads, 0, st>>>(b, nullptr, entries, outs ? chunks : 0, part, blocks, max_norm, scale, norm);
    else k_clip<false><<<clip_blocks, kThreads, 0, st>>>(Batch{}, table, entries, outs ? chunks : 0, part, blocks, max_norm, scale, norm);
    prof_end(st);
    return hipGetLastError();
}

}  // namespace dart
