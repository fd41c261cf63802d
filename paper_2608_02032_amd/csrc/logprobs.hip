// logprobs.hip -- log probabilities of given tokens over a vocabulary, with
// the entropy and the best alternatives, and their gradient.  For a row l of V
// logits with the maximum m:
//   s = sum exp(l_j - m),  c = sum exp(l_j - m) (l_j - m),
//   logprob = (l_t - m) - log s,  entropy = log s - c / s.
// The pieces m and log s stay apart: their sum rounds at the size of m, their
// difference from a logit does not.  Backward, with p_j = exp(l_j - m - log s):
//   dl_j = p_j (dlse - dlogprob - dentropy (log p_j + entropy)) + [j = t] dlogprob.
// A logit of -infinity has p = 0 and takes no part; a row of nothing else has
// no distribution (m = log s = -infinity, entropy 0, p = 0).
//
// Bound by HBM, with the vector units close behind: some eight instructions per
// logit forward and seven for the gradient, one of each an exponential, against
// two or four bytes.  A workgroup holds a row, packed as stored, in its registers
// (up to 131072 bf16 or 65536 float): every load of the row is in flight at once,
// the maximum comes before the exponentials, and the alternatives and the
// gradient are formed from the registers.  Longer rows, and few rows for the card,
// are cut into segments, one per workgroup, whose results a second launch joins.
// 16384 rows of 50257 bf16: forward 287 us (5.7 TB/s), the gradient after it 556 us
// (5.9 TB/s), both in one pass 680 us (4.8 TB/s, as a copy); with five alternatives
// 8192 rows take 213 us instead of 147; 4096 rows of 131072 forward 180 us (6.0 TB/s),
// with the gradient, a row in 1024 threads, 469 us (4.6 TB/s; 8192 of 50257 float 700,
// 4.7 TB/s); one row of 131072 with twenty alternatives 10 us and 8 us for the join.
#include "dart_common.hpp"
#include "dart_internal.hpp"

#include <type_traits>

namespace dart {
namespace {

constexpr float kLowest = -3.402823466e+38f;
constexpr float kFar = -200.f;  // stands for any distance below it, where exp and exp2 are 0 in float

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
template <typename T> constexpr int kVec = 16 / sizeof(T);  // elements of 16 bytes

__device__ __forceinline__ float bits_f(uint32_t u) { return __builtin_bit_cast(float, u); }
__device__ __forceinline__ void unpack(u32x4 r, float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = bits_f(r[i] << 16);
        v[2 * i + 1] = bits_f(r[i] & 0xFFFF0000u);
    }
}
__device__ __forceinline__ void unpack(u32x4 r, float (&v)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = bits_f(r[i]);
}
// The compiler takes what it unpacked before for unknown: unpacked again it costs
// an instruction per element, kept a register (twice the packed row's).
__device__ __forceinline__ u32x4 again(u32x4& r) {
    asm volatile("" : "+v"(r));
    return r;
}
template <typename T> __device__ __forceinline__ u32x4 all_ninf() {
    const uint32_t u = sizeof(T) == 2 ? 0xFF80FF80u : 0xFF800000u;
    return u32x4{u, u, u, u};
}
// (fmaxf would first quiet every operand, an instruction each; a NaN shows in the sums)
__device__ __forceinline__ float max3(float a, float b, float c) {
    float r;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
    return r;
}
template <int N>
__device__ __forceinline__ float max_of(const float (&v)[N]) {
    float m = max3(v[0], v[1], v[2]);
#pragma unroll
    for (int i = 3; i + 1 < N; i += 2) m = max3(m, v[i], v[i + 1]);
    return max3(m, v[N - 1], v[N - 1]);
}
__device__ __forceinline__ float exp_f(float d) { return fast_exp2(d * kLog2e); }

// Sum and maximum over the wave, in every lane, without LDS (uniform control flow).
__device__ __forceinline__ float wave_sum(float v) { return row4_sum(dpp_group_sum<16>(v)); }
__device__ __forceinline__ float wave_max(float v) {
    v = fmaxf(v, dpp_mov<0xB1>(v));
    v = fmaxf(v, dpp_mov<0x4E>(v));
    v = fmaxf(v, dpp_mov<0x141>(v));
    v = fmaxf(v, dpp_mov<0x140>(v));
    float a = v, b = v;
    asm volatile("s_nop 1\n\tv_permlane32_swap_b32 %0, %1" : "+v"(a), "+v"(b));
    float c = fmaxf(a, b), d = c;
    asm volatile("s_nop 1\n\tv_permlane16_swap_b32 %0, %1" : "+v"(c), "+v"(d));
    return fmaxf(c, d);
}

// Order of the alternatives: by value (a NaN above all, -0 as 0), then by the
// lowest index; as one integer, larger first, never 0 and never all ones.
__device__ __forceinline__ uint64_t order_key(float v, uint32_t index) {
    const float z = v + 0.f;
    uint32_t u = __builtin_bit_cast(uint32_t, z);
    u = z != z ? 0xFFFFFFFEu : (u >> 31 ? ~u : u | 0x80000000u);
    return (uint64_t)u << 32 | (uint32_t)~index;
}
__device__ __forceinline__ float key_value(uint64_t key) {
    const uint32_t u = (uint32_t)(key >> 32);
    return bits_f(u >> 31 ? u & 0x7FFFFFFFu : ~u);
}
__device__ __forceinline__ uint32_t key_index(uint64_t key) { return ~(uint32_t)key; }
__device__ __forceinline__ uint64_t lane_key(uint64_t v, int lane) {
    const uint32_t lo = __builtin_amdgcn_readlane((int)(uint32_t)v, lane);
    const uint32_t hi = __builtin_amdgcn_readlane((int)(uint32_t)(v >> 32), lane);
    return (uint64_t)hi << 32 | lo;
}
__device__ __forceinline__ uint32_t wave_max_u32(uint32_t v) {
    const auto dpp = [](auto ctrl, uint32_t x) { return (uint32_t)__builtin_amdgcn_mov_dpp((int)x, decltype(ctrl)::value, 0xF, 0xF, false); };
    const auto pick = [](uint32_t x, uint32_t y) { return x < y ? y : x; };
    v = pick(v, dpp(std::integral_constant<int, 0xB1>{}, v));
    v = pick(v, dpp(std::integral_constant<int, 0x4E>{}, v));
    v = pick(v, dpp(std::integral_constant<int, 0x141>{}, v));
    v = pick(v, dpp(std::integral_constant<int, 0x140>{}, v));
    uint32_t a = v, b = v;
    asm volatile("s_nop 1\n\tv_permlane32_swap_b32 %0, %1" : "+v"(a), "+v"(b));
    uint32_t c = pick(a, b), d = c;
    asm volatile("s_nop 1\n\tv_permlane16_swap_b32 %0, %1" : "+v"(c), "+v"(d));
    return pick(c, d);
}
__device__ __forceinline__ uint64_t wave_max64(uint64_t v) {
    const uint32_t hi = wave_max_u32((uint32_t)(v >> 32));
    const uint32_t lo = wave_max_u32((uint32_t)(v >> 32) == hi ? (uint32_t)v : 0);
    return (uint64_t)hi << 32 | lo;
}

// Distances from the maximum in units of log 2, l log2(e) - m2, one instruction
// each: m2 is m log2(e) rounded, off by `off`, which shifts every exponent of the
// row alike and is taken out of the sums (exp2(l log2(e) - m2) = 2^off exp(l - m)).
// A row whose maximum is past 2^20 (where `off` could be any size), infinite or
// NaN is `steep`: it takes l - m itself, element by element from memory.
struct Scale {
    float m, m2, off;
    bool steep;
    __device__ __forceinline__ explicit Scale(float max) : m(max), m2(max * kLog2e), off(__builtin_fmaf(max, kLog2e, -m2)) {
        steep = !(fabsf(max) < 1048576.f);
        if (steep) off = 0.f;
    }
    __device__ __forceinline__ float of(float l) const { return __builtin_fmaf(l, kLog2e, -m2); }
};

// What a row's gradient needs: dl_j = p_j (f + h log p_j) + [j = t] a.
struct RowGrad {
    float m, ls, f, h, a;
    int64_t t;
    bool zero;
};
// What a row's results need beside its logits, asked for ahead of them: the
// target, its logit, the row's weights.
struct RowIn {
    int64_t t;
    float at_t, dlogprob, dentropy, dlse;
    bool has;
};
template <typename T>
__device__ __forceinline__ RowIn row_in(int64_t r, const LogprobArgs& a, const LogprobGrad* g) {
    RowIn o{-1, 0.f, 0.f, 0.f, 0.f, false};
    if (a.targets) {
        o.t = a.targets[r];
        o.has = o.t != a.ignore_index;
        if (a.logprob && o.has && o.t >= 0 && o.t < a.vocab) o.at_t = to_f(((const T*)a.logits)[r * a.stride + o.t]);
    }
    if (g) {
        if (g->dlogprob) o.dlogprob = g->dlogprob[r];
        if (g->dentropy) o.dentropy = g->dentropy[r];
        if (g->dlse) o.dlse = g->dlse[r];
    }
    return o;
}
__device__ __forceinline__ RowGrad row_grad(const RowIn& in, int64_t vocab, float m, float ls, float ent) {
    RowGrad o;
    o.t = in.has ? in.t : -1;
    o.a = in.has ? in.dlogprob : 0.f;
    if (in.has && (in.t < 0 || in.t >= vocab)) o.a = __builtin_nanf("");
    o.f = in.dlse - o.a - (in.dentropy != 0.f ? in.dentropy * ent : 0.f);
    o.h = -in.dentropy;
    const bool none = m == -INFINITY;  // nothing but -infinity
    o.m = none ? 0.f : m;
    o.ls = none ? 0.f : ls;
    o.zero = o.a == 0.f && o.f == 0.f && o.h == 0.f;
    return o;
}
__device__ __forceinline__ float grad_of(const RowGrad& g, float l) {
    const float q = (l - g.m) - g.ls, p = exp_f(q);
    return p * (g.f + g.h * fmaxf(q, kFar));
}
// The same in a Scale's units, e (a + b d) with d its distance and e = exp2(d):
// with s' the sum of the e, p = e / s' and log p = d log 2 - log s'.
struct FastGrad {
    Scale sc;
    float a, b;
    __device__ __forceinline__ FastGrad(const RowGrad& g, const Scale& scale, float inv_s, float log_s)
        : sc(scale), a(inv_s * (g.f - g.h * log_s)), b(inv_s * g.h * kLn2) {}
    template <bool ENT>
    __device__ __forceinline__ float of(float l) const {
        const float d = sc.of(l), e = fast_exp2(d);
        return ENT ? e * __builtin_fmaf(fmaxf(d, kFar), b, a) : e * a;
    }
};
// The gradients of a vector at element j of the row, with the target's own term.
template <bool ENT, int N>
__device__ __forceinline__ void grads_of(const FastGrad& f, const RowGrad& g, int64_t j, float (&v)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = f.of<ENT>(v[i]);
    const int64_t hot = g.t - j;
    if (hot >= 0 && hot < N) {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] += i == hot ? g.a : 0.f;
    }
}

// A vector's elements, stored at any alignment of an element.
__device__ __forceinline__ void store_any(bf16* p, const float (&v)[8]) {
    typedef u32x4 mem __attribute__((aligned(2)));
    bf16x8 r;
#pragma unroll
    for (int i = 0; i < 8; ++i) r[i] = (bf16)v[i];
    *reinterpret_cast<mem*>(p) = __builtin_bit_cast(u32x4, r);
}
template <int N>
__device__ __forceinline__ void store_any(float* p, const float (&v)[N]) {
    typedef f32x4 mem __attribute__((aligned(4)));
#pragma unroll
    for (int i = 0; i < N; i += 4) *reinterpret_cast<mem*>(p + i) = f32x4{v[i], v[i + 1], v[i + 2], v[i + 3]};
}

// A stretch of a row cut at boundaries of ALIGN bytes: `nv` whole vectors from
// element `head`, and head + tail single elements around them, one per thread.  16
// bytes for a wave's rows; 128 for a workgroup's, so that its waves' accesses cover
// whole lines (16384 rows of 50257 bf16, forward and gradient: 733 us, 696 so).  A
// stretch of 2 ALIGN bytes or more has a whole vector.
constexpr int align_for(int tpr) { return tpr >= 256 ? 128 : 16; }
template <typename T, int ALIGN>
struct Cut {
    const T* p;
    int64_t n;
    int head, edges;
    int nv;
    __device__ __forceinline__ Cut(const T* q, int64_t len, bool single = false) : p(q), n(len) {
        if (single) {
            head = edges = (int)len;
            nv = 0;
            return;
        }
        const int h = (int)(((ALIGN - (uintptr_t)q % ALIGN) % ALIGN) / sizeof(T));
        head = h < len ? h : (int)len;
        nv = (int)((len - head) / kVec<T>);
        edges = (int)(len - (int64_t)nv * kVec<T>);
    }
    __device__ __forceinline__ int64_t at(int v) const { return head + (int64_t)v * kVec<T>; }          // of vector v
    __device__ __forceinline__ int64_t edge(int e) const { return e < head ? e : (int64_t)nv * kVec<T> + e; }
    __device__ __forceinline__ u32x4 load(int v) const {
        return __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p + at(v)));
    }
};

// The k largest of the keys of a workgroup's threads.  Every thread gives the
// largest of its own; of the largest of each lane (over the waves) the k-th
// bounds the k-th of all from below, so that a look at each thread's keys again
// leaves few, which are put in order by counting.  Where more are left than there
// is room for (most of the best in few threads), k rounds over all keys find the
// largest below the last.
constexpr int kRoom = 512;
template <int TPR>
struct TopShared {
    uint64_t own[TPR / 64][64];
    uint64_t room[kRoom];
    uint64_t bound, best[TPR / 64];
    int count;
};
template <int TPR>
struct StatShared {
    float m[TPR / 64], s[TPR / 64], c[TPR / 64];
};

template <int TPR, bool TOP> struct RowShared {
    StatShared<TPR> st;
    TopShared<TPR> top;
};
template <int TPR> struct RowShared<TPR, false> {
    StatShared<TPR> st;
};
template <int TPR, bool TOP>
struct Top {
    __device__ __forceinline__ Top(RowShared<TPR, false>&, int) {}
};
template <int TPR>
struct Top<TPR, true> {
    TopShared<TPR>& s;
    int k;
    uint64_t mine;
    __device__ __forceinline__ Top(RowShared<TPR, true>& sh, int n) : s(sh.top), k(n), mine(0) {}

    // A barrier has to follow each of give, bound and push.
    __device__ __forceinline__ void give(uint64_t key) {
        mine = key;
        s.own[threadIdx.x >> 6][threadIdx.x & 63] = key;
        if (threadIdx.x == 0) {
            s.bound = 1;
            s.count = 0;
        }
    }
    // (by one wave, another for the next row: the first waves of a CU's workgroups
    // may share a SIMD)
    __device__ __forceinline__ void bound(int by) {
        if ((int)(threadIdx.x >> 6) != by) return;
        const int lane = threadIdx.x & 63;
        uint64_t c = 0;
#pragma unroll
        for (int w = 0; w < TPR / 64; ++w) c = s.own[w][lane] > c ? s.own[w][lane] : c;
        uint64_t kth = 0;
        if (k <= 8) {  // the largest k times: 40 instructions each, against 400 to count
            for (int i = 0; i < k; ++i) {
                kth = wave_max64(c);
                if (c == kth) c = 0;
            }
        } else {
            int above = 0;
#pragma unroll 8
            for (int j = 0; j < 64; ++j) above += lane_key(c, j) > c;
            if (above == k - 1) kth = c;
        }
        if (kth > 0) s.bound = kth;
    }
    __device__ __forceinline__ void push(uint64_t key) {
        const int at = atomicAdd(&s.count, 1);
        if (at < kRoom) s.room[at] = key;
    }
    // emit(place, key) of the k largest; each(f) calls f on every key of the thread.
    template <typename Emit, typename Each>
    __device__ __forceinline__ void finish(int by, bool pushed, const Emit& emit, const Each& each) {
        const int n = pushed ? s.count : kRoom + 1;
        if (n <= 64) {
            if ((int)(threadIdx.x >> 6) == by) {
                const int lane = threadIdx.x & 63;
                const uint64_t c = lane < n ? s.room[lane] : 0;
                int above = 0;
                for (int j = 0; j < n; ++j) above += lane_key(c, j) > c;
                if (lane < n && above < k) emit(above, c);
            }
        } else if (n <= kRoom) {
            for (int i = threadIdx.x; i < n; i += TPR) {
                const uint64_t c = s.room[i];
                int above = 0;
                for (int j = 0; j < n; ++j) above += s.room[j] > c;
                if (above < k) emit(above, c);
            }
        } else {
            uint64_t last = ~0ull;
            for (int i = 0; i < k; ++i) {
                uint64_t b = 0;
                each([&](uint64_t key) { b = key > b && key < last ? key : b; });
                b = wave_max64(b);
                __syncthreads();
                if ((threadIdx.x & 63) == 0) s.best[threadIdx.x >> 6] = b;
                __syncthreads();
#pragma unroll
                for (int w = 0; w < TPR / 64; ++w) b = s.best[w] > b ? s.best[w] : b;
                if (threadIdx.x == 0) emit(i, b);
                last = b;
            }
        }
    }
};

// Statistics of a segment.
struct Part {
    float m, s, c, pad;
};

// The row's results but the alternatives, by one thread.
struct RowStat {
    float m, ls;  // 0 in a row of nothing but -infinity
};
__device__ __forceinline__ RowStat put_row(const LogprobArgs& a, int64_t r, const RowIn& in, float m, float s, float c, bool write, float& ent) {
    const bool none = s == 0.f;
    const float ls = none ? -INFINITY : logf(s);
    ent = none ? 0.f : ls - c / s;
    const RowStat o{none ? 0.f : m, none ? 0.f : ls};
    if (write) {
        if (a.row_max) a.row_max[r] = none ? -INFINITY : m;
        if (a.log_sum) a.log_sum[r] = ls;
        if (a.entropy) a.entropy[r] = ent;
        if (a.logprob) a.logprob[r] = !in.has ? 0.f : in.t < 0 || in.t >= a.vocab ? __builtin_nanf("") : (in.at_t - o.m) - o.ls;
    }
    return o;
}

struct SegArgs {
    int nseg;
    int64_t len;    // elements of a segment
    Part* part;     // [rows][nseg]
    uint64_t* top;  // [rows][k][nseg], a segment's largest first; 0 past its elements
};

// The gradients of a steep row's vectors `from`, from + TPR, ... below `to`, and of
// an edge element.
template <typename T, typename GT, int TPR>
__device__ __forceinline__ void put_steep(const Cut<T, align_for(TPR)>& cut, GT* out, const RowGrad& g, int from, int to, bool has_edge) {
    constexpr int V = kVec<T>;
    for (int v = from; v < to; v += TPR) {
        float l[V];
        unpack(cut.load(v), l);
        const int64_t j = cut.at(v);
#pragma unroll
        for (int i = 0; i < V; ++i) l[i] = grad_of(g, l[i]) + (j + i == g.t ? g.a : 0.f);
        store_any(out + j, l);
    }
    if (has_edge) {
        const int64_t j = cut.edge(threadIdx.x % TPR);
        out[j] = from_f<GT>(grad_of(g, to_f(cut.p[j])) + (j == g.t ? g.a : 0.f));
    }
}

// Waves a SIMD is to hold (by the registers of NV packed vectors), and with them
// the workgroups of a CU: the grid of the whole-row kernels.  More of them hide the
// sums of one row behind the loads of others (16384 rows of 50257 bf16, 13 vectors: six
// 284 us, four 306; 65536 of 10000, 8 vectors: eight 332, five 359; with five
// alternatives and 4 vectors, 33554 rows of 4000 float: eight 120, seven 147; but with
// one and 13 vectors six, which spill, 401 and four 372).  At these the forward's whole
// rows spill nothing; with the gradient 2 registers of 8 vectors, 4 of 13 and 21 to 32
// of 16 are spilt, with alternatives as well 2 to 10 up to two vectors, 14 to 22 of 8 and 13, 36 of 16.
constexpr int waves_per_simd(int nv, bool grad, bool top) {
    return nv <= 2 || (!grad && nv <= (top ? 4 : 8)) ? 8 : nv <= 8 ? 5 : !grad && !top && nv <= 13 ? 6 : 4;
}

// One workgroup per row or segment at a time, NV vectors per thread.  GT = void:
// the forward; else the gradient too (whole rows).
template <typename T, typename GT, int TPR, int NV, bool SEG, bool TOP>
__global__ __launch_bounds__(TPR, waves_per_simd(NV, !std::is_void_v<GT>, TOP)) void k_token_logprobs(const LogprobArgs a, const LogprobGrad g, const SegArgs sg) {
    constexpr int V = kVec<T>;
    constexpr bool GRAD = !std::is_void_v<GT>;
    __shared__ RowShared<TPR, TOP> sh;
    const int tid = threadIdx.x, wave = tid >> 6;
    const int64_t items = a.rows * (SEG ? sg.nseg : 1), step = (int64_t)gridDim.x * gridDim.y;
    const auto cut_of = [&](int64_t item) {
        const int64_t r = SEG ? item / sg.nseg : item, e0 = SEG ? (item - r * sg.nseg) * sg.len : 0;
        return Cut<T, align_for(TPR)>((const T*)a.logits + r * a.stride + e0, SEG ? (a.vocab - e0 < sg.len ? a.vocab - e0 : sg.len) : a.vocab, NV == 0);
    };
    for (int64_t item = flat_block(); item < items; item += step) {
        const int64_t r = SEG ? item / sg.nseg : item;
        const uint32_t e0 = SEG ? (uint32_t)((item - r * sg.nseg) * sg.len) : 0;
        const auto cut = cut_of(item);
        const RowIn in = SEG ? RowIn{} : row_in<T>(r, a, GRAD ? &g : nullptr);
        u32x4 raw[NV > 0 ? NV : 1];
        // (past the row its last vector again: no branch keeps the loads apart)
#pragma unroll
        for (int q = 0; q < NV; ++q) raw[q] = cut.load(tid + q * TPR < cut.nv ? tid + q * TPR : cut.nv - 1);
        const bool has_edge = tid < cut.edges;
        const float edge = has_edge ? to_f(cut.p[cut.edge(tid)]) : -INFINITY;

        // the maximum, and which vector of the thread has it first
        float best = -INFINITY;
        int bq = 0;
#pragma unroll
        for (int q = 0; q < NV; ++q) {
            if (tid + q * TPR >= cut.nv) raw[q] = all_ninf<T>();
            float v[V];
            unpack(again(raw[q]), v);
            const float m = max_of(v);
            if (m > best) {
                best = m;
                bq = q;
            }
        }
        Top<TPR, TOP> top(sh, a.top_k);
        const int by = (int)((uint64_t)item % (TPR / 64));
        const auto edge_key = [&] { return has_edge ? order_key(edge, e0 + (uint32_t)cut.edge(tid)) : 0; };
        if constexpr (TOP) {
            __syncthreads();  // (the row before is done with the shared memory)
            const uint64_t kv = tid < cut.nv ? order_key(best, e0 + (uint32_t)cut.at(tid + bq * TPR)) : 0, ke = edge_key();
            top.give(kv > ke ? kv : ke);
        }
        float m = wave_max(fmaxf(fmaxf(best, edge), kLowest));
        if constexpr (TPR > 64) {
            if ((tid & 63) == 0) sh.st.m[wave] = m;
        }
        __syncthreads();
        if constexpr (TPR > 64) {
#pragma unroll
            for (int w = 0; w < TPR / 64; ++w) m = fmaxf(m, sh.st.m[w]);
        }
        if constexpr (TOP) {
            top.bound(by);  // (the other waves go on)
        }
        const Scale scale(m);
        float s = 0.f, c = 0.f;
        if (!scale.steep) {
#pragma unroll
            for (int q = 0; q < NV; ++q) {
                float v[V];
                unpack(again(raw[q]), v);
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const float d = scale.of(v[i]), e = fast_exp2(d);
                    s += e;
                    c += e * fmaxf(d, kFar);  // (the maximum drops a NaN, e keeps it)
                }
            }
            const float d = scale.of(edge), e = fast_exp2(d);
            s += e;
            c += e * fmaxf(d, kFar);
        } else {
            const auto add = [&](float l) {
                const float d = l - m, e = exp_f(d);
                s += e;
                c += e * fmaxf(d * kLog2e, kFar);
            };
            for (int v = tid; v < cut.nv; v += TPR) {
                float l[V];
                unpack(cut.load(v), l);
#pragma unroll
                for (int i = 0; i < V; ++i) add(l[i]);
            }
            if (has_edge) add(edge);
        }
        s = wave_sum(s);
        c = wave_sum(c);
        if constexpr (TPR > 64) {
            if ((tid & 63) == 0) {
                sh.st.s[wave] = s;
                sh.st.c[wave] = c;
            }
            __syncthreads();
            s = c = 0.f;
#pragma unroll
            for (int w = 0; w < TPR / 64; ++w) {
                s += sh.st.s[w];
                c += sh.st.c[w];
            }
        } else if constexpr (TOP) {
            __syncthreads();  // (the bound; the waves' sums give larger workgroups theirs)
        }
        const float scaled_sum = s;
        {
            const float unit = fast_exp2(-scale.off);
            c = (c - s * scale.off) * (unit * kLn2);
            s *= unit;
        }
        float ent = 0.f;
        RowStat row{m, 0.f};
        if constexpr (SEG) {
            if (tid == 0) sg.part[item] = Part{m, s, c, 0.f};
        } else {
            row = put_row(a, r, in, m, s, c, tid == 0, ent);
        }

        if constexpr (TOP) {
            const bool orderly = s == s;  // a NaN has no place among the floats compared
            const auto emit = [&](int at, uint64_t key) {
                if constexpr (SEG) {
                    if (at < cut.n) sg.top[(r * a.top_k + at) * sg.nseg + (item - r * sg.nseg)] = key;
                } else {
                    a.top_ids[r * a.top_k + at] = key_index(key);
                    a.top_logprobs[r * a.top_k + at] = (key_value(key) - row.m) - row.ls;
                }
            };
            const auto each = [&](auto f) {
                for (int v = tid; v < cut.nv; v += TPR) {
                    float l[V];
                    unpack(cut.load(v), l);
#pragma unroll
                    for (int i = 0; i < V; ++i) f(order_key(l[i], e0 + (uint32_t)cut.at(v) + i));
                }
                if (has_edge) f(edge_key());
            };
            const uint64_t bound = sh.top.bound;
            if (orderly && top.mine >= bound) {
                const float bv = bound > 1 ? key_value(bound) : -INFINITY;
                uint32_t look = 0;  // vectors that may hold some of the best
#pragma unroll
                for (int q = 0; q < NV; ++q) {
                    float v[V];
                    unpack(again(raw[q]), v);
                    look |= max_of(v) >= bv && tid + q * TPR < cut.nv ? 1u << q : 0;
                }
                for (; look; look &= look - 1) {
                    const int w = __ffs(look) - 1;
                    u32x4 one = raw[0];
#pragma unroll
                    for (int q = 1; q < NV; ++q) one = w == q ? raw[q] : one;
                    float v[V];
                    unpack(one, v);
                    const uint32_t j = e0 + (uint32_t)cut.at(tid + w * TPR);
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        // (by the vector's first index, as the bound: none of the best is lost)
                        if (v[i] >= bv && order_key(v[i], j) >= bound) top.push(order_key(v[i], j + i));
                    }
                }
                const uint64_t ke = edge_key();
                if (ke >= bound) top.push(ke);
            }
            __syncthreads();
            if constexpr (SEG) {
                if (tid >= cut.n && tid < a.top_k) sg.top[(r * a.top_k + tid) * sg.nseg + (item - r * sg.nseg)] = 0;
            }
            top.finish(by, orderly, emit, each);
        }

        if constexpr (GRAD) {
            const RowGrad rg = row_grad(in, a.vocab, s == 0.f ? -INFINITY : m, row.ls, ent);
            GT* out = (GT*)g.dlogits + r * g.stride;
            const FastGrad fast(rg, scale, 1.0f / scaled_sum, row.ls + scale.off * kLn2);
            const auto put = [&](auto with_entropy) {
                constexpr bool ENT = decltype(with_entropy)::value;
#pragma unroll
                for (int q = 0; q < NV; ++q) {
                    float v[V];
                    unpack(again(raw[q]), v);
                    const int64_t j = cut.at(tid + q * TPR);
                    grads_of<ENT>(fast, rg, j, v);
                    if (tid + q * TPR < cut.nv) store_any(out + j, v);
                }
                if (has_edge) {
                    const int64_t j = cut.edge(tid);
                    out[j] = from_f<GT>(fast.of<ENT>(edge) + (j == rg.t ? rg.a : 0.f));
                }
            };
            if (rg.zero) {
                const float z[V] = {};
#pragma unroll
                for (int q = 0; q < NV; ++q) {
                    if (tid + q * TPR < cut.nv) store_any(out + cut.at(tid + q * TPR), z);
                }
                if (has_edge) out[cut.edge(tid)] = from_f<GT>(0.f);
            } else if (scale.steep) {
                put_steep<T, GT, TPR>(cut, out, rg, tid, cut.nv, has_edge);
            } else if (rg.h != 0.f) {
                put(std::true_type{});
            } else {
                put(std::false_type{});
            }
        }
    }
}

// One workgroup per row: the segments' statistics and alternatives joined.
template <typename T, bool TOP>
__global__ __launch_bounds__(256) void k_token_logprobs_join(const LogprobArgs a, const SegArgs sg) {
    __shared__ RowShared<256, TOP> sh;
    const int64_t r = flat_block();
    if (r >= a.rows) return;
    const int tid = threadIdx.x, wave = tid >> 6;
    const Part* part = sg.part + r * sg.nseg;
    const RowIn in = row_in<T>(r, a, nullptr);
    // candidates in the order of their places, so that the segments' first ones spread
    // over the lanes; a thread keeps its first four
    const int n = sg.nseg * a.top_k;
    const uint64_t* cand = sg.top + r * n;
    uint64_t kept[4] = {};
    if constexpr (TOP) {
#pragma unroll
        for (int i = 0; i < 4; ++i) kept[i] = tid + 256 * i < n ? cand[tid + 256 * i] : 0;
    }
    const auto each = [&](auto f) {
#pragma unroll
        for (int i = 0; i < 4; ++i) f(kept[i]);
        for (int i = tid + 1024; i < n; i += 256) f(cand[i]);
    };
    Top<256, TOP> top(sh, a.top_k);
    if constexpr (TOP) {
        uint64_t b = 0;
        each([&](uint64_t key) { b = key > b ? key : b; });
        top.give(b);
    }
    float m = kLowest;
    for (int i = tid; i < sg.nseg; i += 256) m = fmaxf(m, part[i].m);
    m = wave_max(m);
    if ((tid & 63) == 0) sh.st.m[wave] = m;
    __syncthreads();
    m = fmaxf(fmaxf(sh.st.m[0], sh.st.m[1]), fmaxf(sh.st.m[2], sh.st.m[3]));
    if constexpr (TOP) top.bound(0);
    float s = 0.f, c = 0.f;
    for (int i = tid; i < sg.nseg; i += 256) {
        const Part p = part[i];
        const float d = fmaxf(p.m - m, kFar), f = exp_f(d);
        s += f * p.s;
        c += f * (p.c + p.s * d);
    }
    s = wave_sum(s);
    c = wave_sum(c);
    if ((tid & 63) == 0) {
        sh.st.s[wave] = s;
        sh.st.c[wave] = c;
    }
    __syncthreads();
    s = sh.st.s[0] + sh.st.s[1] + sh.st.s[2] + sh.st.s[3];
    c = sh.st.c[0] + sh.st.c[1] + sh.st.c[2] + sh.st.c[3];
    float ent;
    const RowStat row = put_row(a, r, in, m, s, c, tid == 0, ent);
    if constexpr (TOP) {
        const uint64_t bound = sh.top.bound;
        if (top.mine >= bound) each([&](uint64_t key) { if (key >= bound) top.push(key); });
        __syncthreads();
        top.finish(0, true, [&](int at, uint64_t key) {
            a.top_ids[r * a.top_k + at] = key_index(key);
            a.top_logprobs[r * a.top_k + at] = (key_value(key) - row.m) - row.ls;
        }, each);
    }
}

// The gradient alone: TPR lanes per stretch of TPR NV vectors of a row.
template <typename T, typename GT, int TPR, int NV>
__global__ __launch_bounds__(256) void k_token_logprobs_bwd(const LogprobArgs a, const LogprobGrad g, int stretches) {
    constexpr int V = kVec<T>, GR = 256 / TPR;
    const int tid = threadIdx.x % TPR;
    const int64_t items = a.rows * stretches, step = (int64_t)gridDim.x * gridDim.y * GR;
    int64_t item = flat_block() * GR + threadIdx.x / TPR;
    if constexpr (TPR == 64) item = flat_block() * GR + __builtin_amdgcn_readfirstlane((int)threadIdx.x / 64);
    for (; item < items; item += step) {
        const int64_t r = item / stretches;
        const int v0 = (int)(item - r * stretches) * (TPR * NV);
        const Cut<T, align_for(TPR)> cut((const T*)a.logits + r * a.stride, a.vocab);
        GT* out = (GT*)g.dlogits + r * g.stride;
        const RowGrad rg = row_grad(row_in<T>(r, a, &g), a.vocab, a.row_max[r], a.log_sum[r], g.dentropy ? a.entropy[r] : 0.f);
        const bool has_edge = v0 == 0 && tid < cut.edges;
        if (rg.zero) {
            const float z[V] = {};
#pragma unroll
            for (int q = 0; q < NV; ++q) {
                const int v = v0 + tid + q * TPR;
                if (v < cut.nv) store_any(out + cut.at(v), z);
            }
            if (has_edge) out[cut.edge(tid)] = from_f<GT>(0.f);
            continue;
        }
        const Scale scale(rg.m);
        if (scale.steep) {
            put_steep<T, GT, TPR>(cut, out, rg, v0 + tid, v0 + TPR * NV < cut.nv ? v0 + TPR * NV : cut.nv, has_edge);
            continue;
        }
        u32x4 raw[NV];
#pragma unroll
        for (int q = 0; q < NV; ++q) {
            const int v = v0 + tid + q * TPR;
            if (v < cut.nv) raw[q] = cut.load(v);
        }
        const float edge = has_edge ? to_f(cut.p[cut.edge(tid)]) : 0.f;
        // exp(-log s') with the product's rounding carried along: it would be the largest
        const float log_s = rg.ls + scale.off * kLn2, hi = rg.ls * kLog2e, lo = __builtin_fmaf(rg.ls, kLog2e, -hi) + scale.off;
        const FastGrad fast(rg, scale, fast_exp2(-hi) * fast_exp2(-lo), log_s);
        const auto put = [&](auto with_entropy) {
            constexpr bool ENT = decltype(with_entropy)::value;
#pragma unroll
            for (int q = 0; q < NV; ++q) {
                const int v = v0 + tid + q * TPR;
                if (v < cut.nv) {
                    float l[V];
                    unpack(raw[q], l);
                    const int64_t j = cut.at(v);
                    grads_of<ENT>(fast, rg, j, l);
                    store_any(out + j, l);
                }
            }
            if (has_edge) {
                const int64_t j = cut.edge(tid);
                out[j] = from_f<GT>(fast.of<ENT>(edge) + (j == rg.t ? rg.a : 0.f));
            }
        };
        if (rg.h != 0.f) put(std::true_type{});
        else put(std::false_type{});
    }
}

// How the forward cuts its rows: segments of `len`, `nseg` to a row (1: whole
// rows), in workgroups of `tpr` threads with `nv` vectors each.
struct Plan {
    int nseg, tpr, nv;
    int64_t len;
};
Plan plan_for(int64_t rows, int64_t vocab, int dtype, int top_k, bool grad) {
    const int vec = dtype == 1 ? 8 : 4;
    // (13 vectors, between 8 and 16: the most that six waves hold forward, and with few
    // spilt in the gradient; 12288 rows of 53248 bf16 in 13 and of 53256 in 16: forward
    // 231 and 274 us, with five alternatives 328 and 385, with the gradient 541 and 582)
    static const int forms[][2] = {{64, 0}, {64, 1}, {64, 2}, {64, 4}, {256, 2}, {256, 4}, {256, 8}, {512, 8}, {512, 13}, {512, 16}, {1024, 16}};
    const int64_t most = 1024 * 16 * vec;
    // long rows without alternatives or gradient in segments of 256 threads, if those
    // are nearly full: more of them are resident, and nothing waits for a whole row
    // (4096 rows of 131072 bf16 179 us, 6.0 TB/s, whole 242; of 50257 float 134 and 160;
    // but 8192 of 50257 bf16, 0.77 full, 241 and 190, and with five alternatives,
    // which every segment sorts, 4096 of 131072 322 and 286)
    const int64_t full = 256 * 8 * vec, parts = (vocab + full - 1) / full;
    if (!grad && top_k == 0 && parts > 1 && rows * parts >= 2 * device_cu_count() && 8 * vocab >= 7 * parts * full)
        return {(int)parts, 256, 8, (vocab + parts - 1) / parts};
    // whole rows where they fit and fill the card, or are short
    if (vocab <= 2048 || (vocab <= most && rows >= device_cu_count() / (grad ? 4 : 2))) {
        for (const auto& f : forms)
            if (f[1] ? vocab <= (int64_t)f[0] * f[1] * vec : vocab < 2 * vec) return {1, f[0], f[1], vocab};
    }
    // segments for a workgroup per CU, of two to eight vectors per thread
    int64_t want = (device_cu_count() + rows - 1) / rows;
    int nv = 8;
    while (nv > 2 && (vocab + 256 * nv * vec - 1) / (256 * nv * vec) < want) nv /= 2;
    // (even segments: the last one is shorter than the others by less than their
    // number, below 2^24 / 8192, and so never too short for a whole vector)
    const int64_t each = (int64_t)256 * nv * vec, nseg = (vocab + each - 1) / each;
    return {(int)nseg, 256, nv, (vocab + nseg - 1) / nseg};
}

template <typename T, typename GT, bool SEG, bool TOP>
void run_rows(const Plan& p, const LogprobArgs& a, const LogprobGrad& g, const SegArgs& sg, hipStream_t st) {
    const int64_t items = a.rows * p.nseg;
#define DART_ROW(TPR, NV)                                                                                        \
    if (p.tpr == TPR && p.nv == NV) {                                                                            \
        const int64_t cap = (int64_t)device_cu_count() * (waves_per_simd(NV, !std::is_void_v<GT>, TOP) * 256 / TPR); \
        k_token_logprobs<T, GT, TPR, NV, SEG, TOP><<<flat_grid(items < cap ? items : cap, TPR), TPR, 0, st>>>(a, g, sg); \
        return;                                                                                                  \
    }
    DART_ROW(256, 2)
    DART_ROW(256, 4)
    DART_ROW(256, 8)
    if constexpr (!SEG) {
        DART_ROW(64, 0)
        DART_ROW(64, 1)
        DART_ROW(64, 2)
        DART_ROW(64, 4)
        DART_ROW(512, 8)
        DART_ROW(512, 13)
        DART_ROW(512, 16)
        DART_ROW(1024, 16)
    }
#undef DART_ROW
}

template <typename T, typename GT>
void run_bwd(const LogprobArgs& a, const LogprobGrad& g, hipStream_t st) {
    const int64_t nv = (a.vocab + kVec<T> - 1) / kVec<T>;
#define DART_BWD(TPR, NV)                                                                              \
    {                                                                                                  \
        const int64_t n = (nv + TPR * NV - 1) / (TPR * NV), b = (a.rows * n * TPR + 255) / 256;        \
        k_token_logprobs_bwd<T, GT, TPR, NV><<<flat_grid(b, 256), 256, 0, st>>>(a, g, (int)n);         \
    }
    if (nv <= 64) DART_BWD(64, 1)
    else if (nv <= 256) DART_BWD(64, 4)
    else DART_BWD(256, 4)
#undef DART_BWD
}

}  // namespace

size_t token_logprobs_workspace_bytes(int64_t rows, int64_t vocab, int dtype, int top_k) {
    size_t need = 0;
    if (rows == 0) return need;
    for (const bool grad : {false, true}) {
        const Plan p = plan_for(rows, vocab, dtype, top_k, grad);
        if (p.nseg > 1) {
            const size_t n = (size_t)rows * p.nseg, b = align256(n * sizeof(Part)) + n * top_k * sizeof(uint64_t);
            need = b > need ? b : need;
        }
    }
    return need;
}

hipError_t launch_token_logprobs(const LogprobArgs& a, const LogprobGrad* grad, void* ws, hipStream_t st) {
    if (a.rows == 0) return hipSuccess;
    const Plan p = plan_for(a.rows, a.vocab, a.dtype, a.top_k, grad != nullptr);
    SegArgs sg{p.nseg, p.len, nullptr, nullptr};
    const LogprobGrad none{};
    if (p.nseg > 1) {
        sg.part = (Part*)ws;
        sg.top = (uint64_t*)((char*)ws + align256((size_t)a.rows * p.nseg * sizeof(Part)));
    }
    prof_begin("k_token_logprobs", st);
#define DART_RUN(T, GT, SEG, G)                                     \
    (a.top_k ? run_rows<T, GT, SEG, true>(p, a, G, sg, st) : run_rows<T, GT, SEG, false>(p, a, G, sg, st))
    if (p.nseg > 1) {
        if (a.dtype == 1) DART_RUN(bf16, void, true, none);
        else DART_RUN(float, void, true, none);
    } else if (!grad) {
        if (a.dtype == 1) DART_RUN(bf16, void, false, none);
        else DART_RUN(float, void, false, none);
    } else if (a.dtype == 0) {
        DART_RUN(float, float, false, *grad);
    } else if (grad->dtype == 0) {
        DART_RUN(bf16, float, false, *grad);
    } else {
        DART_RUN(bf16, bf16, false, *grad);
    }
#undef DART_RUN
    prof_end(st);
    if (p.nseg == 1) return hipGetLastError();
    const dim3 grid = flat_grid(a.rows, 256);
    prof_begin("k_token_logprobs_join", st);
    if (a.dtype == 1) {
        if (a.top_k) k_token_logprobs_join<bf16, true><<<grid, 256, 0, st>>>(a, sg);
        else k_token_logprobs_join<bf16, false><<<grid, 256, 0, st>>>(a, sg);
    } else {
        if (a.top_k) k_token_logprobs_join<float, true><<<grid, 256, 0, st>>>(a, sg);
        else k_token_logprobs_join<float, false><<<grid, 256, 0, st>>>(a, sg);
    }
    prof_end(st);
    return grad ? launch_token_logprobs_bwd(a, *grad, st) : hipGetLastError();
}

hipError_t launch_token_logprobs_bwd(const LogprobArgs& a, const LogprobGrad& g, hipStream_t st) {
    if (a.rows == 0) return hipSuccess;
    prof_begin("k_token_logprobs_bwd", st);
    if (a.dtype == 0) run_bwd<float, float>(a, g, st);
    else if (g.dtype == 0) run_bwd<bf16, float>(a, g, st);
    else run_bwd<bf16, bf16>(a, g, st);
    prof_end(st);
    return hipGetLastError();
}

}  // namespace dart
