// norm.hip -- layer norm of the residual stream (and its form without
// centring, the RMS norm of the language model), with the residual addition
// ahead of it, and its backward.  With s = x + residual as stored,
//   mu = mean(s) (0 without centring),  r = (mean((s - mu)^2) + eps)^-1/2,
//   out = (s - mu) r (.) w + b;
// backward, with xh = (s - mu) r and g = dout (.) w:
//   dx = r (g - mean(g) - xh mean(g xh)) + dsum   (mean(g) only if centred),
//   dw = sum_rows dout (.) xh,  db = sum_rows dout.
// The mean square is taken of the deviations, never as a difference of
// squares, which would lose what a large mean leaves.
//
// Both are bound by HBM: some ten operations per element against two to eight
// bytes.  A row stays in the registers of the TPR lanes that share it (16, a
// wave, four to sixteen waves, ITEMS vectors of V elements each), so every
// input is read once; the next row's loads are issued ahead of the present
// row's sums, and a lane keeps its columns' weights for all its rows.  In the
// backward it keeps their sums of dw and db too: one partial row per
// workgroup, added in a second launch in a fixed order.
// 16384 rows of 4096 bf16 with residual: forward 80 us, 6.7 TB/s, backward 91 us,
// 5.9 TB/s, and 4 us to add the partial rows; 32768 rows of 768: 35 and 38 us.
#include "dart_common.hpp"
#include "dart_internal.hpp"

#include <algorithm>

namespace dart {
namespace {

// V elements of T as they are loaded and stored: 16 bytes of the wider type of a
// kernel at any alignment of an element (a lane's 16 bytes are one access
// whether they lie on 16 or not), or single elements in rows shorter than that.
typedef unsigned int u32x2_nt __attribute__((ext_vector_type(2)));
template <typename T, int V> struct Raw;
template <> struct Raw<bf16, 8> { using type = u32x4_nt; typedef u32x4_nt mem __attribute__((aligned(2))); };
template <> struct Raw<bf16, 4> { using type = u32x2_nt; typedef u32x2_nt mem __attribute__((aligned(2))); };
template <> struct Raw<bf16, 1> { using type = uint32_t; typedef uint16_t mem; };
template <> struct Raw<float, 4> { using type = f32x4; typedef f32x4 mem __attribute__((aligned(4))); };
template <> struct Raw<float, 1> { using type = float; typedef float mem; };
template <typename T, int V> using RawT = typename Raw<T, V>::type;

template <typename T, int V>
__device__ __forceinline__ RawT<T, V> load_raw(const T* p) {
    return __builtin_nontemporal_load(reinterpret_cast<const typename Raw<T, V>::mem*>(p));
}
__device__ __forceinline__ float bits_f(uint32_t u) { return __builtin_bit_cast(float, u); }
__device__ __forceinline__ void unpack(u32x4_nt r, float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = bits_f(r[i] << 16);
        v[2 * i + 1] = bits_f(r[i] & 0xFFFF0000u);
    }
}
__device__ __forceinline__ void unpack(u32x2_nt r, float (&v)[4]) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        v[2 * i] = bits_f(r[i] << 16);
        v[2 * i + 1] = bits_f(r[i] & 0xFFFF0000u);
    }
}
__device__ __forceinline__ void unpack(uint32_t r, float (&v)[1]) { v[0] = bits_f(r << 16); }
__device__ __forceinline__ void unpack(f32x4 r, float (&v)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = r[i];
}
__device__ __forceinline__ void unpack(float r, float (&v)[1]) { v[0] = r; }
template <int V>
__device__ __forceinline__ void store_v(bf16* p, const float (&v)[V]) {
    if constexpr (V == 1) {
        *p = (bf16)v[0];
    } else {
        typedef bf16 vec __attribute__((ext_vector_type(V)));
        vec r;
#pragma unroll
        for (int i = 0; i < V; ++i) r[i] = (bf16)v[i];
        *reinterpret_cast<typename Raw<bf16, V>::mem*>(p) = __builtin_bit_cast(RawT<bf16, V>, r);
    }
}
template <int V>
__device__ __forceinline__ void store_v(float* p, const float (&v)[V]) {
    if constexpr (V == 1) *p = v[0];
    else *reinterpret_cast<Raw<float, 4>::mem*>(p) = f32x4{v[0], v[1], v[2], v[3]};
}

// Which elements of its vector q a lane owns.  In rows that are no multiple of
// V elements (RAGGED) the last vector is moved back to end with the row; what
// it shares with the one before belongs to that one (both store the same).
template <int V, int TPR, int ITEMS, bool RAGGED>
struct Columns {
    int first[ITEMS];  // first column; lanes past the row repeat its last vector
    int skip[ITEMS];   // elements that are not the lane's own, from the front
    __device__ __forceinline__ Columns(int lane, int D) {
#pragma unroll
        for (int q = 0; q < ITEMS; ++q) {
            const int c = (lane + q * TPR) * V;
            first[q] = c <= D - V ? c : D - V;
            skip[q] = c < D ? c - first[q] : V;
        }
    }
    __device__ __forceinline__ bool any(int q) const { return skip[q] < V; }
    __device__ __forceinline__ bool own(int q, int i) const { return RAGGED ? i >= skip[q] : skip[q] == 0; }
};

// Sums of N values over the TPR lanes of a row, in every one of them.  Rows of
// several waves meet in LDS; `turn` alternates its halves, so that one barrier
// per exchange keeps a write from the reads two exchanges before.
template <int N, int TPR>
struct RowSum {
    static constexpr int kWaves = TPR / 64;
    float (*s)[2][kWaves > 0 ? kWaves : 1];
    int turn;
    template <int M>
    __device__ __forceinline__ void operator()(float (&v)[M]) {
        static_assert(M <= N, "room for the exchange");
#pragma unroll
        for (int k = 0; k < M; ++k) {
#pragma unroll
            for (int o = (TPR < 64 ? TPR : 64) / 2; o >= 1; o >>= 1) v[k] += __shfl_xor(v[k], o, 64);
        }
        if constexpr (TPR > 64) {
            if ((threadIdx.x & 63) == 0) {
#pragma unroll
                for (int k = 0; k < M; ++k) s[k][turn][threadIdx.x >> 6] = v[k];
            }
            __syncthreads();
#pragma unroll
            for (int k = 0; k < M; ++k) {
                v[k] = 0.f;
#pragma unroll
                for (int i = 0; i < kWaves; ++i) v[k] += s[k][turn][i];
            }
            turn ^= 1;
        }
    }
};

// sum / d with inv_d the nearest to 1 / d: the product corrected once by its remainder
// (the step of a division after Markstein), which is the quotient itself where that is a
// float.  The product alone is off by a step or so of a mean that every deviation is
// taken from: in a row of 300 in 4095 columns 3e-5 of deviation where there is none.
__device__ __forceinline__ float mean_of(float sum, int d, float inv_d) {
    const float q = sum * inv_d;
    return __builtin_fmaf(__builtin_fmaf(-q, (float)d, sum), inv_d, q);
}

constexpr int block_threads(int tpr) { return tpr > 256 ? tpr : 256; }

// The row of a workgroup's rows at a time that a lane works on, as a scalar where
// its whole wave shares it.
template <int TPR>
__device__ __forceinline__ int row_group() {
    if constexpr (TPR >= 256) return 0;
    else if constexpr (TPR == 64) return __builtin_amdgcn_readfirstlane((int)threadIdx.x / 64);
    else return (int)threadIdx.x / TPR;
}

// Weights of V columns, or `none` where there are none.  A lane keeps those of its
// columns for all its rows, except where 1024 lanes leave it 128 registers and
// more than 8 elements each: it loads them again for every row there, and loads
// no row ahead.
constexpr bool keeps_weights(int tpr, int e) { return tpr < 1024 || e <= 8; }
template <int V>
__device__ __forceinline__ void load_cols(const float* w, int c, float none, float (&v)[V]) {
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = w ? w[c + i] : none;
}

struct NormArgs {
    const void *x, *res;
    int64_t xs, rs, rows;
    const float *w, *b;
    float eps, inv_d;
    void *out, *sum;
    int D, center;
};

template <typename T, int V, int TPR, int ITEMS, bool RAGGED>
__global__ __launch_bounds__(block_threads(TPR)) void k_layernorm(const NormArgs a) {
    constexpr int GR = block_threads(TPR) / TPR;  // rows at a time
    __shared__ float s_sum[1][2][TPR > 64 ? TPR / 64 : 1];
    const int lane = threadIdx.x % TPR, group = row_group<TPR>();
    const T* x = (const T*)a.x;
    const T* res = (const T*)a.res;
    RowSum<1, TPR> row_sum{s_sum, 0};
    constexpr bool keep = keeps_weights(TPR, ITEMS * V), ahead = keep;
    float wv[keep ? ITEMS : 1][V], bv[keep ? ITEMS : 1][V];
    const Columns<V, TPR, ITEMS, RAGGED> cols(lane, a.D);
#pragma unroll
    for (int q = 0; q < ITEMS; ++q) {
        if constexpr (keep) {
            load_cols(a.w, cols.first[q], 1.f, wv[q]);
            load_cols(a.b, cols.first[q], 0.f, bv[q]);
        }
    }
    RawT<T, V> xr[ITEMS] = {}, rr[ITEMS] = {};
    const auto load = [&](int64_t r) {
        const int64_t rc = r < a.rows ? r : a.rows - 1;
#pragma unroll
        for (int q = 0; q < ITEMS; ++q) {
            xr[q] = load_raw<T, V>(x + rc * a.xs + cols.first[q]);
            if (res) rr[q] = load_raw<T, V>(res + rc * a.rs + cols.first[q]);
        }
    };
    const int64_t step = (int64_t)gridDim.x * GR;
    int64_t base = (int64_t)blockIdx.x * GR;
    if constexpr (ahead) load(base + group);
    for (; base < a.rows; base += step) {
        const int64_t r = base + group;
        if constexpr (!ahead) load(r);
        float v[ITEMS][V], m[1] = {0.f};
#pragma unroll
        for (int q = 0; q < ITEMS; ++q) {
            unpack(xr[q], v[q]);
            if (res) {
                float u[V];
                unpack(rr[q], u);
#pragma unroll
                for (int i = 0; i < V; ++i) v[q][i] = to_f(from_f<T>(v[q][i] + u[i]));
            }
#pragma unroll
            for (int i = 0; i < V; ++i) m[0] += cols.own(q, i) ? v[q][i] : 0.f;
        }
        if constexpr (ahead) load(r + step);
        float mu = 0.f, ss[1] = {0.f};
        if (a.center) {
            row_sum(m);
            mu = mean_of(m[0], a.D, a.inv_d);
        }
#pragma unroll
        for (int q = 0; q < ITEMS; ++q) {
#pragma unroll
            for (int i = 0; i < V; ++i) ss[0] += cols.own(q, i) ? (v[q][i] - mu) * (v[q][i] - mu) : 0.f;
        }
        row_sum(ss);
        const float inv = 1.0f / sqrtf(ss[0] * a.inv_d + a.eps);
#pragma unroll
        for (int q = 0; q < ITEMS; ++q) {
            if (cols.any(q) && r < a.rows) {
                const int64_t at = r * a.D + cols.first[q];
                if constexpr (!keep) {
                    load_cols(a.w, cols.first[q], 1.f, wv[0]);
                    load_cols(a.b, cols.first[q], 0.f, bv[0]);
                }
                if (a.sum) store_v((T*)a.sum + at, v[q]);
                float o[V];
#pragma unroll
                for (int i = 0; i < V; ++i) o[i] = (v[q][i] - mu) * inv * wv[keep ? q : 0][i] + bv[keep ? q : 0][i];
                store_v((T*)a.out + at, o);
            }
        }
    }
}

struct NormBwdArgs {
    const void* x;
    int64_t xs, rows;
    const float* w;
    float eps, inv_d;
    const void *dout, *dsum;
    void* dx;
    float* part;  // [blocks][2][D]
    int D, center;
};

template <typename T, typename GT, int V, int TPR, int ITEMS, bool RAGGED>
__global__ __launch_bounds__(block_threads(TPR)) void k_layernorm_bwd(const NormBwdArgs a) {
    constexpr int GR = block_threads(TPR) / TPR;
    constexpr int W = TPR * ITEMS * V;  // columns, with those past the row
    __shared__ float s_sum[3][2][TPR > 64 ? TPR / 64 : 1];
    constexpr bool keep = keeps_weights(TPR, ITEMS * V), ahead = keep;
    // the column sums of the groups but the first; of rows whose weights are not
    // kept all of them, from the start
    __shared__ float s_col[!keep ? 2 * W : GR > 1 ? (GR - 1) * W : 1];
    const int lane = threadIdx.x % TPR, group = row_group<TPR>();
    const T* x = (const T*)a.x;
    const GT* dout = (const GT*)a.dout;
    const GT* dsum = (const GT*)a.dsum;
    RowSum<3, TPR> row_sum{s_sum, 0};
    float wv[keep ? ITEMS : 1][V], aw[keep ? ITEMS : 1][V], ab[keep ? ITEMS : 1][V];
    const auto slot = [&](int q, int i) { return (i * ITEMS + q) * TPR + lane; };
    const Columns<V, TPR, ITEMS, RAGGED> cols(lane, a.D);
#pragma unroll
    for (int q = 0; q < ITEMS; ++q) {
        if constexpr (keep) load_cols(a.w, cols.first[q], 1.f, wv[q]);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            if constexpr (keep) aw[q][i] = ab[q][i] = 0.f;
            else s_col[slot(q, i)] = s_col[W + slot(q, i)] = 0.f;
        }
    }
    RawT<T, V> xr[ITEMS] = {};
    RawT<GT, V> dr[ITEMS] = {}, sr[ITEMS] = {};
    const auto load = [&](int64_t r) {
        const int64_t rc = r < a.rows ? r : a.rows - 1;
#pragma unroll
        for (int q = 0; q < ITEMS; ++q) {
            xr[q] = load_raw<T, V>(x + rc * a.xs + cols.first[q]);
            dr[q] = load_raw<GT, V>(dout + rc * a.D + cols.first[q]);
            if (dsum) sr[q] = load_raw<GT, V>(dsum + rc * a.D + cols.first[q]);
        }
    };
    const int64_t step = (int64_t)gridDim.x * GR;
    int64_t base = (int64_t)blockIdx.x * GR;
    if constexpr (ahead) load(base + group);
    for (; base < a.rows; base += step) {
        const int64_t r = base + group;
        if constexpr (!ahead) load(r);
        float v[ITEMS][V], m[1] = {0.f};
        // (the gradients stay packed: a row of theirs in float would cost resident waves)
        RawT<GT, V> dc[ITEMS], sc[ITEMS];
#pragma unroll
        for (int q = 0; q < ITEMS; ++q) {
            unpack(xr[q], v[q]);
            dc[q] = dr[q];
            sc[q] = sr[q];
#pragma unroll
            for (int i = 0; i < V; ++i) m[0] += cols.own(q, i) ? v[q][i] : 0.f;
        }
        if constexpr (ahead) load(r + step);
        if (a.center) {
            row_sum(m);
            const float mu = mean_of(m[0], a.D, a.inv_d);
#pragma unroll
            for (int q = 0; q < ITEMS; ++q) {
#pragma unroll
                for (int i = 0; i < V; ++i) v[q][i] -= mu;
            }
        }
        float t[3] = {0.f, 0.f, 0.f};
#pragma unroll
        for (int q = 0; q < ITEMS; ++q) {
            float d[V];
            unpack(dc[q], d);
            if constexpr (!keep) load_cols(a.w, cols.first[q], 1.f, wv[0]);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float g = d[i] * wv[keep ? q : 0][i];
                t[0] += cols.own(q, i) ? v[q][i] * v[q][i] : 0.f;
                t[1] += cols.own(q, i) ? g * v[q][i] : 0.f;
                t[2] += cols.own(q, i) ? g : 0.f;
            }
        }
        row_sum(t);
        const float inv = 1.0f / sqrtf(t[0] * a.inv_d + a.eps);
        const float m1 = a.center ? t[2] * a.inv_d : 0.f, m2 = t[1] * a.inv_d * inv;
        if (r < a.rows) {
#pragma unroll
            for (int q = 0; q < ITEMS; ++q) {
                float o[V], d[V], e[V];
                unpack(dc[q], d);
                unpack(sc[q], e);
                if constexpr (!keep) load_cols(a.w, cols.first[q], 1.f, wv[0]);
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const float xh = v[q][i] * inv;
                    o[i] = inv * (d[i] * wv[keep ? q : 0][i] - m1 - xh * m2) + (dsum ? e[i] : 0.f);
                    if constexpr (keep) {
                        aw[q][i] += d[i] * xh;
                        ab[q][i] += d[i];
                    } else {
                        s_col[slot(q, i)] += d[i] * xh;
                        s_col[W + slot(q, i)] += d[i];
                    }
                }
                if (cols.any(q)) store_v((GT*)a.dx + r * a.D + cols.first[q], o);
            }
        }
    }
    // the groups' column sums in the order of the groups
    float* part = a.part + (int64_t)blockIdx.x * 2 * a.D;
    const auto put = [&](int q, const float (&v)[V], float* out) {
        const int c = cols.first[q];
        if constexpr (RAGGED || V == 1) {
#pragma unroll
            for (int i = 0; i < V; ++i) {
                if (cols.own(q, i)) out[c + i] = v[i];
            }
        } else if (cols.any(q)) {
#pragma unroll
            for (int i = 0; i < V; i += 4) {
                const float o[4] = {v[i], v[i + 1], v[i + 2], v[i + 3]};
                store4(out + c + i, o);
            }
        }
    };
    if constexpr (!keep) {
#pragma unroll
        for (int q = 0; q < ITEMS; ++q) {
            float w[V], b[V];
#pragma unroll
            for (int i = 0; i < V; ++i) {
                w[i] = s_col[slot(q, i)];
                b[i] = s_col[W + slot(q, i)];
            }
            put(q, w, part);
            put(q, b, part + a.D);
        }
    } else {
        const auto finish = [&](float (&acc)[ITEMS][V], float* out) {
            if constexpr (GR > 1) {
                __syncthreads();
                if (group > 0) {
#pragma unroll
                    for (int q = 0; q < ITEMS; ++q)
#pragma unroll
                        for (int i = 0; i < V; ++i) s_col[(group - 1) * W + slot(q, i)] = acc[q][i];
                }
                __syncthreads();
            }
            if (group > 0) return;
#pragma unroll
            for (int q = 0; q < ITEMS; ++q) {
                for (int k = 0; k + 1 < GR; ++k) {
#pragma unroll
                    for (int i = 0; i < V; ++i) acc[q][i] += s_col[k * W + slot(q, i)];
                }
                put(q, acc[q], out);
            }
        };
        finish(aw, part);
        finish(ab, part + a.D);
    }
}

// Waves a CU holds of a form that keeps E elements per lane (by its registers): the
// grid is that, and a workgroup walks the rows.  More workgroups than that read
// the weights again and leave a last round that is not full (16384 rows of 4096
// bf16 with residual: forward 512 workgroups 80 us, 6.7 TB/s, 1024 85, one per
// row 285; 32768 rows of 768 backward 768 workgroups 38 us, 5.3 TB/s, 512 44, 1024 47;
// of 1280 forward 768 workgroups 30 us, 512 33).
constexpr int waves_per_cu(bool bwd, int v, int e) {
    return e <= 8 ? 16 : e <= 12 || (e == 24 && !bwd) || (e == 16 && (v == 8 || !bwd)) ? 12 : 8;
}
template <int TPR, int ITEMS, int V>
unsigned blocks_for(bool bwd, int64_t rows) {
    constexpr int threads = block_threads(TPR), waves = threads / 64;
    const int64_t b = (rows + threads / TPR - 1) / (threads / TPR);
    const int per = waves_per_cu(bwd, V, ITEMS * V) / waves;
    int64_t cap = (int64_t)device_cu_count() * (per > 0 ? per : 1);
    // in the backward four rounds or more where two workgroups per CU are left: each
    // ends in sums and a partial row (2048 rows of 2048 float 512 workgroups 19 us, 1024 24;
    // 16384 of 64 float 8.3 and 9.8; but 256 where 512 are had, 8192 of 128 bf16, 9.6 and 8.3)
    if (bwd && cap > b / 4) cap = std::min<int64_t>(cap, std::max<int64_t>(b / 4, 2 * (int64_t)device_cu_count()));
    return (unsigned)(b < cap ? b : cap);
}
// Most workgroups of any form of the backward: each leaves a partial row.
int64_t bwd_cap() { return (int64_t)device_cu_count() * 4; }

// The form that holds a row of n vectors: few idle lanes, few lanes to exchange sums
// between, and registers for two waves per SIMD.  A row to a wave needs no barrier: with
// up to 24 elements per lane in the backward (32768 rows of 1280 bf16 55 us, 256 lanes to
// a row 78; but 32, 8192 of 2048, 34.5 and 33.4) and 32 in the forward (32768 of 2048 bf16
// 44.5 us, 6.0 TB/s, and 55), where there are rows for it (300 of 2048 4.3 and 3.5).
// Float rows, with two vectors for one of bf16: up to 16 (100000 of 800, backward 182 and
// 208, forward 119 and 131; 8192 of 2048 at 32 28.1 and 24.9).  Beyond that at most 16 per
// lane.  Backward of more than 8192 columns, 16 elements in each of 1024
// lanes: the column sums stand in LDS (4096 rows of 16384 bf16 with dsum 136 us, 4.0 TB/s, 8
// registers still spilt; with the sums in registers 246), with float gradients at 46 registers
// spilt (4096 of 16384 float with dsum 288 us, 3.7 TB/s; bf16 without dsum 220).  Rows that are no multiple of a vector, at any alignment:
// 16384 rows of 4095 bf16 forward 5.0 TB/s, of 4096 6.7 (element by element 1.5).
#define DART_NORM_FORMS(V, BWD, FEW, F)                 \
    if constexpr (V == 8) {                             \
        if (n <= 16) F(8, 16, 1);                       \
        else if (n <= 64) F(8, 64, 1);                  \
        else if (n <= 128) F(8, 64, 2);                 \
        else if (n <= 192 && !(FEW)) F(8, 64, 3);       \
        else if (n <= 256) {                            \
            if constexpr (BWD) F(8, 256, 1);            \
            else if (FEW) F(8, 256, 1);                 \
            else F(8, 64, 4);                           \
        }                                               \
        else if (n <= 512) F(8, 512, 1);                \
        else if (n <= 1024) F(8, 1024, 1);              \
        else F(8, 1024, 2);                             \
    } else if constexpr (V == 4) {                      \
        if (n <= 16) F(4, 16, 1);                       \
        else if (n <= 64) F(4, 64, 1);                  \
        else if (n <= 128) F(4, 64, 2);                 \
        else if (n <= 192) F(4, 64, 3);                 \
        else if (n <= 256) {                            \
            if constexpr (BWD) F(4, 64, 4);             \
            else if (FEW) F(4, 256, 1);                 \
            else F(4, 64, 4);                           \
        }                                               \
        else if (n <= 512) F(4, 256, 2);                \
        else if (n <= 1024) F(4, 512, 2);               \
        else if (n <= 2048) F(4, 1024, 2);              \
        else F(4, 1024, 4);                             \
    } else {                                            \
        F(1, 16, 1); /* rows of less than one vector */ \
    }

template <typename T, int V>
void run_layernorm(const NormArgs& a, hipStream_t st) {
    const int n = (a.D + V - 1) / V;
#define DART_F(V_, TPR, ITEMS)                                                                                          \
    a.D % V_ == 0                                                                                                       \
        ? k_layernorm<T, V_, TPR, ITEMS, false><<<blocks_for<TPR, ITEMS, V_>(false, a.rows), block_threads(TPR), 0, st>>>(a) \
        : k_layernorm<T, V_, TPR, ITEMS, true><<<blocks_for<TPR, ITEMS, V_>(false, a.rows), block_threads(TPR), 0, st>>>(a)
    const bool few = a.rows < 4 * (int64_t)device_cu_count();
    DART_NORM_FORMS(V, false, few, DART_F)
#undef DART_F
}

// Returns the number of partial rows.
template <typename T, typename GT, int V>
unsigned run_layernorm_bwd(const NormBwdArgs& a, hipStream_t st) {
    const int n = (a.D + V - 1) / V;
    unsigned blocks = 0;
#define DART_F(V_, TPR, ITEMS)                                                                        \
    (blocks = blocks_for<TPR, ITEMS, V_>(true, a.rows),                                               \
     a.D % V_ == 0 ? k_layernorm_bwd<T, GT, V_, TPR, ITEMS, false><<<blocks, block_threads(TPR), 0, st>>>(a) \
                   : k_layernorm_bwd<T, GT, V_, TPR, ITEMS, true><<<blocks, block_threads(TPR), 0, st>>>(a))
    DART_NORM_FORMS(V, true, false, DART_F)
#undef DART_F
    return blocks;
}

}  // namespace

hipError_t launch_layernorm(int dtype, int64_t rows, int D, int center, const void* x, int64_t xs,
                            const void* res, int64_t rs, const float* w, const float* b, float eps,
                            void* out, void* sum, hipStream_t st) {
    if (rows == 0) return hipSuccess;
    const NormArgs a{x, res, xs, rs, rows, w, b, eps, 1.0f / D, out, sum, D, center};
    const bool wide = D >= (dtype == 1 ? 8 : 4);
    prof_begin("k_layernorm", st);
    if (dtype == 1) wide ? run_layernorm<bf16, 8>(a, st) : run_layernorm<bf16, 1>(a, st);
    else wide ? run_layernorm<float, 4>(a, st) : run_layernorm<float, 1>(a, st);
    prof_end(st);
    return hipGetLastError();
}

size_t layernorm_bwd_workspace_bytes(int64_t rows, int D) {
    const int64_t cap = bwd_cap();
    return align256(sizeof(float) * (size_t)(rows < cap ? rows : cap) * 2 * D);
}

hipError_t launch_layernorm_bwd(int dtype, int gdtype, int64_t rows, int D, int center, const void* x,
                                int64_t xs, const float* w, float eps, const void* dout,
                                const void* dsum, void* dx, float* dw, float* db, void* ws,
                                hipStream_t st) {
    float* part = reinterpret_cast<float*>(ws);
    unsigned nb = 0;
    if (rows > 0) {
        const NormBwdArgs a{x, xs, rows, w, eps, 1.0f / D, dout, dsum, dx, part, D, center};
        const bool wide = D >= (gdtype == 1 ? 8 : 4);
        prof_begin("k_layernorm_bwd", st);
        if (dtype == 0)
            nb = wide ? run_layernorm_bwd<float, float, 4>(a, st) : run_layernorm_bwd<float, float, 1>(a, st);
        else if (gdtype == 0)
            nb = wide ? run_layernorm_bwd<bf16, float, 4>(a, st) : run_layernorm_bwd<bf16, float, 1>(a, st);
        else
            nb = wide ? run_layernorm_bwd<bf16, bf16, 8>(a, st) : run_layernorm_bwd<bf16, bf16, 1>(a, st);
        prof_end(st);
    }
    // a partial row is one item of 2 D values: the first D are the weight's sums
    if (dw || db) sum_parts(part, nb, 2 * (int64_t)D, dw, 2 * D, D, db, st);
    return hipGetLastError();
}

}  // namespace dart
