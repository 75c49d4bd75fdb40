// Attention of single queries over a cache in slices of rows: the records that a slice leaves behind, how slices are
// joined, and how the weights are added to the rows' accumulated weights.
//
// Record of (query row, slice): max and sum of the weights in log2 units, then d unnormalised output values, fp32.
#pragma once
#include "common.h"

namespace lrsa {

constexpr int DEC_THREADS = 256;
constexpr int DEC_WAVES = DEC_THREADS / 64;
constexpr int DEC_MAX_SPLITS = 256;
constexpr int COMB_U = 4;
constexpr int ACC_ROWS = 4 * DEC_THREADS;     // cache rows per workgroup of the weight sums

// What the weight sums read besides the records: logits [unit][cols][stride], in log2 units after the factor `mul`, -inf where
// masked; a unit is one (sequence, KV head), its columns the query rows that read it.
struct AccArgs {
    const float* logits;
    float mul;
    int64_t stride;          // floats between columns, a multiple of 4
    int cols;
    const float* in;         // [units][cap] or NULL: zeros
    float* out;              // [units][cap]
    int64_t cap;
    float decay;
};

#if defined(__HIPCC__)
// (m, l, o) of two disjoint key sets -> of their union
__device__ __forceinline__ void merge_state(float& m, float& l, float m2, float l2, float& a, float& b2) {
    const float mn = fmaxf(m, m2);
    a = m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m - mn);
    b2 = m2 == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m2 - mn);
    l = l * a + l2 * b2;
    m = mn;
}

// Max, sum and the slices' weights of one query row, by a whole wave: lane l holds slices l, l + 64, ...
__device__ __forceinline__ void merge_records(const float* src, int rec, int splits, float (&w)[DEC_MAX_SPLITS / 64], float& M, float& L) {
    const int lane = threadIdx.x & 63;
    float m[DEC_MAX_SPLITS / 64], l[DEC_MAX_SPLITS / 64];
    M = -INFINITY;
    L = 0.0f;
#pragma unroll
    for (int i = 0; i < DEC_MAX_SPLITS / 64; ++i) {
        const int s = lane + 64 * i;
        m[i] = -INFINITY; l[i] = 0.0f;
        if (s < splits) {
            const float2 ml = *reinterpret_cast<const float2*>(src + int64_t(s) * rec);
            m[i] = ml.x; l[i] = ml.y;
        }
        M = fmaxf(M, m[i]);
    }
    M = wave_max(M);
#pragma unroll
    for (int i = 0; i < DEC_MAX_SPLITS / 64; ++i) {
        w[i] = m[i] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m[i] - M);
        L = __builtin_fmaf(l[i], w[i], L);
    }
    L = wave_sum(L);
}

struct CombineLds {
    float w[DEC_MAX_SPLITS];
    float2 o[DEC_THREADS];
};
// One query row per workgroup: the weights of all slices first (two loads per lane and 64 slices), then the records are
// summed by all lanes, two channels each, COMB_U loads in flight; fixed order.  A row that sees nothing (no slices, or no
// weight in any) gets zeros and -inf.
template <typename T>
__device__ __forceinline__ void combine_row(const float* src, int d, int splits, T* O, float* lse, CombineLds& sh) {
    const int tid = threadIdx.x, lane = tid & 63, rec = d + 2;
    float w[DEC_MAX_SPLITS / 64], M, L;
    merge_records(src, rec, splits, w, M, L);
#pragma unroll
    for (int i = 0; i < DEC_MAX_SPLITS / 64; ++i)
        if (tid < 64) sh.w[lane + 64 * i] = w[i];
    __syncthreads();
    const int pairs = d / 2, ways = DEC_THREADS / pairs, ch = tid % pairs, way = tid / pairs;
    float2 o = {0.0f, 0.0f};
    for (int s0 = way; s0 < splits; s0 += COMB_U * ways) {
        float2 v[COMB_U];
        float w[COMB_U];
#pragma unroll
        for (int u = 0; u < COMB_U; ++u) {
            const int s = s0 + u * ways, sc = min(s, splits - 1);
            w[u] = s < splits ? sh.w[sc] : 0.0f;
            v[u] = *reinterpret_cast<const float2*>(src + int64_t(sc) * rec + 2 + 2 * ch);
        }
#pragma unroll
        for (int u = 0; u < COMB_U; ++u) {
            o.x = __builtin_fmaf(w[u], v[u].x, o.x);
            o.y = __builtin_fmaf(w[u], v[u].y, o.y);
        }
    }
    sh.o[tid] = o;
    __syncthreads();
    if (tid < pairs) {
        for (int w = 1; w < ways; ++w) { o.x += sh.o[w * pairs + tid].x; o.y += sh.o[w * pairs + tid].y; }
        const bool none = L == 0.0f;
        Elem<T>::put(O + 2 * ch, none ? 0.0f : o.x / L);
        Elem<T>::put(O + 2 * ch + 1, none ? 0.0f : o.y / L);
        if (lse && tid == 0)   // one rounding at the end: ln 2 as its fp32 value plus the rest
            *lse = none ? -INFINITY : __builtin_fmaf(M, 0.69314718246459961f, __builtin_fmaf(M, -1.9046542e-9f, __builtin_log2f(L) * 0.6931471805599453f));
    }
}

// acc_out[r] = decay acc_in[r] + sum over the columns of exp2(logit - log2 of the column's whole weight), for rows [r0, r0 +
// ACC_ROWS) below `len`, by one workgroup; 4 neighbouring rows per thread.  `first`: record of the unit's first column,
// `splits` of them per column, columns `col_floats` apart.
constexpr int ACC_COLS = 256;      // columns whose log-sum-exp is in LDS at once
__device__ __forceinline__ void acc_rows(const AccArgs& A, int unit, const float* first, int64_t col_floats, int rec, int splits, int r0, int len,
                                         float (&sLse)[ACC_COLS]) {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, r = r0 + 4 * tid;
    float4 t = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int c0 = 0; c0 < A.cols; c0 += ACC_COLS) {
        const int cn = min(ACC_COLS, A.cols - c0);
        if (c0) __syncthreads();
        for (int c = wave; c < cn; c += DEC_WAVES) {
            float w[DEC_MAX_SPLITS / 64], M, L;
            merge_records(first + (c0 + c) * col_floats, rec, splits, w, M, L);
            if (lane == 0) sLse[c] = L == 0.0f ? INFINITY : M + __builtin_log2f(L);
        }
        __syncthreads();
        if (r < len) {
            const float* s = A.logits + (int64_t(unit) * A.cols + c0) * A.stride + r;
            for (int c = 0; c < cn; ++c) {
                const float4 x = *reinterpret_cast<const float4*>(s + c * A.stride);
                const float n = sLse[c];
                t.x += __builtin_amdgcn_exp2f(__builtin_fmaf(x.x, A.mul, -n));
                t.y += __builtin_amdgcn_exp2f(__builtin_fmaf(x.y, A.mul, -n));
                t.z += __builtin_amdgcn_exp2f(__builtin_fmaf(x.z, A.mul, -n));
                t.w += __builtin_amdgcn_exp2f(__builtin_fmaf(x.w, A.mul, -n));
            }
        }
    }
    const float v[4] = {t.x, t.y, t.z, t.w};
    const int64_t at = int64_t(unit) * A.cap + r;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (r + i < len) A.out[at + i] = A.in ? __builtin_fmaf(A.decay, A.in[at + i], v[i]) : v[i];
}
#endif

}  // namespace lrsa
