// Attention of single queries over a cache in slices of rows: the records that a slice leaves behind, how slices are
// joined, and how the weights are added to the rows' accumulated weights.
//
// Record of (query row, slice): max and sum of the weights in log2 units, then d unnormalised output values, fp32.  The slices of a
// query row are `step` floats apart.
#pragma once
#include "common.h"

namespace lrsa {

constexpr int DEC_THREADS = 256;
constexpr int DEC_WAVES = DEC_THREADS / 64;
constexpr int DEC_MAX_SPLITS = 256;
constexpr int COMB_U = 4;

// What the weight sums read besides the records: logits [unit][rows][pitch], in log2 units after the factor `mul`, -inf where
// masked; a unit is one (sequence, KV head), its `cols` columns the query rows that read it, in the first cols of pitch values.
// Row by row, so that a tile's logits are one piece of memory.
struct AccArgs {
    const float* logits;
    float mul;
    int64_t rows;
    int cols, pitch;         // pitch: the columns rounded up to a multiple of 4
    const float* in;         // [units][cap] or NULL: zeros
    float* out;              // [units][cap]
    int64_t cap;
    float decay;
};
// cache rows per workgroup of the weight sums
__host__ __device__ inline int acc_wg_rows(int pitch) { return DEC_THREADS * (pitch <= 8 ? 4 : pitch <= 16 ? 2 : 1); }

#if defined(__HIPCC__)
// A wave's logits on their way to memory.  They stay in LDS until it is full or the walk over the slice ends: a stream of reads that
// a few writes are mixed into runs at the rate of a copy, not of a read (8 requests of 32K rows of 8 bits, 4
// columns: 119.7 us with a store per tile, 107.1, and 91.7 without logits).  Tiles of 32 rows
// x up to 16 columns (lane l: column l % 16, 8 of the rows), `step` rows apart.
constexpr int LOGIT_FLOATS = 4096;       // per wave: 32 tiles of 4 columns
struct LogitBuffer {
    float *lds, *dst;        // dst: the columns' first in the first row of the first tile that is held
    int pitch, gn, used, most;
    int64_t skip;            // floats between tiles in memory
};
// lds: `floats` of it; gn columns, none where 0
__device__ __forceinline__ LogitBuffer logit_buffer(float* lds, int floats, float* dst, int pitch, int gn, int step) {
    const int width = (gn + 3) & ~3;
    return LogitBuffer{lds, dst, pitch, gn, 0, floats / (32 * max(width, 4)), int64_t(step) * pitch};
}
__device__ __forceinline__ void flush_logits(LogitBuffer& B) {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    const int pieces = (B.gn + 3) >> 2, lane = threadIdx.x & 63;
    for (int t = 0; t < B.used; ++t, B.dst += B.skip)
        for (int l = lane; l < 32 * pieces; l += 64) {
            const int row = pieces == 3 ? l / 3 : l >> (pieces >> 1), part = l - row * pieces;      // what lies in pad columns is never read
            *reinterpret_cast<float4*>(B.dst + int64_t(row) * B.pitch + part * 4) = *reinterpret_cast<const float4*>(B.lds + (t * 32 * pieces + l) * 4);
        }
    B.used = 0;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
}
// the next tile; row(j): of the lane's value j
template <class Row>
__device__ __forceinline__ void keep_logits(LogitBuffer& B, const float (&p)[8], Row row) {
    const int width = (B.gn + 3) & ~3, c = threadIdx.x & 15;
    if (B.used == B.most) flush_logits(B);
    if (c < width)
#pragma unroll
        for (int j = 0; j < 8; ++j) B.lds[(B.used * 32 + row(j)) * width + c] = p[j];
    ++B.used;
}

// (m, l, o) of two disjoint key sets -> of their union
__device__ __forceinline__ void merge_state(float& m, float& l, float m2, float l2, float& a, float& b2) {
    const float mn = fmaxf(m, m2);
    a = m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m - mn);
    b2 = m2 == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m2 - mn);
    l = l * a + l2 * b2;
    m = mn;
}

// Max, sum and the slices' weights of one query row, by a whole wave: lane l holds slices l, l + 64, ...
__device__ __forceinline__ void merge_records(const float* src, int64_t step, int splits, float (&w)[DEC_MAX_SPLITS / 64], float& M, float& L) {
    const int lane = threadIdx.x & 63;
    float m[DEC_MAX_SPLITS / 64], l[DEC_MAX_SPLITS / 64];
    M = -INFINITY;
    L = 0.0f;
#pragma unroll
    for (int i = 0; i < DEC_MAX_SPLITS / 64; ++i) {
        const int s = lane + 64 * i;
        m[i] = -INFINITY; l[i] = 0.0f;
        if (s < splits) {
            const float2 ml = *reinterpret_cast<const float2*>(src + s * step);
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

// log2 of the whole weight of U query rows, `cols` floats apart, by a wave; +inf where there is none.  One record per lane: all rows'
// records are asked for at once
template <int U>
__device__ __forceinline__ void merge_logs(const float* src, int64_t cols, int64_t step, int splits, float (&out)[U]) {
    const int lane = threadIdx.x & 63;
    float2 ml[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        ml[u] = float2{-INFINITY, 0.0f};
        if (lane < splits) ml[u] = *reinterpret_cast<const float2*>(src + u * cols + lane * step);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const float M = wave_max(ml[u].x);
        const float L = wave_sum(ml[u].x == -INFINITY ? 0.0f : ml[u].y * __builtin_amdgcn_exp2f(ml[u].x - M));
        out[u] = L == 0.0f ? INFINITY : M + __builtin_log2f(L);
    }
}

// natural log of 2^M * L.  One rounding at the end: ln 2 as its fp32 value plus the rest
__device__ __forceinline__ float log2_to_ln(float M, float L) {
    return __builtin_fmaf(M, 0.69314718246459961f, __builtin_fmaf(M, -1.9046542e-9f, __builtin_log2f(L) * 0.6931471805599453f));
}

struct CombineLds {
    float w[DEC_MAX_SPLITS];
    float2 o[DEC_THREADS];
};
// One query row per workgroup: the weights of all slices first (two loads per lane and 64 slices), then the records are
// summed by all lanes, two channels each, COMB_U loads in flight; fixed order.  A row that sees nothing (no slices, or no
// weight in any) gets zeros and -inf.
template <typename T>
__device__ __forceinline__ void combine_row(const float* src, int64_t step, int d, int splits, T* O, float* lse, CombineLds& sh) {
    const int tid = threadIdx.x, lane = tid & 63;
    float w[DEC_MAX_SPLITS / 64], M, L;
    merge_records(src, step, splits, w, M, L);
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
            v[u] = *reinterpret_cast<const float2*>(src + sc * step + 2 + 2 * ch);
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
        if (lse && tid == 0) *lse = none ? -INFINITY : log2_to_ln(M, L);
    }
}

// acc_out[r] = decay acc_in[r] + sum over the columns of exp2(logit - log2 of the column's whole weight), for rows r0 .. below `len`, U
// per thread, by one workgroup.  `first`: record of the unit's first column, columns `col_floats` apart.  Eight 16-byte reads of logits
// per thread are on their way at once, the first ones while the columns' weights are put together.
constexpr int ACC_COLS = 256;      // columns whose log-sum-exp is in LDS at once
template <int U>
__device__ __forceinline__ void acc_rows_u(const AccArgs& A, int unit, const float* first, int64_t col_floats, int64_t step, int splits, int r0, int len,
                                           float* sLse) {
    constexpr int C = 8 / U;                 // groups of 4 columns at once
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const float* s = A.logits + int64_t(unit) * A.rows * A.pitch;
    const float* row[U];
#pragma unroll
    for (int u = 0; u < U; ++u) row[u] = s + int64_t(min(r0 + u * DEC_THREADS + tid, len - 1)) * A.pitch;
    float4 x[C][U];
    auto load = [&](int c0) {
#pragma unroll
        for (int i = 0; i < C; ++i)
#pragma unroll
            for (int u = 0; u < U; ++u) x[i][u] = *reinterpret_cast<const float4*>(row[u] + min(c0 + 4 * i, A.pitch - 4));
    };
    load(0);
    float sum[U] = {};
    for (int c0 = 0; c0 < A.cols; c0 += ACC_COLS) {
        const int cn = min(ACC_COLS, A.cols - c0);
        if (c0) __syncthreads();
        // a wave takes a column, of many columns four at once
        const int batch = cn > 8 && splits <= 64 ? 4 : 1;
        for (int c = wave * batch; c < cn; c += DEC_WAVES * batch) {
            if (c + batch <= cn && batch > 1) {
                float logs[4];
                merge_logs<4>(first + (c0 + c) * col_floats, col_floats, step, splits, logs);
                if (lane == 0) *reinterpret_cast<float4*>(&sLse[c]) = float4{logs[0], logs[1], logs[2], logs[3]};
                continue;
            }
            for (int k = c; k < min(c + batch, cn); ++k) {
                float w[DEC_MAX_SPLITS / 64], M, L;
                merge_records(first + (c0 + k) * col_floats, step, splits, w, M, L);
                if (lane == 0) sLse[k] = L == 0.0f ? INFINITY : M + __builtin_log2f(L);
            }
        }
        __syncthreads();
        for (int cb = 0; cb < cn; cb += 4 * C) {
            if (c0 + cb) load(c0 + cb);
#pragma unroll
            for (int i = 0; i < C; ++i) {
                const int c = cb + 4 * i;
                if (c >= cn) break;
                const float4 n = *reinterpret_cast<const float4*>(&sLse[c]);
                // a pad column's value is whatever was there
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    sum[u] += __builtin_amdgcn_exp2f(__builtin_fmaf(x[i][u].x, A.mul, -n.x));
                    if (c + 1 < cn) sum[u] += __builtin_amdgcn_exp2f(__builtin_fmaf(x[i][u].y, A.mul, -n.y));
                    if (c + 2 < cn) sum[u] += __builtin_amdgcn_exp2f(__builtin_fmaf(x[i][u].z, A.mul, -n.z));
                    if (c + 3 < cn) sum[u] += __builtin_amdgcn_exp2f(__builtin_fmaf(x[i][u].w, A.mul, -n.w));
                }
            }
        }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int r = r0 + u * DEC_THREADS + tid;
        const int64_t at = int64_t(unit) * A.cap + r;
        if (r < len) A.out[at] = A.in ? __builtin_fmaf(A.decay, A.in[at], sum[u]) : sum[u];
    }
}
__device__ __forceinline__ void acc_rows(const AccArgs& A, int unit, const float* first, int64_t col_floats, int64_t step, int splits, int r0, int len,
                                         float* sLse /* [ACC_COLS], 16-byte aligned */) {
    if (A.pitch <= 8) acc_rows_u<4>(A, unit, first, col_floats, step, splits, r0, len, sLse);
    else if (A.pitch <= 16) acc_rows_u<2>(A, unit, first, col_floats, step, splits, r0, len, sLse);
    else acc_rows_u<1>(A, unit, first, col_floats, step, splits, r0, len, sLse);
}
#endif

}  // namespace lrsa
