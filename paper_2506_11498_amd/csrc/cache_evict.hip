// Eviction by accumulated attention weight: a cache that has outgrown its budget keeps its first `sink` rows, its last
// `recent` rows and, of the rows between, those with the largest weight (ties to the lowest position), in position order.
// The rows go to another cache, which a program swaps with the old one: every row is read and written once, whatever the
// order in which workgroups run.  In place, the rows would go through a workspace of the same size first.
//
// k_evict_select    one workgroup per (sequence, KV head): the list of rows that stay
// k_evict_rows      fp32 and bf16 caches: rows, positions and weights by that list
// k_evict_quant     8-bit caches: the same, in blocks with a scale of their own
#include "quant_block.h"
#include "select_block.h"

namespace lrsa {

constexpr int EVICT_THREADS = 1024;
constexpr int EVICT_BINS = 2048;

struct EvictArgs {
    const int32_t* lens;     // rows of every sequence, or NULL: `len`
    int len, budget, recent;
    int64_t cap;
    const int32_t* pos;      // [units][cap] or NULL
    const float* acc;
    int32_t* pos_o;
    float* acc_o;
    int32_t* lens_o;         // or NULL
};
__device__ __forceinline__ int evict_len(const EvictArgs& E, int b) { return E.lens ? max(0, min(E.lens[b], E.len)) : E.len; }

// Order of weights as of unsigned numbers, with room for 0 and the largest: those are rows that are not there and rows that
// stay whatever their weight.  -0 equals 0.
__device__ __forceinline__ uint32_t weight_key(float x) {
    uint32_t u = __float_as_uint(x + 0.0f);
    u ^= u >> 31 ? 0xffffffffu : 0x80000000u;
    return min(max(u, 1u), 0xfffffffeu);
}

// Radix select of the budget-th largest key (digits of 11, 11 and 10 bits: a weight's first 11 bits are sign, exponent and two
// bits of fraction, which spreads the LDS atomics), then an ordered compaction.  Integer work only: deterministic.
__global__ __launch_bounds__(EVICT_THREADS) void k_evict_select(Dims D, EvictArgs E, int32_t* __restrict__ keep) {
    __shared__ int hist[EVICT_BINS];
    __shared__ int sm[EVICT_THREADS / 64];
    __shared__ uint32_t s_prefix;
    __shared__ int s_need, s_all;
    const int unit = blockIdx.x, b = unit / D.Hkv, tid = threadIdx.x;
    const int len = evict_len(E, b);
    if (E.lens_o && unit % D.Hkv == 0 && tid == 0) E.lens_o[b] = min(len, E.budget);
    keep += int64_t(unit) * E.budget;
    if (len <= E.budget) {
        for (int r = tid; r < len; r += EVICT_THREADS) keep[r] = r;
        return;
    }
    const float* acc = E.acc + int64_t(unit) * E.cap;
    const int tail = len - E.recent;
    auto key = [&](int r) { return r < D.S || r >= tail ? 0xffffffffu : weight_key(acc[r]); };
    uint32_t prefix = 0, mask = 0;
    int need = E.budget;
    for (int pass = 0; pass < 3; ++pass) {
        const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bits = pass == 2 ? 10 : 11;
        for (int i = tid; i < EVICT_BINS; i += EVICT_THREADS) hist[i] = 0;
        __syncthreads();
        for (int r = tid; r < len; r += EVICT_THREADS) {
            const uint32_t k = key(r);
            if ((k & mask) == prefix) atomicAdd(&hist[(k >> shift) & ((1u << bits) - 1)], 1);
        }
        __syncthreads();
        const int top = EVICT_BINS - 1 - 2 * tid, c0 = hist[top], c1 = hist[top - 1];
        int total;
        const int above = block_exscan<EVICT_THREADS>(c0 + c1, sm, &total);
        if (above < need && need <= above + c0) {
            s_prefix = prefix | uint32_t(top) << shift;
            s_need = need - above;
            s_all = need - above == c0;
        } else if (above + c0 < need && need <= above + c0 + c1) {
            s_prefix = prefix | uint32_t(top - 1) << shift;
            s_need = need - above - c0;
            s_all = need - above - c0 == c1;
        }
        __syncthreads();
        prefix = s_prefix;
        need = s_need;
        mask |= ((1u << bits) - 1) << shift;
        if (s_all) break;
    }
    // larger than the threshold, or among the first `need` equal to it on the decided bits
    constexpr int RUN = 4;
    int gt_seen = 0, eq_seen = 0;
    for (int b0 = 0; b0 < len; b0 += RUN * EVICT_THREADS) {
        const int r0 = b0 + tid * RUN;
        uint32_t km[RUN];
        int ngt = 0, neq = 0;
#pragma unroll
        for (int i = 0; i < RUN; ++i) {
            km[i] = r0 + i < len ? key(r0 + i) & mask : 0u;
            ngt += (r0 + i < len && km[i] > prefix) ? 1 : 0;
            neq += (r0 + i < len && km[i] == prefix) ? 1 : 0;
        }
        int total;
        const int before = block_exscan<EVICT_THREADS>(ngt | (neq << 16), sm, &total);
        int g = gt_seen + (before & 0xffff), e = eq_seen + (before >> 16);
#pragma unroll
        for (int i = 0; i < RUN; ++i) {
            if (r0 + i >= len) break;
            const bool is_gt = km[i] > prefix, is_eq = km[i] == prefix;
            if (is_gt || (is_eq && e < need)) keep[g + min(e, need)] = r0 + i;
            g += is_gt ? 1 : 0;
            e += is_eq ? 1 : 0;
        }
        gt_seen += total & 0xffff;
        eq_seen += total >> 16;
    }
}

// positions and weights of the rows that stay; weights behind them are zero, for the rows that come next
__device__ __forceinline__ void evict_lists(const EvictArgs& E, int unit, int len, const int32_t* keep, int part, int parts) {
    const int rows = min(len, E.budget);
    const int64_t at = int64_t(unit) * E.cap;
    for (int64_t i = int64_t(part) * blockDim.x + threadIdx.x; i < E.cap; i += int64_t(parts) * blockDim.x) {
        const int src = i < rows ? keep[i] : 0;
        E.acc_o[at + i] = i < rows ? E.acc[at + src] : 0.0f;
        if (E.pos && i < rows) E.pos_o[at + i] = E.pos[at + src];
    }
}

// 16 bytes per thread
template <typename T>
__global__ __launch_bounds__(256) void k_evict_rows(Dims D, EvictArgs E, const T* __restrict__ K, const T* __restrict__ V, const int32_t* __restrict__ keep,
                                                    T* __restrict__ Ko, T* __restrict__ Vo) {
    const int z = blockIdx.y, unit = blockIdx.z, b = unit / D.Hkv, h = unit % D.Hkv;
    const int len = evict_len(E, b);
    keep += int64_t(unit) * E.budget;
    if (z == 2) {
        evict_lists(E, unit, len, keep, blockIdx.x, gridDim.x);
        return;
    }
    const int lpr = D.d / Elem<T>::VEC;
    const int64_t e = int64_t(blockIdx.x) * 256 + threadIdx.x;
    const int64_t i = e / lpr;
    if (i >= min(len, E.budget)) return;
    const int64_t at = b * D.ks[0] + h * D.ks[1] + e % lpr * Elem<T>::VEC;
    *reinterpret_cast<uint4*>((z ? Vo : Ko) + at + i * D.ks[2]) = *reinterpret_cast<const uint4*>((z ? V : K) + at + int64_t(keep[i]) * D.ks[2]);
}

// One workgroup per block of the new cache
template <int DH, int FMT>
__global__ __launch_bounds__(256) void k_evict_quant(Dims D, EvictArgs E, QuantDims Q, const int32_t* __restrict__ keep, QuantDims N) {
    constexpr int LPR = DH / 8, RPP = 256 / LPR, PASSES = QUANT_MAX_BLOCK / RPP;
    __shared__ float sm[4];
    const int z = blockIdx.y, unit = blockIdx.z, b = unit / D.Hkv, h = unit % D.Hkv;
    const int len = evict_len(E, b);
    keep += int64_t(unit) * E.budget;
    if (z == 2) {
        evict_lists(E, unit, len, keep, blockIdx.x, gridDim.x);
        return;
    }
    const int64_t row0 = int64_t(blockIdx.x) << N.log_block;
    const int rows = int(min(int64_t(N.block), min(len, E.budget) - row0));
    if (rows <= 0) return;
    const int sub = threadIdx.x % LPR, rg = threadIdx.x / LPR;
    const uint8_t* src = (z ? Q.V : Q.K) + b * Q.st[0] + h * Q.st[1] + sub * 8;
    const float* scales = (z ? Q.Vs : Q.Ks) + int64_t(unit) * Q.nb;
    float v[PASSES][8], top = 0.0f;
#pragma unroll
    for (int p = 0; p < PASSES; ++p) {
        const int r = p * RPP + rg;
        if (r < rows) {
            const int from = keep[row0 + r];
            const float s = scales[from >> Q.log_block];
            code_values<FMT>(*reinterpret_cast<const uint2*>(src + from * Q.st[2]), v[p]);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[p][i] *= s;
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[p][i] = 0.0f;
        }
    }
#pragma unroll
    for (int p = 0; p < PASSES; ++p)
#pragma unroll
        for (int i = 0; i < 8; ++i) top = fmaxf(top, fabsf(v[p][i]));
    const float s = quant_scale<FMT>(block_max<256>(top, sm));
    const float inv = 1.0f / s;
    if (threadIdx.x == 0) (z ? N.Vs : N.Ks)[int64_t(unit) * N.nb + blockIdx.x] = s;
    uint8_t* dst = (z ? N.V : N.K) + b * N.st[0] + h * N.st[1] + row0 * N.st[2] + sub * 8;
#pragma unroll
    for (int p = 0; p < PASSES; ++p) {
        const int r = p * RPP + rg;
        if (r < rows) *reinterpret_cast<uint2*>(dst + r * N.st[2]) = make_codes<FMT>(v[p], inv);
    }
}

size_t cache_evict_ws_bytes(const Dims& D, int budget) { return align256(size_t(D.B) * D.Hkv * budget * 4); }
bool cache_evict_grid_fits(const Dims& D, int budget) { return grid_fits((int64_t(budget) * 32 + 255) / 256 + 1, 256); }

static EvictArgs evict_args(const Dims& D, const int32_t* lens, int len, int budget, int recent, const int32_t* pos, const float* acc, int32_t* pos_o,
                            float* acc_o, int32_t* lens_o) {
    EvictArgs E = {};
    E.lens = lens;
    E.len = len;
    E.budget = budget;
    E.recent = recent;
    E.cap = D.n;
    E.pos = pos;
    E.acc = acc;
    E.pos_o = pos_o;
    E.acc_o = acc_o;
    E.lens_o = lens_o;
    return E;
}

template <typename T>
static hipError_t run_evict(const Dims& D, const EvictArgs& E, const void* K, const void* V, void* Ko, void* Vo, int32_t* keep, hipStream_t st) {
    const int rows = E.len < E.budget ? E.len : E.budget;
    LRSA_TIMED_LAUNCH("k_evict_select", st, k_evict_select, dim3(D.B * D.Hkv), dim3(EVICT_THREADS), 0, st, D, E, keep);
    const unsigned blocks = unsigned((int64_t(rows) * (D.d / Elem<T>::VEC) + 255) / 256);
    LRSA_TIMED_LAUNCH("k_evict_rows", st, k_evict_rows<T>, dim3(blocks ? blocks : 1, 3, D.B * D.Hkv), dim3(256), 0, st, D, E, (const T*)K, (const T*)V,
                      keep, (T*)Ko, (T*)Vo);
    return hipGetLastError();
}
hipError_t launch_cache_evict(const Dims& D, const void* K, const void* V, const int32_t* pos, const float* acc, int len, int budget, int recent,
                              void* Ko, void* Vo, int32_t* pos_o, float* acc_o, void* ws, hipStream_t st) {
    const EvictArgs E = evict_args(D, nullptr, len, budget, recent, pos, acc, pos_o, acc_o, nullptr);
    return D.dtype == 1 ? run_evict<bf16_t>(D, E, K, V, Ko, Vo, (int32_t*)ws, st) : run_evict<float>(D, E, K, V, Ko, Vo, (int32_t*)ws, st);
}
hipError_t launch_cache_evict_quant(const Dims& D, const QuantDims& Q, const QuantDims& N, const int32_t* lens, int max_len, int budget, int recent,
                                    const int32_t* pos, const float* acc, int32_t* pos_o, float* acc_o, int32_t* lens_o, void* ws, hipStream_t st) {
    const EvictArgs E = evict_args(D, lens, max_len, budget, recent, pos, acc, pos_o, acc_o, lens_o);
    int32_t* keep = (int32_t*)ws;
    const int rows = max_len < budget ? max_len : budget;
    LRSA_TIMED_LAUNCH("k_evict_select", st, k_evict_select, dim3(D.B * D.Hkv), dim3(EVICT_THREADS), 0, st, D, E, keep);
    const dim3 grid(unsigned((rows + N.block - 1) / N.block ? (rows + N.block - 1) / N.block : 1), 3, D.B * D.Hkv);
#define LRSA_EVICT_QUANT(DH_, FMT_) LRSA_TIMED_LAUNCH("k_evict_quant", st, (k_evict_quant<DH_, FMT_>), grid, dim3(256), 0, st, D, E, Q, keep, N)
    if (Q.fmt == QUANT_INT8) {
        if (D.d == 64) LRSA_EVICT_QUANT(64, QUANT_INT8); else LRSA_EVICT_QUANT(128, QUANT_INT8);
    } else {
        if (D.d == 64) LRSA_EVICT_QUANT(64, QUANT_E4M3); else LRSA_EVICT_QUANT(128, QUANT_E4M3);
    }
#undef LRSA_EVICT_QUANT
    return hipGetLastError();
}

}  // namespace lrsa
