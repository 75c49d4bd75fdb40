// Eviction by accumulated attention weight: a cache that has outgrown its budget keeps its first `sink` rows, its last
// `recent` rows and, of the rows between, those with the largest weight (ties to the lowest position), in position order.
// The rows go to another cache, which a program swaps with the old one: every row is read and written once, whatever the
// order in which workgroups run.  In place, the rows would go through a workspace of the same size first.
//
// k_evict_select    one workgroup per (sequence, KV head): the list of rows that stay
// k_evict_rows      fp32 and bf16 caches: rows, positions and weights by that list
// k_evict_quant     8-bit caches: the same, in blocks with a scale of their own
// k_evict_short, k_evict_quant_short  both steps in one launch, for short caches
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

// Order of weights as of unsigned numbers.  -0 equals 0; what is no number goes to either end.  Of weights, the first 11 bits are
// neither all zeros nor all ones: those are rows that are not there and rows that stay whatever their weight.
constexpr uint32_t KEY_ABSENT = 0u, KEY_STAYS = 0xffffffffu;
__device__ __forceinline__ uint32_t weight_key(float x) {
    uint32_t u = __float_as_uint(x + 0.0f);
    u ^= u >> 31 ? 0xffffffffu : 0x80000000u;
    return min(max(u, 0x00400000u), 0xffbfffffu);
}

// Radix select of the smallest key that stays (digits of 11, 11 and 10 bits: a weight's first 11 bits are sign, exponent and two
// bits of fraction, which spreads the LDS atomics; two histograms, a lane's by its number, so that equal keys collide in 32
// lanes and not in 64), then an ordered compaction by ballots.  Integer work only: deterministic.
// A wave holds 64 * KPT neighbouring rows' keys in registers, four neighbours per lane and group, so the weights are read once; a cache of
// more than 16 waves' keys is taken in parts, read again in every pass.  One workgroup, because its passes depend on each other; bound by
// what one CU reads and by some 20 instructions and an LDS atomic per row: 4.5K rows 7.6 us, 32K rows 16.5 us for 8 heads and 18 to 20 for 32 to
// 64 (keys in LDS, an atomic behind a branch per row and pass: 1.1 and 1.4 times as long); in parts 32K rows and one 38, 64K 35, 128K 63,
// more than the move of the rows that stay (8 heads, a quarter of 128K rows of bf16: 51).
// put(i, r): row r of the old cache becomes row i of the new one.
template <int KPT, class Put>
__device__ __forceinline__ void select_rows(const Dims& D, const EvictArgs& E, int unit, int len, Put put) {
    constexpr int WAVES = EVICT_THREADS / 64, PART = EVICT_THREADS * KPT, GROUPS = KPT / 4, COPIES = 2, PITCH = EVICT_BINS + 4;
    __shared__ __attribute__((aligned(16))) int hist[COPIES * PITCH + 64];
    __shared__ int sm[WAVES];
    __shared__ int2 s_count[WAVES];
    __shared__ uint32_t s_prefix;
    __shared__ int s_need, s_all;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    if (len <= E.budget) {
        for (int r = tid; r < len; r += EVICT_THREADS) put(r, r);
        return;
    }
    struct __attribute__((packed, aligned(4))) Four { uint32_t v[4]; };
    const uint32_t* acc = reinterpret_cast<const uint32_t*>(E.acc + int64_t(unit) * E.cap);
    const int tail = len - E.recent, parts = (len + PART - 1) / PART;
    uint4 k[GROUPS];                         // of group g: rows 256 g + 4 lane .. + 3 of the wave's
    auto first_row = [&](int part) { return part * PART + wave * 64 * KPT; };
    auto load = [&](int part) {
        const int first = first_row(part);
        if (first + 64 * KPT <= len) {
            const uint32_t* src = acc + first;
#pragma unroll
            for (int g = 0; g < GROUPS; ++g) {
                const Four f = *reinterpret_cast<const Four*>(src + 256 * g + uint32_t(4 * lane));
                // opaque: or the compiler makes one set of loads, word by word, of this branch's and the other's
                k[g] = uint4{as_loaded(f.v[0]), as_loaded(f.v[1]), as_loaded(f.v[2]), as_loaded(f.v[3])};
            }
        } else {
            const uint32_t* src = acc + min(first, len - 1);
            const uint32_t last = max(len - 1 - first, 0);
#pragma unroll
            for (int g = 0; g < GROUPS; ++g) {
                const uint32_t r = 256 * g + 4 * lane;
                k[g] = uint4{src[min(r, last)], src[min(r + 1, last)], src[min(r + 2, last)], src[min(r + 3, last)]};
            }
        }
        const bool plain = first >= D.S && first + 64 * KPT <= tail;
#pragma unroll
        for (int g = 0; g < GROUPS; ++g) {
            uint32_t v[4] = {k[g].x, k[g].y, k[g].z, k[g].w};
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = weight_key(__uint_as_float(v[i]));
            if (!plain)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int r = first + 256 * g + 4 * lane + i;
                    v[i] = r >= len ? KEY_ABSENT : r < D.S || r >= tail ? KEY_STAYS : v[i];
                }
            k[g] = uint4{v[0], v[1], v[2], v[3]};
        }
    };
    auto each_group = [&](auto use) {
#pragma unroll
        for (int g = 0; g < GROUPS; ++g) use(g, k[g]);
    };
    if (parts == 1) load(0);
    // Rows between that stay: those above the threshold on the decided bits, and the first `need` that equal it.  None: a threshold
    // between weights and KEY_STAYS
    uint32_t prefix = 0xffc00000u, mask = 0xffe00000u;
    int need = E.budget - D.S - E.recent;
    if (need > 0) {
        prefix = mask = 0;
        for (int pass = 0; pass < 3; ++pass) {
            const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0;
            const uint32_t bins = pass == 2 ? 1023u : 2047u;
            for (int i = tid; i < COPIES * PITCH / 4; i += EVICT_THREADS) reinterpret_cast<int4*>(hist)[i] = int4{0, 0, 0, 0};
            __syncthreads();
            for (int part = 0; part < parts; ++part) {
                if (parts > 1) load(part);
                const uint32_t own = uint32_t((lane & (COPIES - 1)) * PITCH), dust = uint32_t(COPIES * PITCH + lane);
                if (pass == 0 && first_row(part) >= D.S && first_row(part) + 64 * KPT <= tail)
                    each_group([&](int, const uint4& k4) {       // all rows are there, and none stays whatever its weight
                        const uint32_t k[4] = {k4.x, k4.y, k4.z, k4.w};
#pragma unroll
                        for (int i = 0; i < 4; ++i) atomicAdd(&hist[own + (k[i] >> 21)], 1);
                    });
                else if (pass == 0)
                    each_group([&](int, const uint4& k4) {
                        const uint32_t k[4] = {k4.x, k4.y, k4.z, k4.w};
#pragma unroll
                        for (int i = 0; i < 4; ++i) atomicAdd(&hist[k[i] + 1u > 1u ? own + (k[i] >> 21) : dust], 1);
                    });
                else
                    each_group([&](int, const uint4& k4) {
                        // few keys match: one atomic for the first of a lane's four (the lane's own dustbin if there is none), without a branch
                        const uint32_t k[4] = {k4.x, k4.y, k4.z, k4.w};
                        bool m[4], seen = false, more = false;
                        uint32_t at = dust;
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            m[i] = (k[i] & mask) == prefix;
                            more |= seen && m[i];
                            at = !seen && m[i] ? own + ((k[i] >> shift) & bins) : at;
                            m[i] = m[i] && seen;
                            seen |= (k[i] & mask) == prefix;
                        }
                        atomicAdd(&hist[at], 1);
                        if (__builtin_amdgcn_ballot_w64(more) != 0)
#pragma unroll
                            for (int i = 1; i < 4; ++i)
                                if (m[i]) atomicAdd(&hist[own + ((k[i] >> shift) & bins)], 1);
                    });
            }
            __syncthreads();
            const int top = EVICT_BINS - 1 - 2 * tid;
            int c0 = 0, c1 = 0;
#pragma unroll
            for (int i = 0; i < COPIES; ++i) {
                const int2 c = *reinterpret_cast<const int2*>(&hist[i * PITCH + top - 1]);
                c0 += c.y;
                c1 += c.x;
            }
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
            mask |= bins << shift;
            if (s_all) {                     // every key that equals it is wanted: above the number below it, in what is decided
                prefix -= mask & (0u - mask);
                need = 0;
                break;
            }
        }
    }
    int above = 0, equal = 0;                // of the rows before
    for (int part = 0; part < parts; ++part) {
        if (parts > 1) load(part);
        int na = 0, ne = 0;                  // of the wave
        each_group([&](int, const uint4& k4) {
            const uint32_t k[4] = {k4.x & mask, k4.y & mask, k4.z & mask, k4.w & mask};
#pragma unroll
            for (int i = 0; i < 4; ++i) na += __builtin_popcountll(__builtin_amdgcn_ballot_w64(k[i] > prefix));
            if (need > 0)
#pragma unroll
                for (int i = 0; i < 4; ++i) ne += __builtin_popcountll(__builtin_amdgcn_ballot_w64(k[i] == prefix));
        });
        __syncthreads();
        if (lane == 0) s_count[wave] = int2{na, ne};
        __syncthreads();
        int a = above, e = equal;
        {
            const int2 c = lane < WAVES ? s_count[lane] : int2{0, 0};
            const int sa = wave_iscan(c.x), se = wave_iscan(c.y);
            a += __builtin_amdgcn_readlane(sa, wave) - na;
            e += __builtin_amdgcn_readlane(se, wave) - ne;
            above += __builtin_amdgcn_readlane(sa, 63);
            equal += __builtin_amdgcn_readlane(se, 63);
        }
        const int r0 = first_row(part) + 4 * lane;
        each_group([&](int g, const uint4& k4) {
            const uint32_t k[4] = {k4.x & mask, k4.y & mask, k4.z & mask, k4.w & mask};
            int my_a = a, my_e = e;          // rows above, rows equal before the lane's first one
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint64_t m = __builtin_amdgcn_ballot_w64(k[i] > prefix);
                my_a = __builtin_amdgcn_mbcnt_hi(uint32_t(m >> 32), __builtin_amdgcn_mbcnt_lo(uint32_t(m), my_a));
                a += __builtin_popcountll(m);
            }
            if (need == 0) {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (k[i] > prefix) put(my_a++, r0 + 256 * g + i);
                return;
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint64_t m = __builtin_amdgcn_ballot_w64(k[i] == prefix);
                my_e = __builtin_amdgcn_mbcnt_hi(uint32_t(m >> 32), __builtin_amdgcn_mbcnt_lo(uint32_t(m), my_e));
                e += __builtin_popcountll(m);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const bool ia = k[i] > prefix, ie = k[i] == prefix;
                if (ia || (ie && my_e < need)) put(my_a + min(my_e, need), r0 + 256 * g + i);
                my_a += ia ? 1 : 0;
                my_e += ie ? 1 : 0;
            }
        });
    }
}
template <int KPT>
__global__ __launch_bounds__(EVICT_THREADS) void k_evict_select(Dims D, EvictArgs E, int32_t* __restrict__ keep) {
    const int unit = blockIdx.x, b = unit / D.Hkv, len = evict_len(E, b);
    if (E.lens_o && unit % D.Hkv == 0 && threadIdx.x == 0) E.lens_o[b] = min(len, E.budget);
    keep += int64_t(unit) * E.budget;
    select_rows<KPT>(D, E, unit, len, [&](int i, int r) { keep[i] = r; });
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

// 16 bytes per thread.  Bound by memory, which reads and writes at the rate of a copy: 4 x 8 heads, 8192 rows of 512 bytes, 52.8 us = 5.1 TB/s
// (58.3 through the caches; several rows per thread: 61).
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
    const int64_t e = int64_t(blockIdx.x) * 256 + threadIdx.x, i = e / lpr;
    if (i >= min(len, E.budget)) return;
    const int64_t at = b * D.ks[0] + h * D.ks[1] + e % lpr * Elem<T>::VEC;
    stream_store((z ? Vo : Ko) + at + i * D.ks[2], stream_load((z ? V : K) + at + keep[i] * D.ks[2]));
}

// One workgroup: 256 neighbouring rows of the new cache, of one (sequence, KV head, K or V), which are whole blocks of it; 16 codes of a
// row per lane.  List, rows and scales are a chain of three reads, so many rows are asked for at once: 8 x 8 heads,
// 8192 rows, 55 us = 4.9 TB/s (a block per workgroup: 119; through the caches the rows' next reader waits for the writes: 55 us here, but 87
// instead of 77 us there).
constexpr int EVICT_WG_ROWS = 256;
struct QuantMoveLds { float top[EVICT_WG_ROWS / 8], scale[EVICT_WG_ROWS / 16]; };
// By NT threads, `tid` of them: rows row0 .. of the new cache, `rows` of them, ROWS at most (none where not positive); from_row(i): the old
// cache's row for i of these.  All threads of the workgroup call.
template <int DH, int FMT, int NT, int ROWS, class Row>
__device__ __forceinline__ void move_quant_rows(const QuantDims& Q, const QuantDims& N, int z, int unit, int b, int h, int64_t row0, int rows, int tid,
                                                QuantMoveLds& sh, Row from_row) {
    constexpr int LPR = DH / 16, RPP = NT / LPR, PASSES = ROWS / RPP, WROWS = 64 / LPR;      // rows of a wave and pass: 8 or 16
    const int sub = tid % LPR, rg = tid / LPR;
    const uint8_t* src = (z ? Q.V : Q.K) + b * Q.st[0] + h * Q.st[1] + sub * 16;
    const float* scales = (z ? Q.Vs : Q.Ks) + int64_t(unit) * Q.nb;
    int from[PASSES];
    uint4 codes[PASSES];
    float scale[PASSES];
#pragma unroll
    for (int p = 0; p < PASSES; ++p) from[p] = rows > 0 ? from_row(min(p * RPP + rg, rows - 1)) : 0;      // rows past the end repeat the last one
#pragma unroll
    for (int p = 0; p < PASSES; ++p) {
        codes[p] = stream_load(src + from[p] * Q.st[2]);
        scale[p] = scales[from[p] >> Q.log_block];
    }
#pragma unroll
    for (int p = 0; p < PASSES; ++p) {
        float lo[8], hi[8], top = 0.0f;
        code_values<FMT>(uint2{as_loaded(codes[p].x), as_loaded(codes[p].y)}, lo);
        code_values<FMT>(uint2{as_loaded(codes[p].z), as_loaded(codes[p].w)}, hi);
#pragma unroll
        for (int i = 0; i < 8; ++i) top = fmaxf(top, fmaxf(fabsf(lo[i]), fabsf(hi[i])));
        top = wave_max(top * scale[p]);                                // a row past the end repeats the last one: its block's maximum is the same
        if ((tid & 63) == 0) sh.top[p * (NT / 64) + (tid >> 6)] = top;         // rows WROWS * (NT / 64 * p + wave) ..
    }
    __syncthreads();
    const int per = N.block / WROWS;                                   // such groups of rows in a block
    if (tid * N.block < rows) {
        float top = 0.0f;
        for (int i = 0; i < per; ++i) top = fmaxf(top, sh.top[tid * per + i]);
        const float s = quant_scale<FMT>(top);
        sh.scale[tid] = s;
        (z ? N.Vs : N.Ks)[int64_t(unit) * N.nb + (row0 >> N.log_block) + tid] = s;
    }
    __syncthreads();
    uint8_t* dst = (z ? N.V : N.K) + b * N.st[0] + h * N.st[1] + row0 * N.st[2] + sub * 16;
#pragma unroll
    for (int p = 0; p < PASSES; ++p) {
        const int r = p * RPP + rg;
        if (r >= rows) continue;
        // Exact for powers of two.  Beyond 2^127 where a row of zeros leaves a large scale for a block of zeros: a number all the same, for 0 * ratio
        // is to be 0 (a code that is not zero asks for 2^18 at most)
        const float ratio = fminf(scale[p] * (1.0f / sh.scale[r >> N.log_block]), 0x1p127f);
        uint4 c = codes[p];
        if (ratio != 1.0f) {
            float lo[8], hi[8];
            code_values<FMT>(uint2{as_loaded(c.x), as_loaded(c.y)}, lo);
            code_values<FMT>(uint2{as_loaded(c.z), as_loaded(c.w)}, hi);
            const uint2 a = make_codes<FMT>(lo, ratio), e = make_codes<FMT>(hi, ratio);
            c = uint4{a.x, a.y, e.x, e.y};
        }
        stream_store(dst + r * N.st[2], c);
    }
}
template <int DH, int FMT>
__global__ __launch_bounds__(256) void k_evict_quant(Dims D, EvictArgs E, QuantDims Q, const int32_t* __restrict__ keep, QuantDims N) {
    __shared__ QuantMoveLds sh;
    const int z = blockIdx.y, unit = blockIdx.z, b = unit / D.Hkv, h = unit % D.Hkv;
    const int len = evict_len(E, b);
    keep += int64_t(unit) * E.budget;
    if (z == 2) {
        evict_lists(E, unit, len, keep, blockIdx.x, gridDim.x);
        return;
    }
    const int64_t row0 = int64_t(blockIdx.x) * EVICT_WG_ROWS;
    const int rows = int(min(int64_t(EVICT_WG_ROWS), min(len, E.budget) - row0));
    if (rows <= 0) return;
    move_quant_rows<DH, FMT, 256, EVICT_WG_ROWS>(Q, N, z, unit, b, h, row0, rows, threadIdx.x, sh, [&](int i) { return keep[row0 + i]; });
}

// Short caches (EVICT_SHORT rows at most): every workgroup selects the rows of its unit for itself, keeps those that become rows row0 .. of
// the new cache in LDS, and moves them: one launch instead of two, which bound such calls, and no list in memory.  A workgroup takes as
// many rows as give each CU one (SHORT_PIECES pieces of 16 bytes of K at most), in 8 bits the largest block.
constexpr int EVICT_KPT = 8, EVICT_SHORT = EVICT_THREADS * EVICT_KPT, SHORT_CHUNK = 512, SHORT_PIECES = 8192, SHORT_QUANT_CHUNK = QUANT_MAX_BLOCK;
__device__ __forceinline__ int select_chunk(const Dims& D, const EvictArgs& E, int unit, int len, int row0, int chunk, int32_t* list) {
    if (E.lens_o && unit % D.Hkv == 0 && row0 == 0 && threadIdx.x == 0) E.lens_o[unit / D.Hkv] = min(len, E.budget);
    select_rows<EVICT_KPT>(D, E, unit, len, [&](int i, int r) {
        if (uint32_t(i - row0) < uint32_t(chunk)) list[i - row0] = r;
    });
    __syncthreads();
    const int rows = max(0, min(chunk, min(len, E.budget) - row0));
    const int64_t at = int64_t(unit) * E.cap;
    for (int i = threadIdx.x; i < rows; i += EVICT_THREADS) {
        E.acc_o[at + row0 + i] = E.acc[at + list[i]];
        if (E.pos) E.pos_o[at + row0 + i] = E.pos[at + list[i]];
    }
    for (int64_t i = min(len, E.budget) + int64_t(blockIdx.x) * EVICT_THREADS + threadIdx.x; i < E.cap; i += int64_t(gridDim.x) * EVICT_THREADS)
        E.acc_o[at + i] = 0.0f;
    return rows;
}
// strides and rows in 16-byte pieces.  Through the caches, which hold as much as moves here, so that the next attention finds it there: 32
// heads, 2048 of 4501 rows, 17.7 us, and 33.1 with the attention; past them 20.5 and 38.5.
__global__ __launch_bounds__(EVICT_THREADS) void k_evict_short(Dims D, EvictArgs E, const uint4* __restrict__ K, const uint4* __restrict__ V, int pieces,
                                                               int chunk, uint4* __restrict__ Ko, uint4* __restrict__ Vo) {
    __shared__ int32_t list[SHORT_CHUNK];
    const int unit = blockIdx.y, b = unit / D.Hkv, h = unit % D.Hkv, row0 = blockIdx.x * chunk;
    const int rows = select_chunk(D, E, unit, evict_len(E, b), row0, chunk, list);
    const int64_t at = b * D.ks[0] + h * D.ks[1];
    const int sub = threadIdx.x % pieces, step = EVICT_THREADS / pieces;
    for (int i = threadIdx.x / pieces; i < rows; i += 2 * step) {
        const int j = min(i + step, rows - 1);               // the last row twice rather than loads in a branch
        const int64_t a = at + list[i] * D.ks[2] + sub, c = at + list[j] * D.ks[2] + sub;
        const uint4 k0 = K[a], v0 = V[a], k1 = K[c], v1 = V[c];
        uint4 *Kn = Ko + at + row0 * D.ks[2] + sub, *Vn = Vo + at + row0 * D.ks[2] + sub;
        Kn[i * D.ks[2]] = k0;
        Vn[i * D.ks[2]] = v0;
        if (i + step < rows) {
            Kn[j * D.ks[2]] = k1;
            Vn[j * D.ks[2]] = v1;
        }
    }
}
template <int DH, int FMT>
__global__ __launch_bounds__(EVICT_THREADS) void k_evict_quant_short(Dims D, EvictArgs E, QuantDims Q, QuantDims N) {
    __shared__ int32_t list[SHORT_QUANT_CHUNK];
    __shared__ QuantMoveLds sh[2];
    const int unit = blockIdx.y, b = unit / D.Hkv, h = unit % D.Hkv, row0 = blockIdx.x * SHORT_QUANT_CHUNK;
    const int rows = select_chunk(D, E, unit, evict_len(E, b), row0, SHORT_QUANT_CHUNK, list);
    const int z = __builtin_amdgcn_readfirstlane(threadIdx.x / (EVICT_THREADS / 2));
    move_quant_rows<DH, FMT, EVICT_THREADS / 2, SHORT_QUANT_CHUNK>(Q, N, z, unit, b, h, row0, rows, threadIdx.x % (EVICT_THREADS / 2), sh[z],
                                                                   [&](int i) { return list[i]; });
}

size_t cache_evict_ws_bytes(const Dims& D, int budget) { return align256(size_t(D.B) * D.Hkv * budget * 4); }
bool cache_evict_grid_fits(const Dims&, int len, int budget) { return len <= 1 << 30 && grid_fits(int64_t(budget) / 8 + 1, 256); }

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

// One launch where a workgroup has all keys of its unit in registers and every workgroup a CU of its own, so that the selections that are
// made several times cost no time.  bf16, d 128, one launch and two: 8 heads, 4501 rows of which 2048 stay 10.4 and 13.0 us, 32 heads (256
// workgroups) 19.4 and 22.6, 256 heads, 500 of 1000 rows (256) 36 and 39, 64 heads, 4501 rows (256, of 512 rows) 37 and 34, 32 heads, 6000 of 8192
// rows (384) 56 and 43; 8 bits, 4 heads, 2048 of 8111 rows, 10.1 and 12.6.  With 256 workgroups it is the length of their selections that
// decides, by 8 % to either side: no rule by length is made of that.
static bool short_eviction(const Dims& D, int len, int rows, int chunk) {
    return len <= EVICT_SHORT && (int64_t(rows) + chunk - 1) / chunk * D.B * D.Hkv <= 256;
}

static void launch_select(const Dims& D, const EvictArgs& E, int32_t* keep, hipStream_t st) {
    const int per = (E.len + EVICT_THREADS - 1) / EVICT_THREADS;      // keys per thread
    LRSA_TIMED_LAUNCH("k_evict_select", st, (per <= 4 ? k_evict_select<4> : per <= 8 ? k_evict_select<8> : per <= 16 ? k_evict_select<16> :
                      k_evict_select<32>), dim3(D.B * D.Hkv), dim3(EVICT_THREADS), 0, st, D, E, keep);
}

template <typename T>
static hipError_t run_evict(const Dims& D, const EvictArgs& E, const void* K, const void* V, void* Ko, void* Vo, int32_t* keep, hipStream_t st) {
    const int rows = E.len < E.budget ? E.len : E.budget;
    const int pieces = D.d / Elem<T>::VEC, step = EVICT_THREADS / pieces;      // 16-byte pieces of a row; rows that move at once
    const int64_t share = (int64_t(rows) * D.B * D.Hkv + 255) / 256, up = (share + step - 1) / step * step;
    const int most = SHORT_PIECES / pieces < SHORT_CHUNK ? SHORT_PIECES / pieces : SHORT_CHUNK, chunk = up < step ? step : up < most ? int(up) : most;
    if (short_eviction(D, E.len, rows, chunk)) {
        Dims P = D;
        for (int i = 0; i < 3; ++i) P.ks[i] = D.ks[i] / Elem<T>::VEC;
        LRSA_TIMED_LAUNCH("k_evict_short", st, k_evict_short, dim3(rows ? (rows + chunk - 1) / chunk : 1, D.B * D.Hkv), dim3(EVICT_THREADS), 0, st, P, E,
                          (const uint4*)K, (const uint4*)V, pieces, chunk, (uint4*)Ko, (uint4*)Vo);
        return hipGetLastError();
    }
    launch_select(D, E, keep, st);
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
    if (short_eviction(D, max_len, rows, SHORT_QUANT_CHUNK)) {
        const dim3 grid(rows ? (rows + SHORT_QUANT_CHUNK - 1) / SHORT_QUANT_CHUNK : 1, D.B * D.Hkv);
#define LRSA_EVICT_SHORT(DH_, FMT_) \
    LRSA_TIMED_LAUNCH("k_evict_quant_short", st, (k_evict_quant_short<DH_, FMT_>), grid, dim3(EVICT_THREADS), 0, st, D, E, Q, N)
        if (Q.fmt == QUANT_INT8) {
            if (D.d == 64) LRSA_EVICT_SHORT(64, QUANT_INT8); else LRSA_EVICT_SHORT(128, QUANT_INT8);
        } else {
            if (D.d == 64) LRSA_EVICT_SHORT(64, QUANT_E4M3); else LRSA_EVICT_SHORT(128, QUANT_E4M3);
        }
#undef LRSA_EVICT_SHORT
        return hipGetLastError();
    }
    launch_select(D, E, keep, st);
    const dim3 grid(unsigned(rows ? (rows + EVICT_WG_ROWS - 1) / EVICT_WG_ROWS : 1), 3, D.B * D.Hkv);
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
