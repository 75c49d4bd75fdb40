// The inference-time cache in 8 bits: rows written into it, rows read back, attention of a few query tokens over it.  Codes
// and scales: quant_block.h.  Every sequence has a length of its own, in device memory, so that a captured graph can be
// replayed while the sequences grow.
//
// k_append_quant      new rows into the blocks of the cache that they belong to
// k_read_quant        rows of the cache as values
// k_decode_quant      attention of the query rows of a KV group over a slice of the cache rows, on the matrix cores
// k_decode_quant_short  the same over whole short caches, with everything that follows, in one launch
// k_quant_combine     merges the slices; with accumulated weights the same workgroup kinds as k_decode_combine_acc
#include "decode_merge.h"
#include "mfma_tiles.h"
#include "quant_block.h"

namespace lrsa {

constexpr int QUANT_THREADS = 256;

__device__ __forceinline__ int seq_len(const int32_t* lens, int b, int most) { return max(0, min(lens[b], most)); }

// ------------------------------------------------------------------------------------ writing
// One workgroup: one block of one (sequence, KV head, K or V) that new rows fall into.  A lane takes 8 channels of a row, all
// of the block's new rows stay in registers between the maximum and the codes.  A block that holds older rows keeps its
// scale where that is large enough; where it is not, the scale grows and the older codes follow.  Bound by memory: 32K rows of 8 heads,
// bf16, 38.7 us = 5.1 TB/s (with a branch around each row's load, at whose end the compiler waits for it, 42.2; through the caches 50.5).
template <typename T, int DH, int FMT, int PASSES>
__global__ __launch_bounds__(QUANT_THREADS) void k_append_quant(Dims D, QuantDims Q, const T* __restrict__ K, const T* __restrict__ V, int tokens,
                                                                const int32_t* __restrict__ lens, const int32_t* __restrict__ counts) {
    constexpr int LPR = DH / 8, RPP = QUANT_THREADS / LPR;      // PASSES * RPP rows: a block at least
    __shared__ float sm[QUANT_THREADS / 64];
    const int z = blockIdx.y, bh = blockIdx.z, b = bh / D.Hkv, h = bh % D.Hkv;
    const int len = seq_len(lens, b, D.n);
    const int count = counts ? max(0, min(counts[b], tokens)) : tokens;
    const int64_t end = min(int64_t(len) + count, int64_t(D.n));
    const int64_t j = (len >> Q.log_block) + int64_t(blockIdx.x), row0 = j << Q.log_block;
    if (max(row0, int64_t(len)) >= end) return;               // no new row in this block: also where count is 0 or the cache full
    const int r0 = int(max(row0, int64_t(len)) - row0), r1 = int(min(end - row0, int64_t(Q.block)));      // new rows of the block
    const int sub = threadIdx.x % LPR, rg = threadIdx.x / LPR;
    const T* src = (z ? V : K) + b * D.ks[0] + h * D.ks[1] + (row0 - len) * D.ks[2] + sub * 8;
    uint8_t* dst = (z ? Q.V : Q.K) + b * Q.st[0] + h * Q.st[1] + row0 * Q.st[2] + sub * 8;
    float* scale = (z ? Q.Vs : Q.Ks) + int64_t(bh) * Q.nb + j;
    const float before = r0 > 0 ? *scale : 0.0f;

    float v[PASSES][8], top = 0.0f;
#pragma unroll
    for (int p = 0; p < PASSES; ++p)
        stream_load8(src + min(max(p * RPP + rg, r0), r1 - 1) * D.ks[2], v[p]);      // a row of the block that is not new: the nearest new one again
#pragma unroll
    for (int p = 0; p < PASSES; ++p)
#pragma unroll
        for (int i = 0; i < 8; ++i) top = fmaxf(top, fabsf(v[p][i]));
    top = block_max<QUANT_THREADS>(top, sm);
    if (top > QUANT_LARGEST<FMT>)
#pragma unroll
        for (int p = 0; p < PASSES; ++p)
#pragma unroll
            for (int i = 0; i < 8; ++i) v[p][i] = __builtin_amdgcn_fmed3f(v[p][i], -QUANT_LARGEST<FMT>, QUANT_LARGEST<FMT>);
    const float s = fmaxf(quant_scale<FMT>(top), before);
    const float inv = 1.0f / s;
    if (s > before) {
        for (int r = rg; r < r0; r += RPP) {
            uint2* at = reinterpret_cast<uint2*>(dst + r * Q.st[2]);
            float c[8];
            code_values<FMT>(*at, c);
            *at = make_codes<FMT>(c, before / s);
        }
        if (threadIdx.x == 0) *scale = s;
    }
#pragma unroll
    for (int p = 0; p < PASSES; ++p) {
        const int r = p * RPP + rg;
        if (r >= r0 && r < r1) *reinterpret_cast<uint2*>(dst + r * Q.st[2]) = make_codes<FMT>(v[p], inv);
    }
}

// ------------------------------------------------------------------------------------ reading
template <typename T, int DH, int FMT>
__global__ __launch_bounds__(QUANT_THREADS) void k_read_quant(Dims D, QuantDims Q, const int32_t* __restrict__ lens, int rows,
                                                              const int32_t* __restrict__ first, T* __restrict__ K, T* __restrict__ V) {
    constexpr int LPR = DH / 8;
    const int z = blockIdx.y, bh = blockIdx.z, b = bh / D.Hkv, h = bh % D.Hkv;
    const int64_t e = int64_t(blockIdx.x) * QUANT_THREADS + threadIdx.x;
    const int64_t i = e / LPR;
    const int sub = int(e % LPR);
    if (i >= rows) return;
    const int64_t r = (first ? first[b] : 0) + i;
    float v[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
    if (r >= 0 && r < seq_len(lens, b, D.n)) {
        code_values<FMT>(*reinterpret_cast<const uint2*>((z ? Q.V : Q.K) + b * Q.st[0] + h * Q.st[1] + r * Q.st[2] + sub * 8), v);
        const float s = (z ? Q.Vs : Q.Ks)[int64_t(bh) * Q.nb + (r >> Q.log_block)];
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] *= s;
    }
    store8((z ? V : K) + b * D.ks[0] + h * D.ks[1] + i * D.ks[2] + sub * 8, v);
}

// ------------------------------------------------------------------------------------ attention
// How the rows are cut into slices, W workgroups being what runs at once.
//   even  Where all sequences of max_len rows give no more than W slices of 4 tiles, a slice has that length: workgroup
//         (b * Hkv + h) * splits + s takes slice s, and exits where the sequence is shorter.
//   else  The sequences' lengths are known on the device only, so every workgroup takes them from there: with t_b tiles in
//         sequence b, a slice is sum(t_b) * Hkv / W tiles if that gives W slices at most (the last of a sequence is short), or
//         sum(t_b) * Hkv / (W - B * Hkv), which always does (estimates in floating point that are never too small).  Slices of
//         equal length then begin and end together however the lengths are mixed: 8 requests of 11K to 32K rows, 8 KV heads, 78 us,
//         with slices by max_len 88.  Slice s of KV head h of sequence b is workgroup Hkv * (slices of the sequences before) + h *
//         n_b + s.
constexpr int QT = 32;                       // rows of a tile: per wave and step
struct QuantSlices {
    int splits;                              // even: slices per unit, else 0
    int most, least;                         // W; the least tiles of a slice
    float share, safe;                       // Hkv / W, Hkv / (W - B * Hkv), rounded up
};
struct QuantSeq { int base, n; };            // of one sequence: workgroup of its first slice, slices per KV head

// The sequences' lengths, of the first 64 one per lane
struct SeqLens {
    const int32_t* lens;
    int most, mine;
    __device__ __forceinline__ SeqLens(const Dims& D, const int32_t* l, int max_len) : lens(l), most(max_len) {
        const int lane = threadIdx.x & 63;
        mine = lane < D.B ? seq_len(l, lane, max_len) : 0;
    }
    __device__ __forceinline__ int of(int b) const { return b < 64 ? __builtin_amdgcn_readlane(mine, b) : seq_len(lens, b, most); }
};
// wave-wide; `each` gets the tiles of the sequences in groups of 64, one per lane, until it returns true
template <class Fn>
__device__ __forceinline__ void each_sequence(const Dims& D, const SeqLens& L, Fn each) {
    const int lane = threadIdx.x & 63;
    for (int b0 = 0; b0 < D.B; b0 += 64) {
        const int b = b0 + lane;
        if (each(b, ((b0 == 0 ? L.mine : b < D.B ? seq_len(L.lens, b, L.most) : 0) + QT - 1) / QT)) return;
    }
}
__device__ __forceinline__ int tiles_sum(int v) { return __builtin_amdgcn_readlane(wave_iscan(v), 63); }
__device__ __forceinline__ int slice_tiles(const Dims& D, const SeqLens& L, const QuantSlices& S) {
    int sum = 0, count = 0;
    each_sequence(D, L, [&](int, int t) { sum += t; return false; });
    const float all = float(tiles_sum(sum));
    const int per = max(int(all * S.share) + 1, S.least);
    each_sequence(D, L, [&](int, int t) { count += (t + per - 1) / per; return false; });
    return __builtin_amdgcn_readfirstlane(int64_t(tiles_sum(count)) * D.Hkv <= S.most ? per : max(int(all * S.safe) + 1, S.least));
}

// One workgroup: the query rows of one KV group x a slice of the cache rows, as k_decode_mfma.  A query row ("column") is
// (head of the group, token): q is [B, Hq, T, d], so the columns of a unit are neighbours.  Lane l, c = l % 16, q4 = l / 16,
// v_mfma_f32_16x16x32_bf16:
//   S = K Q^T   row m of block kb is tile row 16*kb + m.  The contraction over the channels may take them in any order: the
//               lane reads 16 neighbouring bytes (channels 64*i + 16*q4 ..), two instructions' worth.  It then holds the
//               logits of rows 4*q4 .. +3 and 16 + 4*q4 .. +3 of column c, which are the k-slots of its B operand below
//   O^T += V^T P^T   the lane reads DH/16 neighbouring channels of those rows and transposes that block
// Codes have at most 8 significant bits, so both operands are exact in bf16 without their scales; the scale of K multiplies
// the logit, that of V the weight, in fp32 (4 such rows share a block: blocks are multiples of 16).  Queries of fp32 enter as
// three bf16 terms, which hold all 24 bits, and so do the weights.
// A wave takes 16 * NG columns.  If these are all, the 4 waves take the tiles in turn (SOLE): every code is read by one wave of the
// chip, and past the caches (PAST) where the cache is as large as the Infinity Cache (256 MB), which would keep little of it until the next call.  8 KV
// heads of 4 query heads, us per call on the same cache, through and past the caches: 40 MB 14.6 and 16.2, 159 MB 32.5 and 35.3, 269 MB
// 47.6 and 51.9, 537 MB 102 and 95; on others in turn: 16.2 and 16.8, 37.8 and 36.5, 54.5 and 52.3, 102 and 95 (NG = 2: decode_quant_kernel).  Where there are more, `groups` (2 or 4) waves take the same tile, so that its codes come from memory once, and
// beyond 4 times as many columns the slice is walked again.  NG = 2 halves the unpacking of codes, which bounds many columns (8 requests of
// 32K rows, 20 columns: 107 us, with NG = 1 128; 64 columns: 171 and 212); it needs registers that fp32 queries of 128 channels do not
// leave, and long walks.
// The next tile's loads are in flight while a tile is used.  They are issued in every turn (the last one asks for its own tile
// again, from the caches): loads in a branch make the compiler wait for all of them at its end, the next tile's too.
constexpr float NO_WEIGHT = -1e30f;          // running maximum before the first visible row: finite, so that differences are
template <int DH> struct QPiece { typedef u32x2 type; };
template <> struct QPiece<64> { typedef uint32_t type; };
template <int DH> struct QuantTile {
    u32x4 k[2][DH / 64];
    typename QPiece<DH>::type v[8];
    float ks[2], vs[2];
};
struct QuantRows {                           // of one unit
    const uint8_t *K, *V;
    const float *Ks, *Vs;
    int64_t st;
    int log_block;
};
template <bool PAST, typename V>
__device__ __forceinline__ V load_codes(const uint8_t* p) {
    if constexpr (PAST) return __builtin_nontemporal_load(reinterpret_cast<const V*>(p));
    return *reinterpret_cast<const V*>(p);
}

// 4 codes -> two bf16 pairs
template <int FMT>
__device__ __forceinline__ void codes_bf16(uint32_t w, uint32_t& lo, uint32_t& hi) {
    if constexpr (FMT == QUANT_INT8) {
        const float a = float(int8_t(w)), b = float(int8_t(w >> 8)), c = float(int8_t(w >> 16)), d = float(int8_t(w >> 24));
        lo = __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u);
        hi = __builtin_amdgcn_perm(__float_as_uint(d), __float_as_uint(c), 0x07060302u);
    } else {
        lo = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, false));
        hi = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, true));
    }
}
// 4 codes of a row and the 4 below them -> for each of the 4 columns a bf16 pair (upper row first)
template <int FMT>
__device__ __forceinline__ void codes_bf16_columns(uint32_t w0, uint32_t w1, uint32_t (&col)[4]) {
    if constexpr (FMT == QUANT_INT8) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            col[i] = __builtin_amdgcn_perm(__float_as_uint(float(int8_t(w1 >> (8 * i)))), __float_as_uint(float(int8_t(w0 >> (8 * i)))), 0x07060302u);
    } else {
        const uint32_t lo = __builtin_amdgcn_perm(w1, w0, 0x05010400u), hi = __builtin_amdgcn_perm(w1, w0, 0x07030602u);
        codes_bf16<FMT>(lo, col[0], col[1]);
        codes_bf16<FMT>(hi, col[2], col[3]);
    }
}

// r: the tile's first row (wave-uniform), of rows up to `last`: rows past the end repeat it, their weight will be 0
template <int DH, bool PAST>
__device__ __forceinline__ void load_quant_tile(QuantTile<DH>& t, const QuantRows& R, int r, int q4, int c, int last) {
    const uint8_t *K = R.K + r * R.st, *V = R.V + r * R.st;
    const uint32_t most = min(last - r, QT - 1), st = uint32_t(R.st);        // rows are less than 2^24 bytes apart
    auto off = [&](uint32_t row) { return __umul24(min(row, most), st); };
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
        const uint32_t row = off(16 * kb + c) + q4 * 16;
#pragma unroll
        for (int i = 0; i < DH / 64; ++i) t.k[kb][i] = load_codes<PAST, u32x4>(K + row + i * 64);
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) t.v[j] = load_codes<PAST, typename QPiece<DH>::type>(V + (off(4 * q4 + j % 4 + j / 4 * 16) + c * (DH / 16)));
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const uint32_t block = (r + min(uint32_t(16 * i + 4 * q4), most)) >> R.log_block;
        t.ks[i] = R.Ks[block];
        t.vs[i] = R.Vs[block];
    }
}

// NG groups of 16 columns.  seen: rows from the lane's first one on that its column sees; ACC: the logits go to `out`.
// o is in units of 2^(unit - 127), the power of two of the largest scale of V so far (1 at most, so that no weight gets smaller for it): a weight
// times a scale of 2^-110 or less has terms below the least bf16 number (2^-133), and would keep 14 bits at 2^-120.  A tile's scales are
// the same in all lanes (each 16 rows share one), so the unit is a scalar.  It costs 0.2 us in short
// caches, 1 % where the unpacking of codes binds (64 columns over 4 x 40K rows 131.1 and 132.5 us), nothing where memory does.
constexpr uint32_t LEAST_UNIT = 127 - 120;
__device__ __forceinline__ float unit_value(uint32_t unit) { return __uint_as_float(unit << 23); }
template <int DH, int FMT, int TERMS, bool ACC, int NG>
__device__ __forceinline__ void use_quant_tile(float (&m)[NG], float (&l)[NG], f32x4 (&o)[NG][DH / 16], uint32_t& unit, const QuantTile<DH>& t,
                                               const bf16x8 (&qf)[NG][TERMS][DH / 32], const int (&seen)[NG], float c2, LogitBuffer (&out)[NG]) {
    f32x4 s[NG][2];
#pragma unroll
    for (int g = 0; g < NG; ++g) s[g][0] = s[g][1] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int kk = 0; kk < DH / 32; ++kk)
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
            const u32x4 w = t.k[kb][kk / 2];
            uint32_t a[4];
            codes_bf16<FMT>(as_loaded(kk % 2 ? w.z : w.x), a[0], a[1]);
            codes_bf16<FMT>(as_loaded(kk % 2 ? w.w : w.y), a[2], a[3]);
            const bf16x8 kf = __builtin_bit_cast(bf16x8, a);
#pragma unroll
            for (int g = 0; g < NG; ++g)
#pragma unroll
                for (int i = TERMS - 1; i >= 0; --i) s[g][kb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[g][i][kk], s[g][kb], 0, 0, 0);
        }
    const float c2s[2] = {c2 * t.ks[0], c2 * t.ks[1]};
    const float top = __builtin_amdgcn_fmed3f(fmaxf(fabsf(t.vs[0]), fabsf(t.vs[1])), unit_value(LEAST_UNIT), 1.0f);
    const uint32_t now = max(unit, uint32_t(__builtin_amdgcn_readfirstlane(__float_as_uint(top))) >> 23);
    if (now != unit) {
        const float a = unit_value(127 + unit - now);
#pragma unroll
        for (int g = 0; g < NG; ++g)
#pragma unroll
            for (int e = 0; e < DH / 16; ++e) o[g][e] *= a;
        unit = now;
    }
    const float vs[2] = {t.vs[0] * unit_value(254 - unit), t.vs[1] * unit_value(254 - unit)};
    bf16x8 term[NG][3];
#pragma unroll
    for (int g = 0; g < NG; ++g) {
        float p[8], mx = NO_WEIGHT;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            p[j] = j % 4 + j / 4 * 16 < seen[g] ? s[g][j >> 2][j & 3] * c2s[j >> 2] : -INFINITY;
            mx = fmaxf(mx, p[j]);
        }
        if constexpr (ACC) keep_logits(out[g], p, [](int j) { return 4 * int(threadIdx.x >> 4 & 3) + j % 4 + j / 4 * 16; });
        lanes_u32x2 x = pair32(__float_as_uint(mx));
        mx = fmaxf(__uint_as_float(x.x), __uint_as_float(x.y));
        x = pair16(__float_as_uint(mx));
        mx = fmaxf(__uint_as_float(x.x), __uint_as_float(x.y));
        if (__builtin_amdgcn_ballot_w64(mx > m[g]) != 0) {
            const float mn = fmaxf(m[g], mx), a = __builtin_amdgcn_exp2f(m[g] - mn);
            m[g] = mn;
            l[g] *= a;
#pragma unroll
            for (int e = 0; e < DH / 16; ++e) o[g][e] *= a;
        }
        f32x8 w;
        float ps = 0.0f;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float e = __builtin_amdgcn_exp2f(p[j] - m[g]);
            ps += e;
            w[j] = e * vs[j >> 2];
        }
        l[g] += ps;
#pragma unroll
        for (int i = 0; i < 3; ++i) {
            term[g][i] = __builtin_convertvector(w, bf16x8);
            w -= __builtin_convertvector(term[g][i], f32x8);
        }
    }
#pragma unroll
    for (int e0 = 0; e0 < DH / 16; e0 += 4) {
        uint32_t col[4][4];                  // [pair of rows][column]
#pragma unroll
        for (int i = 0; i < 4; ++i)
            codes_bf16_columns<FMT>(as_loaded(reinterpret_cast<const uint32_t*>(&t.v[2 * i])[e0 / 4]),
                                    as_loaded(reinterpret_cast<const uint32_t*>(&t.v[2 * i + 1])[e0 / 4]), col[i]);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const uint32_t a[4] = {col[0][e], col[1][e], col[2][e], col[3][e]};
            const bf16x8 av = __builtin_bit_cast(bf16x8, a);
#pragma unroll
            for (int g = 0; g < NG; ++g)
#pragma unroll
                for (int i = 2; i >= 0; --i) o[g][e0 + e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(av, term[g][i], o[g][e0 + e], 0, 0, 0);
        }
    }
}

// the query fragment of 8 channels as TERMS bf16 terms
__device__ __forceinline__ void query_terms(const bf16_t* q, bf16x8 (&f)[1]) { f[0] = *reinterpret_cast<const bf16x8*>(q); }
__device__ __forceinline__ void query_terms(const float* q, bf16x8 (&f)[3]) {
    float v[8];
    load8(q, v);
    f32x8 w;
#pragma unroll
    for (int j = 0; j < 8; ++j) w[j] = v[j];
#pragma unroll
    for (int i = 0; i < 3; ++i) {
        f[i] = __builtin_convertvector(w, bf16x8);
        w -= __builtin_convertvector(f[i], f32x8);
    }
}

template <typename T> constexpr int Q_TERMS = sizeof(T) == 2 ? 1 : 3;
template <typename T, int DH> constexpr int MOST_GROUPS = sizeof(T) == 2 || DH == 64 ? 2 : 1;      // NG

template <typename T, int DH, int FMT, int NG, bool SOLE, bool PAST, bool ACC>
__global__ __launch_bounds__(DEC_THREADS, 2) void k_decode_quant(Dims D, QuantDims Q, const T* __restrict__ q, int tokens, const int32_t* __restrict__ lens,
                                                                 int max_len, QuantSlices S, QuantSeq* __restrict__ seqs, float* __restrict__ part,
                                                                 float* __restrict__ logits, int64_t lrows, int pitch) {
    constexpr int CPL = DH / 16, LROW = DH + 4, TERMS = Q_TERMS<T>, REC = DH + 2, CW = 16 * NG;       // CW: columns of a wave
    constexpr int WAVE_FLOATS = ACC && LOGIT_FLOATS > CW * LROW ? LOGIT_FLOATS : CW * LROW;          // a wave's logits, then its output
    __shared__ __attribute__((aligned(16))) float sBuf[DEC_WAVES][WAVE_FLOATS];
    __shared__ float sM[DEC_WAVES][CW], sL[DEC_WAVES][CW];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), c = lane & 15, q4 = lane >> 4;
    const int wg = blockIdx.x;
    const SeqLens L(D, lens, max_len);
    int b = -1, h, r0, per;
    if (S.splits) {
        const int unit = wg / S.splits;
        b = unit / D.Hkv;
        h = unit % D.Hkv;
        per = S.least;
        r0 = wg % S.splits * per * QT;
    } else {
        // the sequence of this workgroup; the first workgroup notes all of them for the merge
        int first = 0, n = 1, before = 0;
        per = slice_tiles(D, L, S);
        each_sequence(D, L, [&](int bb, int t) {
            const int mine = (t + per - 1) / per, upto = before + D.Hkv * wave_iscan(mine);
            if (wg == 0 && wave == 0 && bb < D.B) seqs[bb] = QuantSeq{upto - D.Hkv * mine, mine};
            const uint64_t at = __builtin_amdgcn_ballot_w64(wg >= upto - D.Hkv * mine && wg < upto);
            if (at != 0 && b < 0) {
                const int l = __builtin_ctzll(at);
                b = (bb - lane) + l;
                n = __builtin_amdgcn_readlane(mine, l);
                first = __builtin_amdgcn_readlane(upto, l) - D.Hkv * n;
            }
            before = __builtin_amdgcn_readlane(upto, 63);
            return b >= 0 && wg != 0;
        });
        if (b < 0) return;
        b = __builtin_amdgcn_readfirstlane(b);
        h = (wg - first) / n;
        r0 = (wg - first) % n * per * QT;
    }
    const int bh = b * D.Hkv + h, len = L.of(b), r1 = min(len, r0 + per * QT);
    if (r0 >= r1) return;                                    // an empty slice: the merge does not ask for it
    const int64_t head = b * Q.st[0] + h * Q.st[1];
    const QuantRows R = {Q.K + head, Q.V + head, Q.Ks + int64_t(bh) * Q.nb, Q.Vs + int64_t(bh) * Q.nb, Q.st[2], Q.log_block};
    const float c2 = D.scale * 1.4426950408889634f;          // logits in log2 units
    const int cols = D.G * tokens, groups = SOLE ? 1 : cols <= 2 * CW ? 2 : 4, ways = DEC_WAVES / groups;
    const int64_t col0 = int64_t(bh) * cols;                 // query rows of the units before

    for (int c0 = 0; c0 < cols; c0 += CW * groups) {
        const int g0 = c0 + CW * (wave % groups), gn = min(CW, cols - g0);      // of this wave: none where not positive
        float m[NG], l[NG];
        f32x4 o[NG][CPL];
        uint32_t unit = LEAST_UNIT;
#pragma unroll
        for (int g = 0; g < NG; ++g) {
            m[g] = NO_WEIGHT;
            l[g] = 0.0f;
#pragma unroll
            for (int e = 0; e < CPL; ++e) o[g][e] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        }
        const int step = ways * QT;
        int r = r0 + wave / groups * QT;
        if (gn > 0 && r < r1) {
            const int end = r + (r1 - 1 - r) / step * step;      // the wave's last tile
            auto load = [&](QuantTile<DH>& t, int row) { load_quant_tile<DH, PAST>(t, R, min(row, end), q4, c, r1 - 1); };
            QuantTile<DH> A, B;
            load(A, r);
            bf16x8 qf[NG][TERMS][DH / 32];
            int vis[NG];                                         // rows that the column sees, none where that is not positive
            LogitBuffer out[NG] = {};
#pragma unroll
            for (int g = 0; g < NG; ++g) {
                const int col = g0 + min(16 * g + c, gn - 1);
                vis[g] = min(r1, len - tokens + 1 + col % tokens) - 4 * q4;
                const T* qrow = q + (col0 + col) * DH;
#pragma unroll
                for (int kk = 0; kk < DH / 32; ++kk) {
                    bf16x8 f[TERMS];
                    query_terms(qrow + (kk / 2) * 64 + q4 * 16 + (kk % 2) * 8, f);
#pragma unroll
                    for (int i = 0; i < TERMS; ++i) qf[g][i][kk] = f[i];
                }
                if constexpr (ACC)
                    out[g] = logit_buffer(sBuf[wave] + g * (LOGIT_FLOATS / NG), LOGIT_FLOATS / NG,
                                          logits + (int64_t(bh) * lrows + r) * pitch + g0 + 16 * g, pitch, max(0, min(16, gn - 16 * g)), step);
            }
            auto use = [&](const QuantTile<DH>& t) {
                int seen[NG];
#pragma unroll
                for (int g = 0; g < NG; ++g) seen[g] = vis[g] - r;
                use_quant_tile<DH, FMT, TERMS, ACC, NG>(m, l, o, unit, t, qf, seen, c2, out);
            };
            for (;;) {
                load(B, r + step);
                use(A);
                if ((r += step) >= r1) break;
                load(A, r + step);
                use(B);
                if ((r += step) >= r1) break;
            }
            if constexpr (ACC)
#pragma unroll
                for (int g = 0; g < NG; ++g) flush_logits(out[g]);
        }
#pragma unroll
        for (int g = 0; g < NG; ++g) {
            lanes_u32x2 x = pair32(__float_as_uint(l[g]));
            l[g] = __uint_as_float(x.x) + __uint_as_float(x.y);
            x = pair16(__float_as_uint(l[g]));
            l[g] = __uint_as_float(x.x) + __uint_as_float(x.y);
            const int cw = 16 * g + c;
            if (cw < gn) {
                if (q4 == 0) { sM[wave][cw] = m[g]; sL[wave][cw] = l[g]; }
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int e = 0; e < CPL; e += 4)
                        *reinterpret_cast<f32x4*>(&sBuf[wave][cw * LROW + (4 * q4 + i) * CPL + e]) =
                            f32x4{o[g][e][i], o[g][e + 1][i], o[g][e + 2][i], o[g][e + 3][i]} * unit_value(unit);
            }
        }
        __syncthreads();
        // column g of the walk is in the waves g / CW, + groups, ...
        for (int e = tid; e < min(CW * groups, cols - c0) * DH; e += DEC_THREADS) {
            const int g = e / DH, ch = e % DH, w0 = g / CW, gc = g % CW;
            float mm = sM[w0][gc], ll = sL[w0][gc], oo = sBuf[w0][gc * LROW + ch];
            for (int w = w0 + groups; w < DEC_WAVES; w += groups) {
                float a, b2;
                merge_state(mm, ll, sM[w][gc], sL[w][gc], a, b2);
                oo = oo * a + sBuf[w][gc * LROW + ch] * b2;
            }
            float* dst = part + (int64_t(wg) * cols + c0 + g) * REC;
            dst[2 + ch] = oo;
            if (ch == 0) { dst[0] = mm; dst[1] = ll; }
        }
        __syncthreads();
    }
}

// Short caches (SHORT_ROWS rows at most, 16 columns): one workgroup per unit, whose 8 waves take all tiles, merge, and write O, lse and
// the accumulated weights.  A call is one launch, which bounds it (8.2 us, 11 with slices and their merge, call after call: 1 request
// of 777 rows, 12 heads of 64 on 2); but a unit's rows pass through one CU, where slices would spread few units over many.  See
// short_cache for where that costs more than the launch.
constexpr int SHORT_WAVES = 8, SHORT_TILES = 4, SHORT_ROWS = SHORT_WAVES * SHORT_TILES * QT;
template <typename T, int DH, int FMT, bool ACC>
__global__ __launch_bounds__(64 * SHORT_WAVES) void k_decode_quant_short(Dims D, QuantDims Q, const T* __restrict__ q, int tokens,
                                                                         const int32_t* __restrict__ lens, int max_len, T* __restrict__ O,
                                                                         float* __restrict__ lse, AccArgs A) {
    constexpr int CPL = DH / 16, LROW = DH + 4, TERMS = Q_TERMS<T>, THREADS = 64 * SHORT_WAVES, LOGITS = SHORT_TILES * QT * 16;
    __shared__ __attribute__((aligned(16))) float sO[SHORT_WAVES][16 * LROW];
    __shared__ __attribute__((aligned(16))) float sLogit[ACC ? SHORT_WAVES : 1][ACC ? LOGITS : 1];
    __shared__ float sM[SHORT_WAVES][16], sL[SHORT_WAVES][16], sLse[16];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), c = lane & 15, q4 = lane >> 4;
    const int bh = blockIdx.x, b = bh / D.Hkv, h = bh % D.Hkv, len = seq_len(lens, b, max_len);
    const int64_t head = b * Q.st[0] + h * Q.st[1];
    const QuantRows R = {Q.K + head, Q.V + head, Q.Ks + int64_t(bh) * Q.nb, Q.Vs + int64_t(bh) * Q.nb, Q.st[2], Q.log_block};
    const float c2 = D.scale * 1.4426950408889634f;
    const int cols = D.G * tokens, width = (cols + 3) & ~3;
    const int64_t col0 = int64_t(bh) * cols;
    float m[1] = {NO_WEIGHT}, l[1] = {0.0f};
    f32x4 o[1][CPL];
    uint32_t unit = LEAST_UNIT;
#pragma unroll
    for (int e = 0; e < CPL; ++e) o[0][e] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    int r = wave * QT;
    if (r < len) {
        constexpr int STEP = SHORT_WAVES * QT;
        const int end = r + (len - 1 - r) / STEP * STEP, col = min(c, cols - 1);
        auto load = [&](QuantTile<DH>& t, int row) { load_quant_tile<DH, false>(t, R, min(row, end), q4, c, len - 1); };
        QuantTile<DH> A0, B0;
        load(A0, r);
        bf16x8 qf[1][TERMS][DH / 32];
        const T* qrow = q + (col0 + col) * DH;
#pragma unroll
        for (int kk = 0; kk < DH / 32; ++kk) {
            bf16x8 f[TERMS];
            query_terms(qrow + (kk / 2) * 64 + q4 * 16 + (kk % 2) * 8, f);
#pragma unroll
            for (int i = 0; i < TERMS; ++i) qf[0][i][kk] = f[i];
        }
        const int vis = min(len, len - tokens + 1 + col % tokens) - 4 * q4;
        LogitBuffer out[1] = {};
        if constexpr (ACC) out[0] = logit_buffer(sLogit[wave], LOGITS, nullptr, 0, cols, 0);      // room for all of the wave's tiles
        auto use = [&](const QuantTile<DH>& t) {
            const int seen[1] = {vis - r};
            use_quant_tile<DH, FMT, TERMS, ACC, 1>(m, l, o, unit, t, qf, seen, c2, out);
        };
        for (;;) {
            load(B0, r + STEP);
            use(A0);
            if ((r += STEP) >= len) break;
            load(A0, r + STEP);
            use(B0);
            if ((r += STEP) >= len) break;
        }
    }
    lanes_u32x2 x = pair32(__float_as_uint(l[0]));
    l[0] = __uint_as_float(x.x) + __uint_as_float(x.y);
    x = pair16(__float_as_uint(l[0]));
    l[0] = __uint_as_float(x.x) + __uint_as_float(x.y);
    if (c < cols) {
        if (q4 == 0) { sM[wave][c] = m[0]; sL[wave][c] = l[0]; }
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int e = 0; e < CPL; e += 4)
                *reinterpret_cast<f32x4*>(&sO[wave][c * LROW + (4 * q4 + i) * CPL + e]) =
                    f32x4{o[0][e][i], o[0][e + 1][i], o[0][e + 2][i], o[0][e + 3][i]} * unit_value(unit);
    }
    __syncthreads();
    const int waves = max(1, min(SHORT_WAVES, (len + QT - 1) / QT));         // those that had a tile
    for (int e = tid; e < cols * DH; e += THREADS) {
        const int g = e / DH, ch = e % DH;
        float M = sM[0][g], sum = 0.0f, val = 0.0f;
        for (int w = 1; w < waves; ++w) M = fmaxf(M, sM[w][g]);
        for (int w = 0; w < waves; ++w) {
            const float a = __builtin_amdgcn_exp2f(sM[w][g] - M);
            sum = __builtin_fmaf(sL[w][g], a, sum);
            val = __builtin_fmaf(sO[w][g * LROW + ch], a, val);
        }
        const bool none = sum == 0.0f;
        Elem<T>::put(O + (col0 + g) * DH + ch, none ? 0.0f : val / sum);
        if (ch == 0) {
            sLse[g] = none ? INFINITY : M + __builtin_log2f(sum);
            if (lse) lse[col0 + g] = none ? -INFINITY : log2_to_ln(M, sum);
        }
    }
    if constexpr (ACC) {
        __syncthreads();
        for (int i = tid; i < len; i += THREADS) {
            const int tile = i / QT;
            const float* p = sLogit[tile % SHORT_WAVES] + (tile / SHORT_WAVES * QT + i % QT) * width;
            float t = 0.0f;
            for (int g = 0; g < cols; ++g) t += __builtin_amdgcn_exp2f(p[g] - sLse[g]);
            const int64_t at = int64_t(bh) * A.cap + i;
            A.out[at] = A.in ? __builtin_fmaf(A.decay, A.in[at], t) : t;
        }
    }
}

// The first `rows` workgroups merge the slices of a query row each; the others, where weights are accumulated, take cache rows
// of a unit.
__device__ __forceinline__ void unit_slices(const Dims& D, const QuantSlices& S, const QuantSeq* seqs, int unit, int len, int& base, int& n) {
    if (S.splits) {
        base = unit * S.splits;
        n = (len + S.least * QT - 1) / (S.least * QT);
    } else {
        const QuantSeq s = seqs[unit / D.Hkv];
        base = s.base + unit % D.Hkv * s.n;
        n = s.n;
    }
}
template <typename T>
__global__ __launch_bounds__(DEC_THREADS) void k_quant_combine(Dims D, const float* __restrict__ part, int tokens, const int32_t* __restrict__ lens,
                                                               int max_len, QuantSlices S, const QuantSeq* __restrict__ seqs, T* __restrict__ O,
                                                               float* __restrict__ lse, AccArgs A, int rows, int chunks) {
    __shared__ __attribute__((aligned(16))) union { CombineLds c; float lse[ACC_COLS]; } sh;
    const int rec = D.d + 2, cols = D.G * tokens;
    const int64_t step = int64_t(cols) * rec;
    int base, n;
    if (int(blockIdx.x) < rows) {
        const int row = blockIdx.x, unit = row / cols;
        unit_slices(D, S, seqs, unit, seq_len(lens, unit / D.Hkv, max_len), base, n);
        combine_row<T>(part + base * step + row % cols * rec, step, D.d, n, O + int64_t(row) * D.d, lse ? lse + row : nullptr, sh.c);
        return;
    }
    const int at = int(blockIdx.x) - rows, unit = at / chunks, r0 = at % chunks * acc_wg_rows(A.pitch);
    const int len = seq_len(lens, unit / D.Hkv, max_len);
    if (r0 >= len) return;
    unit_slices(D, S, seqs, unit, len, base, n);
    acc_rows(A, unit, part + base * step, rec, step, n, r0, len, sh.lse);
}

// ------------------------------------------------------------------------------------ launches
#define LRSA_QUANT_PICK(KERNEL, T_)                                                                                        \
    (Q.fmt == QUANT_INT8 ? (D.d == 64 ? KERNEL<T_, 64, QUANT_INT8> : KERNEL<T_, 128, QUANT_INT8>)                         \
                         : (D.d == 64 ? KERNEL<T_, 64, QUANT_E4M3> : KERNEL<T_, 128, QUANT_E4M3>))

template <typename T>
static hipError_t run_append(const Dims& D, const QuantDims& Q, const void* K, const void* V, int tokens, const int32_t* lens, const int32_t* counts,
                             hipStream_t st) {
    // blocks that `tokens` rows can touch, wherever in a block they begin, as far as the cache goes
    const int touched = int((int64_t(tokens) + Q.block - 2) / Q.block + 1), blocks = touched < Q.nb ? touched : Q.nb;
#define LRSA_APPEND(DH_, FMT_, PASSES_)                                                                                                 \
    LRSA_TIMED_LAUNCH("k_append_quant", st, (k_append_quant<T, DH_, FMT_, PASSES_>), dim3(blocks, 2, D.B * D.Hkv), dim3(QUANT_THREADS),  \
                      0, st, D, Q, (const T*)K, (const T*)V, tokens, lens, counts)
#define LRSA_APPEND_128(FMT_) \
    switch (Q.block) { case 128: LRSA_APPEND(128, FMT_, 8); break; case 64: LRSA_APPEND(128, FMT_, 4); break; default: LRSA_APPEND(128, FMT_, 2); }
#define LRSA_APPEND_64(FMT_) \
    switch (Q.block) { case 128: LRSA_APPEND(64, FMT_, 4); break; case 64: LRSA_APPEND(64, FMT_, 2); break; default: LRSA_APPEND(64, FMT_, 1); }
    if (Q.fmt == QUANT_INT8) {
        if (D.d == 64) { LRSA_APPEND_64(QUANT_INT8); } else { LRSA_APPEND_128(QUANT_INT8); }
    } else {
        if (D.d == 64) { LRSA_APPEND_64(QUANT_E4M3); } else { LRSA_APPEND_128(QUANT_E4M3); }
    }
#undef LRSA_APPEND_64
#undef LRSA_APPEND_128
#undef LRSA_APPEND
    return hipGetLastError();
}
hipError_t launch_append_quant(const Dims& D, const QuantDims& Q, const void* K, const void* V, int tokens, const int32_t* lens,
                               const int32_t* counts, hipStream_t st) {
    return D.dtype == 1 ? run_append<bf16_t>(D, Q, K, V, tokens, lens, counts, st) : run_append<float>(D, Q, K, V, tokens, lens, counts, st);
}

template <typename T>
static hipError_t run_read(const Dims& D, const QuantDims& Q, const int32_t* lens, int rows, const int32_t* first, void* K, void* V, hipStream_t st) {
    const unsigned blocks = unsigned((int64_t(rows) * (D.d / 8) + QUANT_THREADS - 1) / QUANT_THREADS);
    LRSA_TIMED_LAUNCH("k_read_quant", st, LRSA_QUANT_PICK(k_read_quant, T), dim3(blocks, 2, D.B * D.Hkv), dim3(QUANT_THREADS), 0, st, D, Q, lens,
                      rows, first, (T*)K, (T*)V);
    return hipGetLastError();
}
bool read_quant_grid_fits(const Dims& D, int rows) { return grid_fits((int64_t(rows) * (D.d / 8) + QUANT_THREADS - 1) / QUANT_THREADS, QUANT_THREADS); }
hipError_t launch_read_quant(const Dims& D, const QuantDims& Q, const int32_t* lens, int rows, const int32_t* first, void* K, void* V,
                             hipStream_t st) {
    return D.dtype == 1 ? run_read<bf16_t>(D, Q, lens, rows, first, K, V, st) : run_read<float>(D, Q, lens, rows, first, K, V, st);
}

// Tiles of a slice from which on a wave takes two groups of columns.  Shorter walks are bound by their latency, of which two groups have
// more.  8 requests on 8 KV heads of 4 query heads, 8 tokens each, bf16, one group and two, us per call: d 128, 4K rows (16 tiles) 35.2 and
// 37.3, 8K (32) 48.3 and 47.7, 16K (62) 74.3 and 67.7; d 64, 24.0 and 24.8, 33.5 and 32.3, 51.6 and 46.1.  With 16 tokens, where the walk is twice as
// much work, two groups gain sooner (d 128: 50.9 and 48.6, 78.3 and 69.4, 131 and 112; d 64: 37.2 and 35.8, 56.4 and 50.2, 92.7 and
// 78.1): the one number is that of few columns.
constexpr int WIDE_TILES = 40;
constexpr int64_t PAST_BYTES = int64_t(256) << 20;      // see k_decode_quant
namespace {
struct QuantPlan { QuantSlices s; int grid, pitch; bool wide; int64_t rows; size_t part, logits, bytes; };
}
// Workspace: a QuantSeq per sequence, the records of `grid` workgroups, the logits.  All of them grow with max_len.
static QuantPlan quant_plan(const Dims& D, int tokens, int max_len, bool acc) {
    QuantPlan P = {};
    const int64_t units = int64_t(D.B) * D.Hkv;
    // Two workgroups share a CU (registers), so 512 run at once.  With more units than half of that some would have two slices and some
    // one: then several rounds, of few more slices than units.  8 KV heads, 64 requests of 2048 rows: units + 256 60 us, + 512 63,
    // + 768 71, + 2048 78; 33 of 4096: 81, 70, 65, 70.
    // With few units of long bf16 rows, one workgroup per CU keeps enough loads in flight, and half as many slices are joined: 8 KV heads, bf16,
    // d 128, 4 columns, 256 and 512 workgroups: 1 request of 16K rows 15.9 us and 17.6, of 128K 50.5 and 54.1, 4 of 40K 59.7 and 62.5, of
    // 13K to 40K each 50.3 and 51.3, but 8 of 11K to 32K 76.5 and 75.1; 20 columns: 1 of 16K 21.5 and 24.1, of 41K 33.0 and 35.5, of 64K 41.5
    // and 45.0, but of 128K 74 and 71 (taken all the same) and 4 of 40K 84 and 80; d 64, 4 of 40K 39.3 and 34.7; fp32 67 and 65.
    const bool few = D.dtype == 1 && D.d == 128 && units <= (D.G * tokens <= 16 ? 32 : 8);
    const int64_t most = few ? 256 : units <= 256 ? 512 : units + 512;
    const int64_t tiles = (int64_t(max_len) + QT - 1) / QT, fine = units * ((tiles + DEC_WAVES - 1) / DEC_WAVES);
    const float up = 1.0f + 0x1p-20f;
    P.s.most = int(most);
    P.s.share = float(D.Hkv) / float(most) * up;
    P.s.safe = float(D.Hkv) / float(most - units) * up;
    P.s.least = int((tiles + DEC_MAX_SPLITS - 1) / DEC_MAX_SPLITS);
    if (P.s.least < DEC_WAVES) P.s.least = DEC_WAVES;          // a tile per wave
    P.grid = int(most < fine ? most : fine);
    if (fine <= most && P.s.least == DEC_WAVES) P.s.splits = int(fine / units);
    P.wide = units * tiles >= most * WIDE_TILES;
    P.rows = tiles * QT;
    const size_t cols = size_t(D.G) * tokens;
    P.part = align256(size_t(D.B) * sizeof(QuantSeq));
    P.logits = P.part + align256(size_t(P.grid) * cols * (D.d + 2) * 4);
    P.pitch = (D.G * tokens + 3) & ~3;
    P.bytes = P.logits + (acc ? align256(size_t(units) * P.pitch * size_t(P.rows) * 4) : 0);
    return P;
}
size_t decode_quant_ws_bytes(const Dims& D, int tokens, int max_len, bool acc) { return quant_plan(D, tokens, max_len, acc).bytes; }
// rows and tiles are counted in 32 bits
bool decode_quant_grid_fits(const Dims& D, int tokens, int max_len) {
    return max_len <= 1 << 30 && int64_t(D.B) * ((max_len + QT - 1) / QT) < int64_t(1) << 31 && grid_fits(int64_t(D.B) * D.Hq * tokens + int64_t(D.B) * D.Hkv * ((int64_t(max_len) + DEC_THREADS - 1) / DEC_THREADS), DEC_THREADS);
}

// One workgroup per unit, or slices?  Heads of 64: one, always (1 request of 1024 rows 9.1 us, slices 11; 64 of 1024 17.8, 24.1).
// Heads of 128 have twice the bytes: one where it is short (12 heads on 2, 100 rows: 7.6, 10.3) or where units fill the card (16 requests
// of 1000 rows: 13.9, 16.1; 64 of 1024: 29.7, 34.2), slices else (1 request of 1024 rows: 13.2, 10.3; 8 of 1024: 13.6, 11.8).
static bool short_cache(const Dims& D, int cols, int max_len) {
    return cols <= 16 && max_len <= SHORT_ROWS && (D.d == 64 || max_len <= SHORT_ROWS / 2 || int64_t(D.B) * D.Hkv >= 128);
}

// Two groups of columns in one wave (17 to 32 columns): heads of 128 go past the caches by size like one group.  8 KV heads of 4 query heads, 5
// tokens, bf16, us per call on the same cache, through and past the caches: 83 MB 34 and 37, 163 MB 46 and 52, 229 MB 55 and 61; on others in
// turn: 33 and 37, 48 and 52, 61 and 60.  At any size heads of 64 do (86 to 204 MB the same, in turn 35 and 34, 43 and 42, 62 and 61), and calls
// that accumulate weights: the logits, 64 bytes or more per row, are then found in the caches when they are read again (d 64, 122 MB, on
// others in turn 87 and 80, on the same cache 73 and 80; d 128, 229 MB 109 and 99, 96 and 99; 537 MB 249 and 238, 243 and 200).
template <typename T, int DH, int FMT>
static auto decode_quant_kernel(int cols, bool wide, bool past, bool acc) {
    constexpr int MOST = MOST_GROUPS<T, DH>;
    if (cols <= 16 && past) return acc ? k_decode_quant<T, DH, FMT, 1, true, true, true> : k_decode_quant<T, DH, FMT, 1, true, true, false>;
    if (cols <= 16) return acc ? k_decode_quant<T, DH, FMT, 1, true, false, true> : k_decode_quant<T, DH, FMT, 1, true, false, false>;
    if constexpr (MOST > 1)
        if (wide) {
            if (cols > 16 * MOST) return acc ? k_decode_quant<T, DH, FMT, MOST, false, false, true> : k_decode_quant<T, DH, FMT, MOST, false, false, false>;
            if (acc) return k_decode_quant<T, DH, FMT, MOST, true, true, true>;
            if constexpr (DH == 128)
                if (!past) return k_decode_quant<T, DH, FMT, MOST, true, false, false>;
            return k_decode_quant<T, DH, FMT, MOST, true, true, false>;
        }
    return acc ? k_decode_quant<T, DH, FMT, 1, false, false, true> : k_decode_quant<T, DH, FMT, 1, false, false, false>;
}

template <typename T>
static hipError_t run_decode_quant(const Dims& D, const QuantDims& Q, const void* q, int tokens, const int32_t* lens, int max_len, void* O, float* lse,
                                   const float* acc_in, float* acc_out, float decay, void* ws, hipStream_t st) {
    const QuantPlan P = quant_plan(D, tokens, max_len, acc_out != nullptr);
    char* w = reinterpret_cast<char*>(ws);
    QuantSeq* seqs = reinterpret_cast<QuantSeq*>(w);
    float* part = reinterpret_cast<float*>(w + P.part);
    float* logits = acc_out ? reinterpret_cast<float*>(w + P.logits) : nullptr;
    const int rows = D.B * D.Hq * tokens, chunks = acc_out ? (max_len - 1) / acc_wg_rows(P.pitch) + 1 : 0;
    AccArgs A = {};
    A.logits = logits;
    A.mul = 1.0f;
    A.rows = P.rows;
    A.cols = D.G * tokens;
    A.pitch = P.pitch;
    A.in = acc_in;
    A.out = acc_out;
    A.cap = D.n;
    A.decay = decay;
    if (short_cache(D, A.cols, max_len)) {
#define LRSA_DECODE_SHORT(DH_, FMT_)                                                                                                      \
    LRSA_TIMED_LAUNCH("k_decode_quant_short", st,                                                                                         \
                      (acc_out ? k_decode_quant_short<T, DH_, FMT_, true> : k_decode_quant_short<T, DH_, FMT_, false>),                    \
                      dim3(D.B * D.Hkv), dim3(64 * SHORT_WAVES), 0, st, D, Q, (const T*)q, tokens, lens, max_len, (T*)O, lse, A)
        if (Q.fmt == QUANT_INT8) {
            if (D.d == 64) LRSA_DECODE_SHORT(64, QUANT_INT8); else LRSA_DECODE_SHORT(128, QUANT_INT8);
        } else {
            if (D.d == 64) LRSA_DECODE_SHORT(64, QUANT_E4M3); else LRSA_DECODE_SHORT(128, QUANT_E4M3);
        }
#undef LRSA_DECODE_SHORT
        return hipGetLastError();
    }
    const bool past = int64_t(D.B) * D.Hkv * max_len * D.d * 2 >= PAST_BYTES;
#define LRSA_DECODE_QUANT(DH_, FMT_)                                                                                                      \
    LRSA_TIMED_LAUNCH("k_decode_quant", st, (decode_quant_kernel<T, DH_, FMT_>(A.cols, P.wide, past, acc_out != nullptr)), dim3(P.grid),   \
                      dim3(DEC_THREADS), 0, st, D, Q, (const T*)q, tokens, lens, max_len, P.s, seqs, part, logits, P.rows, P.pitch)
    if (Q.fmt == QUANT_INT8) {
        if (D.d == 64) LRSA_DECODE_QUANT(64, QUANT_INT8); else LRSA_DECODE_QUANT(128, QUANT_INT8);
    } else {
        if (D.d == 64) LRSA_DECODE_QUANT(64, QUANT_E4M3); else LRSA_DECODE_QUANT(128, QUANT_E4M3);
    }
#undef LRSA_DECODE_QUANT
    LRSA_TIMED_LAUNCH("k_quant_combine", st, k_quant_combine<T>, dim3(unsigned(rows + D.B * D.Hkv * chunks)), dim3(DEC_THREADS), 0, st, D, part, tokens,
                      lens, max_len, P.s, seqs, (T*)O, lse, A, rows, chunks);
    return hipGetLastError();
}
hipError_t launch_decode_quant(const Dims& D, const QuantDims& Q, const void* q, int tokens, const int32_t* lens, int max_len, void* O, float* lse,
                               const float* acc_in, float* acc_out, float decay, void* ws, hipStream_t st) {
    return D.dtype == 1 ? run_decode_quant<bf16_t>(D, Q, q, tokens, lens, max_len, O, lse, acc_in, acc_out, decay, ws, st)
                        : run_decode_quant<float>(D, Q, q, tokens, lens, max_len, O, lse, acc_in, acc_out, decay, ws, st);
}

}  // namespace lrsa
