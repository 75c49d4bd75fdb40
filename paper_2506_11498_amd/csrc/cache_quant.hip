// The inference-time cache in 8 bits: rows written into it, rows read back, attention of a few query tokens over it.  Codes
// and scales: quant_block.h.  Every sequence has a length of its own, in device memory, so that a captured graph can be
// replayed while the sequences grow.
//
// k_append_quant      new rows into the blocks of the cache that they belong to
// k_read_quant        rows of the cache as values
// k_decode_quant      attention of the query rows of a KV group over a slice of the cache rows, on the matrix cores
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
// scale where that is large enough; where it is not, the scale grows and the older codes follow.
template <typename T, int DH, int FMT>
__global__ __launch_bounds__(QUANT_THREADS) void k_append_quant(Dims D, QuantDims Q, const T* __restrict__ K, const T* __restrict__ V, int tokens,
                                                                const int32_t* __restrict__ lens, const int32_t* __restrict__ counts) {
    constexpr int LPR = DH / 8, RPP = QUANT_THREADS / LPR, PASSES = QUANT_MAX_BLOCK / RPP;
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
    for (int p = 0; p < PASSES; ++p) {
        const int r = p * RPP + rg;
        if (r >= r0 && r < r1) load8(src + r * D.ks[2], v[p]);
        else
#pragma unroll
            for (int i = 0; i < 8; ++i) v[p][i] = 0.0f;
    }
#pragma unroll
    for (int p = 0; p < PASSES; ++p)
#pragma unroll
        for (int i = 0; i < 8; ++i) top = fmaxf(top, fabsf(v[p][i]));
    const float s = fmaxf(quant_scale<FMT>(block_max<QUANT_THREADS>(top, sm)), before);
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
// One workgroup: the query rows of one KV group (16 at a time) x rows [split * per, ...) of the cache, as k_decode_mfma.  A
// query row ("column") is (head of the group, token): q is [B, Hq, T, d], so the columns of a unit are neighbours.  Lane l, c =
// l % 16, q4 = l / 16, v_mfma_f32_16x16x32_bf16:
//   S = K Q^T   row m of block kb is tile row 8*(m/4) + 4*kb + m%4.  The contraction over the channels may take them in any
//               order: the lane reads 16 neighbouring bytes (channels 64*i + 16*q4 ..), two instructions' worth
//   O^T += V^T P^T   the lane reads DH/16 neighbouring channels of tile rows 8*q4 .. +7 and transposes that block
// Codes have at most 8 significant bits, so both operands are exact in bf16 without their scales; the scale of K multiplies
// the logit, that of V the weight, in fp32 (8 neighbouring rows of a tile share a block: blocks are multiples of 16).  Queries
// of fp32 enter as three bf16 terms, which hold all 24 bits, and so do the weights.
constexpr int QT = 32;                       // rows per wave and step
constexpr float NO_WEIGHT = -1e30f;          // running maximum before the first visible row: finite, so that differences are
template <int DH> struct QPiece { typedef uint2 type; };
template <> struct QPiece<64> { typedef uint32_t type; };
template <int DH> struct QuantTile {
    uint4 k[2][DH / 64];
    typename QPiece<DH>::type v[8];
    float ks, vs;
};

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

template <int DH>
__device__ __forceinline__ void load_quant_tile(QuantTile<DH>& t, const QuantDims& Q, const uint8_t* Kl, const uint8_t* Vl, const float* Ks,
                                                const float* Vs, int kr, int vr, int last) {
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
        const uint8_t* row = Kl + int64_t(min(kr + 4 * kb, last)) * Q.st[2];   // rows past the end repeat the last one, weight 0
#pragma unroll
        for (int i = 0; i < DH / 64; ++i) t.k[kb][i] = *reinterpret_cast<const uint4*>(row + i * 64);
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) t.v[j] = *reinterpret_cast<const typename QPiece<DH>::type*>(Vl + int64_t(min(vr + j, last)) * Q.st[2]);
    const int block = min(vr, last) >> Q.log_block;
    t.ks = Ks[block];
    t.vs = Vs[block];
}

// r: the first of the lane's rows; seen: rows from there on that its column sees
template <int DH, int FMT, int TERMS>
__device__ __forceinline__ void use_quant_tile(float& m, float& l, f32x4 (&o)[DH / 16], const QuantTile<DH>& t, const bf16x8 (&qf)[TERMS][DH / 32],
                                               int seen, float c2, float* logits) {
    f32x4 s[2] = {{0.0f, 0.0f, 0.0f, 0.0f}, {0.0f, 0.0f, 0.0f, 0.0f}};
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int kk = 0; kk < DH / 32; ++kk) {
            const uint4 w = t.k[kb][kk / 2];
            uint32_t a[4];
            codes_bf16<FMT>(kk % 2 ? w.z : w.x, a[0], a[1]);
            codes_bf16<FMT>(kk % 2 ? w.w : w.y, a[2], a[3]);
            const bf16x8 kf = __builtin_bit_cast(bf16x8, a);
#pragma unroll
            for (int i = TERMS - 1; i >= 0; --i) s[kb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[i][kk], s[kb], 0, 0, 0);
        }
    float p[8], mx = NO_WEIGHT;
    const float c2s = c2 * t.ks;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        p[j] = j < seen ? s[j >> 2][j & 3] * c2s : -INFINITY;
        mx = fmaxf(mx, p[j]);
    }
    if (logits) {
        reinterpret_cast<f32x4*>(logits)[0] = f32x4{p[0], p[1], p[2], p[3]};
        reinterpret_cast<f32x4*>(logits)[1] = f32x4{p[4], p[5], p[6], p[7]};
    }
    lanes_u32x2 x = pair32(__float_as_uint(mx));
    mx = fmaxf(__uint_as_float(x.x), __uint_as_float(x.y));
    x = pair16(__float_as_uint(mx));
    mx = fmaxf(__uint_as_float(x.x), __uint_as_float(x.y));
    if (__builtin_amdgcn_ballot_w64(mx > m) != 0) {
        const float mn = fmaxf(m, mx), a = __builtin_amdgcn_exp2f(m - mn);
        m = mn;
        l *= a;
#pragma unroll
        for (int e = 0; e < DH / 16; ++e) o[e] *= a;
    }
    f32x8 w;
    float ps = 0.0f;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const float e = __builtin_amdgcn_exp2f(p[j] - m);
        ps += e;
        w[j] = e * t.vs;
    }
    l += ps;
    bf16x8 term[3];
#pragma unroll
    for (int i = 0; i < 3; ++i) {
        term[i] = __builtin_convertvector(w, bf16x8);
        w -= __builtin_convertvector(term[i], f32x8);
    }
    constexpr int DW = DH / 64;              // dwords of codes per row
    uint32_t b[8][2 * DW];                   // the same as bf16 pairs
#pragma unroll
    for (int j = 0; j < 8; ++j)
#pragma unroll
        for (int i = 0; i < DW; ++i) codes_bf16<FMT>(reinterpret_cast<const uint32_t*>(&t.v[j])[i], b[j][2 * i], b[j][2 * i + 1]);
#pragma unroll
    for (int e = 0; e < DH / 16; ++e) {
        uint32_t a[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) a[i] = __builtin_amdgcn_perm(b[2 * i + 1][e >> 1], b[2 * i][e >> 1], e & 1 ? 0x07060302u : 0x05040100u);
        const bf16x8 av = __builtin_bit_cast(bf16x8, a);
#pragma unroll
        for (int i = 2; i >= 0; --i) o[e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(av, term[i], o[e], 0, 0, 0);
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

template <typename T, int DH, int FMT>
__global__ __launch_bounds__(DEC_THREADS, 2) void k_decode_quant(Dims D, QuantDims Q, const T* __restrict__ q, int tokens, const int32_t* __restrict__ lens,
                                                                 int max_len, int per, int splits, float* __restrict__ part,
                                                                 float* __restrict__ logits, int64_t lstride) {
    constexpr int CPL = DH / 16, LROW = DH + 4, TERMS = Q_TERMS<T>;
    __shared__ __attribute__((aligned(16))) float sO[DEC_WAVES][16][LROW];
    __shared__ float sM[DEC_WAVES][16], sL[DEC_WAVES][16];
    const int split = blockIdx.x, bh = blockIdx.y, b = bh / D.Hkv, h = bh % D.Hkv;
    const int len = seq_len(lens, b, max_len);
    const int r0 = split * per, r1 = min(len, r0 + per);
    if (r0 >= r1) return;                                    // an empty slice: the merge does not ask for it
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, c = lane & 15, q4 = lane >> 4;
    const uint8_t* Kl = Q.K + b * Q.st[0] + h * Q.st[1] + q4 * 16;
    const uint8_t* Vl = Q.V + b * Q.st[0] + h * Q.st[1] + c * CPL;
    const float *Ks = Q.Ks + int64_t(bh) * Q.nb, *Vs = Q.Vs + int64_t(bh) * Q.nb;
    const int kr = 8 * (c >> 2) + (c & 3), vr = 8 * q4;
    const float c2 = D.scale * 1.4426950408889634f;          // logits in log2 units
    const int cols = D.G * tokens;
    const int64_t col0 = int64_t(bh) * cols;                 // query rows of the units before

    for (int g0 = 0; g0 < cols; g0 += 16) {
        const int gn = min(16, cols - g0), col = g0 + min(c, gn - 1);
        const int vis = len - tokens + 1 + col % tokens;     // rows that the column sees, none where that is not positive
        const T* qrow = q + (col0 + col) * DH;
        bf16x8 qf[TERMS][DH / 32];
#pragma unroll
        for (int kk = 0; kk < DH / 32; ++kk) {
            bf16x8 f[TERMS];
            query_terms(qrow + (kk / 2) * 64 + q4 * 16 + (kk % 2) * 8, f);
#pragma unroll
            for (int i = 0; i < TERMS; ++i) qf[i][kk] = f[i];
        }
        float m = NO_WEIGHT, l = 0.0f;
        f32x4 o[CPL];
#pragma unroll
        for (int e = 0; e < CPL; ++e) o[e] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        constexpr int STEP = DEC_WAVES * QT;
        float* lrow = logits && c < gn ? logits + (col0 + g0 + c) * lstride + vr : nullptr;
        int r = r0 + wave * QT;
        if (r < r1) {
            QuantTile<DH> A, B;
            load_quant_tile<DH>(A, Q, Kl, Vl, Ks, Vs, r + kr, r + vr, r1 - 1);
            for (;;) {
                if (r + STEP < r1) load_quant_tile<DH>(B, Q, Kl, Vl, Ks, Vs, r + STEP + kr, r + STEP + vr, r1 - 1);
                use_quant_tile<DH, FMT, TERMS>(m, l, o, A, qf, min(r1, vis) - r - vr, c2, lrow ? lrow + r : nullptr);
                if ((r += STEP) >= r1) break;
                if (r + STEP < r1) load_quant_tile<DH>(A, Q, Kl, Vl, Ks, Vs, r + STEP + kr, r + STEP + vr, r1 - 1);
                use_quant_tile<DH, FMT, TERMS>(m, l, o, B, qf, min(r1, vis) - r - vr, c2, lrow ? lrow + r : nullptr);
                if ((r += STEP) >= r1) break;
            }
        }
        lanes_u32x2 x = pair32(__float_as_uint(l));
        l = __uint_as_float(x.x) + __uint_as_float(x.y);
        x = pair16(__float_as_uint(l));
        l = __uint_as_float(x.x) + __uint_as_float(x.y);
        if (c < gn) {
            if (q4 == 0) { sM[wave][c] = m; sL[wave][c] = l; }
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int e = 0; e < CPL; e += 4)
                    *reinterpret_cast<f32x4*>(&sO[wave][c][(4 * q4 + i) * CPL + e]) = f32x4{o[e][i], o[e + 1][i], o[e + 2][i], o[e + 3][i]};
        }
        __syncthreads();
        for (int e = tid; e < gn * DH; e += DEC_THREADS) {
            const int g = e / DH, ch = e % DH;
            float mm = sM[0][g], ll = sL[0][g], oo = sO[0][g][ch];
#pragma unroll
            for (int w = 1; w < DEC_WAVES; ++w) {
                float a, b2;
                merge_state(mm, ll, sM[w][g], sL[w][g], a, b2);
                oo = oo * a + sO[w][g][ch] * b2;
            }
            float* dst = part + ((col0 + g0 + g) * splits + split) * (DH + 2);
            dst[2 + ch] = oo;
            if (ch == 0) { dst[0] = mm; dst[1] = ll; }
        }
        __syncthreads();
    }
}

// The first `rows` workgroups merge the slices of a query row each; the others, where weights are accumulated, take ACC_ROWS
// cache rows of a unit each.
template <typename T>
__global__ __launch_bounds__(DEC_THREADS) void k_quant_combine(Dims D, const float* __restrict__ part, int tokens, const int32_t* __restrict__ lens,
                                                               int max_len, int per, int splits, T* __restrict__ O, float* __restrict__ lse,
                                                               AccArgs A, int rows, int chunks) {
    __shared__ union { CombineLds c; float lse[ACC_COLS]; } sh;
    const int rec = D.d + 2, cols = D.G * tokens;
    if (int(blockIdx.x) < rows) {
        const int64_t row = blockIdx.x;
        const int len = seq_len(lens, int(row / (int64_t(D.Hkv) * cols)), max_len);
        combine_row<T>(part + row * splits * rec, D.d, (len + per - 1) / per, O + row * D.d, lse ? lse + row : nullptr, sh.c);
        return;
    }
    const int at = int(blockIdx.x) - rows, unit = at / chunks, r0 = at % chunks * ACC_ROWS;
    const int len = seq_len(lens, unit / D.Hkv, max_len);
    if (r0 >= len) return;
    acc_rows(A, unit, part + int64_t(unit) * cols * splits * rec, int64_t(splits) * rec, rec, (len + per - 1) / per, r0, len, sh.lse);
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
    LRSA_TIMED_LAUNCH("k_append_quant", st, LRSA_QUANT_PICK(k_append_quant, T), dim3(blocks, 2, D.B * D.Hkv), dim3(QUANT_THREADS), 0, st, D, Q,
                      (const T*)K, (const T*)V, tokens, lens, counts);
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

// Slices: as many as fill the chip twice over when every sequence has max_len rows, of 128 rows at least (a tile per wave).
static int quant_splits(const Dims& D, int max_len) {
    const int units = D.B * D.Hkv, most = (max_len + 127) / 128;
    int s = units <= 128 ? 512 / units : 2048 / units;
    s = s < most ? s : most;
    return s < 1 ? 1 : s > DEC_MAX_SPLITS ? DEC_MAX_SPLITS : s;
}
namespace {
struct QuantPlan { int splits, per; int64_t stride; size_t part, bytes; };
}
static QuantPlan quant_plan(const Dims& D, int tokens, int max_len, bool acc) {
    QuantPlan P = {};
    const int splits = quant_splits(D, max_len);
    P.per = ((max_len + splits - 1) / splits + QT - 1) / QT * QT;
    P.splits = (max_len + P.per - 1) / P.per;
    P.stride = (int64_t(max_len) + QT - 1) / QT * QT;
    const size_t rows = size_t(D.B) * D.Hq * tokens;
    P.part = align256(rows * splits * (D.d + 2) * 4);       // grows with max_len, which P.splits does not always: a workspace for a longer one is enough
    P.bytes = P.part + (acc ? align256(rows * size_t(P.stride) * 4) : 0);
    return P;
}
size_t decode_quant_ws_bytes(const Dims& D, int tokens, int max_len, bool acc) { return quant_plan(D, tokens, max_len, acc).bytes; }
bool decode_quant_grid_fits(const Dims& D, int tokens, int max_len) {
    return grid_fits(int64_t(D.B) * D.Hq * tokens + int64_t(D.B) * D.Hkv * ((int64_t(max_len) + ACC_ROWS - 1) / ACC_ROWS), DEC_THREADS);
}

template <typename T>
static hipError_t run_decode_quant(const Dims& D, const QuantDims& Q, const void* q, int tokens, const int32_t* lens, int max_len, void* O, float* lse,
                                   const float* acc_in, float* acc_out, float decay, void* ws, hipStream_t st) {
    const QuantPlan P = quant_plan(D, tokens, max_len, acc_out != nullptr);
    float* part = reinterpret_cast<float*>(ws);
    float* logits = acc_out ? reinterpret_cast<float*>(reinterpret_cast<char*>(ws) + P.part) : nullptr;
    const int rows = D.B * D.Hq * tokens, chunks = acc_out ? (max_len - 1) / ACC_ROWS + 1 : 0;
    AccArgs A = {};
    A.logits = logits;
    A.mul = 1.0f;
    A.stride = P.stride;
    A.cols = D.G * tokens;
    A.in = acc_in;
    A.out = acc_out;
    A.cap = D.n;
    A.decay = decay;
    LRSA_TIMED_LAUNCH("k_decode_quant", st, LRSA_QUANT_PICK(k_decode_quant, T), dim3(P.splits, D.B * D.Hkv), dim3(DEC_THREADS), 0, st, D, Q,
                      (const T*)q, tokens, lens, max_len, P.per, P.splits, part, logits, P.stride);
    LRSA_TIMED_LAUNCH("k_quant_combine", st, k_quant_combine<T>, dim3(unsigned(rows + D.B * D.Hkv * chunks)), dim3(DEC_THREADS), 0, st, D, part, tokens,
                      lens, max_len, P.per, P.splits, (T*)O, lse, A, rows, chunks);
    return hipGetLastError();
}
hipError_t launch_decode_quant(const Dims& D, const QuantDims& Q, const void* q, int tokens, const int32_t* lens, int max_len, void* O, float* lse,
                               const float* acc_in, float* acc_out, float decay, void* ws, hipStream_t st) {
    return D.dtype == 1 ? run_decode_quant<bf16_t>(D, Q, q, tokens, lens, max_len, O, lse, acc_in, acc_out, decay, ws, st)
                        : run_decode_quant<float>(D, Q, q, tokens, lens, max_len, O, lse, acc_in, acc_out, decay, ws, st);
}

}  // namespace lrsa
