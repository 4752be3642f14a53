// Rotary positions, and a cache that grows token by token and is held in 8 bits: the write into it, attention over it, eviction from
// it by accumulated attention weight and the compaction of what stays.
//
// Layout of a cache of L layers: K, V [L][Hkv][T_total][D] E4M3 codes; sequence b owns the rows cu_tok[b] .. cu_tok[b+1] - 1, and its
// block t of `block` rows (counted from its first one, so that no block belongs to two sequences) has the scale
// [L][Hkv][n_scales] at cu_tok[b] / block + b + t.  A code c stands for c * scale.  Scales are powers of two: the format is a floating one, so
// that a scale between two powers would gain nothing, while with these the division by a scale and the change from one scale to
// another are exact until a result is rounded to its code.
#include <math.h>

#include <type_traits>

#include "skv_device.h"

namespace skv {

namespace {

typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x2_t __attribute__((ext_vector_type(2)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));

constexpr uint32_t kInfBits = 0x7f800000u;

// Rows of sequence b in a pool of T_total rows: the first one and their number (none where the offsets do not lie in the pool).
__device__ __forceinline__ void region(const int32_t* __restrict__ cu_tok, int b, int32_t T_total, int32_t* first, int32_t* rows) {
    const int32_t t0 = cu_tok[b], t1 = min(cu_tok[b + 1], T_total);
    const bool ok = t0 >= 0 && t0 < t1;
    *first = ok ? t0 : 0;
    *rows = ok ? t1 - t0 : 0;
}

// The smallest power of two s, at least 2^-100, with a <= 448 s, from the bits of a finite a >= 0: 448 = 1.75 * 2^8, so that a fraction
// above 0.75 takes the next power.
__device__ __forceinline__ float scale_of(uint32_t a) {
    const int e = (int)((a + 0x1fffffu) >> 23) - 8;
    return __uint_as_float((uint32_t)max(e, 27) << 23);
}

// Four codes of values that are at most 448 (nearest, ties to even; what is not finite becomes NaN, which the format has beside no infinity).
__device__ __forceinline__ uint32_t codes_of(float a, float b, float c, float d) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
}
// Four codes times `f`, as codes.
__device__ __forceinline__ uint32_t rescale(uint32_t w, float f) {
    const f32x2_t lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
    return codes_of(lo[0] * f, lo[1] * f, hi[0] * f, hi[1] * f);
}

__device__ __forceinline__ uint32_t bf16_pair(float a, float b) {
    bf16x2_t v;
    v[0] = (__bf16)a;
    v[1] = (__bf16)b;
    return __builtin_bit_cast(uint32_t, v);
}

// ------------------------------------------------------------------------------------------------
// Rotary positions: the pair (x, y) of frequency i becomes (x c - y s, y c + x s), c + i s = mscale * exp(i pos f_i).  Bound by HBM: rows in, rows
// out.  An angle may be 10^6 and more, where 32 bits keep two digits of its fraction of a turn: it is formed and reduced in 64 bits, one frequency
// a lane, once per wave.  A wave takes one token and some of its heads; a lane turns two 16-byte pieces of a row, whose partners lie in one
// another (half layout) or in themselves (interleaved), so that a row may be turned where it lies.
// ------------------------------------------------------------------------------------------------
constexpr int kRotWaves = 4;

struct RotArgs {
    const char *q, *k;
    char *q_out, *k_out;
    const int32_t* pos;
    const double* inv_freq;
    int32_t n, n_q, n_k;        // tokens, heads of q and k (0: none)
    int32_t half, heads_per_wave;
    float mscale;
};

template <int EB> __device__ __forceinline__ void unpack16(const uint4& v, float* f) { Row<EB>::unpack(v, f); }
template <int EB> __device__ __forceinline__ uint4 pack16(const float* f) {
    if constexpr (EB == 2) return make_uint4(bf16_pair(f[0], f[1]), bf16_pair(f[2], f[3]), bf16_pair(f[4], f[5]), bf16_pair(f[6], f[7]));
    else return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
}

// VEC: rot is a multiple of 16.  Otherwise a lane turns one pair, element by element.
template <int EB, bool INTERLEAVED, bool VEC>
__global__ __launch_bounds__(kRotWaves * kWave) void rotary_kernel(RotArgs a) {
    __shared__ float2 table[kRotWaves][kHeadDim / 2];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const int64_t tok = (int64_t)blockIdx.x * kRotWaves + w;
    const bool live = tok < a.n;
    if (live && lane < a.half) {
        const double turns = (double)a.pos[tok] * a.inv_freq[lane] * 0.15915494309189533577;
        const float r = (float)(turns - rint(turns));
        float s, c;
        sincospif(2.0f * r, &s, &c);
        table[w][lane] = make_float2(c * a.mscale, s * a.mscale);
    }
    __syncthreads();
    if (!live) return;
    const int heads = a.n_q + a.n_k, h0 = blockIdx.y * a.heads_per_wave, h1 = min(heads, h0 + a.heads_per_wave);
    const int64_t row_bytes = kHeadDim * EB;
    auto row_in = [&](int h) { return h < a.n_q ? a.q + (tok * a.n_q + h) * row_bytes : a.k + (tok * a.n_k + (h - a.n_q)) * row_bytes; };
    auto row_out = [&](int h) { return h < a.n_q ? a.q_out + (tok * a.n_q + h) * row_bytes : a.k_out + (tok * a.n_k + (h - a.n_q)) * row_bytes; };
    if constexpr (VEC) {
        constexpr int E = 16 / EB, UNITS = kHeadDim / (2 * E), ROWS = kWave / UNITS;
        const int u = lane % UNITS, n_pairs = a.half / E;
        const bool turn = u < n_pairs;
        const int pa = (INTERLEAVED ? 2 * u : turn ? u : 2 * u) * 16, pb = INTERLEAVED || !turn ? pa + 16 : pa + n_pairs * 16;
        float c[E], s[E];
#pragma unroll
        for (int i = 0; i < E; ++i) {
            const float2 t = turn ? table[w][u * E + i] : make_float2(1.0f, 0.0f);
            c[i] = t.x;
            s[i] = t.y;
        }
        for (int h = h0 + lane / UNITS; h < h1; h += ROWS) {
            const char* in = row_in(h);
            char* out = row_out(h);
            uint4 va = *reinterpret_cast<const uint4*>(in + pa), vb = *reinterpret_cast<const uint4*>(in + pb);
            if (turn) {
                float x[2 * E], y[2 * E];
                unpack16<EB>(va, x);
                unpack16<EB>(vb, x + E);
#pragma unroll
                for (int i = 0; i < E; ++i) {
                    const int ia = INTERLEAVED ? 2 * i : i, ib = INTERLEAVED ? 2 * i + 1 : E + i;
                    y[ia] = x[ia] * c[i] - x[ib] * s[i];
                    y[ib] = x[ib] * c[i] + x[ia] * s[i];
                }
                va = pack16<EB>(y);
                vb = pack16<EB>(y + E);
            }
            *reinterpret_cast<uint4*>(out + pa) = va;
            *reinterpret_cast<uint4*>(out + pb) = vb;
        }
    } else {
        const bool turn = lane < a.half;
        const int ea = turn && !INTERLEAVED ? lane : 2 * lane, eb = turn && !INTERLEAVED ? lane + a.half : 2 * lane + 1;
        const float2 t = turn ? table[w][lane] : make_float2(1.0f, 0.0f);
        for (int h = h0; h < h1; ++h) {
            const char* in = row_in(h);
            char* out = row_out(h);
            if constexpr (EB == 2) {
                const uint16_t *i16 = reinterpret_cast<const uint16_t*>(in);
                uint16_t* o16 = reinterpret_cast<uint16_t*>(out);
                uint32_t xa = i16[ea], xb = i16[eb];
                if (turn) {
                    const float x = __uint_as_float(xa << 16), y = __uint_as_float(xb << 16);
                    const uint32_t z = bf16_pair(x * t.x - y * t.y, y * t.x + x * t.y);
                    xa = z & 0xffffu;
                    xb = z >> 16;
                }
                o16[ea] = (uint16_t)xa;
                o16[eb] = (uint16_t)xb;
            } else {
                const float *f = reinterpret_cast<const float*>(in), x = f[ea], y = f[eb];
                float* o = reinterpret_cast<float*>(out);
                o[ea] = turn ? x * t.x - y * t.y : x;
                o[eb] = turn ? y * t.x + x * t.y : y;
            }
        }
    }
}

// ------------------------------------------------------------------------------------------------
// Append: one block per (sequence, head, K or V, scale block that takes new rows).  Bound by HBM for prompts (the rows in, half or a quarter of
// their bytes out), by the chain of its loads for single tokens.  The block's new rows stay in registers between the search for the
// largest magnitude and the rounding.  Where rows are there already the scale can only grow; their codes are then rounded again.
// ------------------------------------------------------------------------------------------------
constexpr int kAppendThreads = 256;
constexpr int kAppendRows = kAppendThreads / 16;          // rows at a time: 16 lanes of 8 elements

struct AppendArgs {
    const char *k, *v;
    uint8_t *K, *V;             // the layer's slices
    float *ks, *vs, *acc;
    const int32_t *cu_new, *cu_tok, *n_tok;
    int32_t n_new, max_new, T_total, n_scales, shift, n_kv;
};

template <int EB, int BLOCK>
__global__ __launch_bounds__(kAppendThreads) void cache_append_kernel(AppendArgs a) {
    __shared__ uint32_t most[kAppendThreads / kWave];
    constexpr int ITERS = BLOCK / kAppendRows;
    const int pair = blockIdx.y, b = pair / a.n_kv, h = pair % a.n_kv;
    const bool is_v = blockIdx.z != 0;
    int32_t first, rows;
    region(a.cu_tok, b, a.T_total, &first, &rows);
    const int32_t held = min(max(a.n_tok[pair], 0), rows);
    const int32_t c0 = max(a.cu_new[b], 0), c1 = min(a.cu_new[b + 1], a.n_new);
    const int32_t m = min(min(c1 > c0 ? c1 - c0 : 0, a.max_new), rows - held);
    const int32_t t = (held >> a.shift) + blockIdx.x, base = t << a.shift;
    const int32_t lo = max(base, held), hi = min(base + BLOCK, held + m);     // the new rows of this block
    if (lo >= hi) return;
    const int tid = threadIdx.x, col = (tid & 15) * 8, r0 = tid >> 4;
    float* scale = (is_v ? a.vs : a.ks) + (int64_t)h * a.n_scales + (first >> a.shift) + b + t;
    const bool has_old = base < held;
    const float old = has_old ? *scale : 0.0f;
    const char* src = is_v ? a.v : a.k;
    uint8_t* dst = (is_v ? a.V : a.K) + ((int64_t)h * a.T_total + first + base) * kHeadDim + col;

    uint4 x[ITERS * EB / 2];
    uint32_t big = 0;
#pragma unroll
    for (int i = 0; i < ITERS; ++i) {
        const int32_t row = base + r0 + i * kAppendRows;
        const bool in = row >= lo && row < hi;
        const char* p = src + (((int64_t)(c0 + (in ? row - held : 0)) * a.n_kv + h) * kHeadDim + col) * EB;
#pragma unroll
        for (int j = 0; j < EB / 2; ++j) x[i * (EB / 2) + j] = in ? *reinterpret_cast<const uint4*>(p + 16 * j) : make_uint4(0, 0, 0, 0);
    }
#pragma unroll
    for (int i = 0; i < ITERS * EB / 2; ++i) {
        float f[16 / EB];
        unpack16<EB>(x[i], f);
#pragma unroll
        for (int j = 0; j < 16 / EB; ++j) {
            const uint32_t u = __float_as_uint(f[j]) & 0x7fffffffu;
            big = max(big, u < kInfBits ? u : 0u);
        }
    }
#pragma unroll
    for (int d = 32; d; d >>= 1) big = max(big, (uint32_t)__shfl_xor((int)big, d));
    if ((tid & 63) == 0) most[tid >> 6] = big;
    __syncthreads();
    big = max(max(most[0], most[1]), max(most[2], most[3]));
    const float s = fmaxf(old, scale_of(big));
    if (has_old && s > old) {
        const float f = old / s;
        for (int32_t row = r0; row < held - base; row += kAppendRows) {
            uint2* p = reinterpret_cast<uint2*>(dst + (int64_t)row * kHeadDim);
            const uint2 w = *p;
            *p = make_uint2(rescale(w.x, f), rescale(w.y, f));
        }
    }
    const float inv = 1.0f / s;
#pragma unroll
    for (int i = 0; i < ITERS; ++i) {
        const int32_t row = base + r0 + i * kAppendRows;
        if (row < lo || row >= hi) continue;
        float f[8];
#pragma unroll
        for (int j = 0; j < EB / 2; ++j) unpack16<EB>(x[i * (EB / 2) + j], f + j * (16 / EB));
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] *= inv;
        *reinterpret_cast<uint2*>(dst + (int64_t)(row - base) * kHeadDim) = make_uint2(codes_of(f[0], f[1], f[2], f[3]), codes_of(f[4], f[5], f[6], f[7]));
    }
    if (tid == 0) *scale = s;
    if (!is_v && a.acc)
        for (int32_t row = lo + tid; row < hi; row += kAppendThreads) a.acc[(int64_t)h * a.T_total + first + row] = 0.0f;
}

// ------------------------------------------------------------------------------------------------
// Attention of one token per sequence over the cache: l_j = q . k_j s_j / sqrt(D), out = sum softmax(l)_j v_j s'_j.  Bound by HBM: 256 bytes per row and KV
// head.  The codes become bf16, which holds them exactly, and go through 16x16x32 matrix instructions as the left operand, with the G
// queries of the head as the right one:
//   scores   rows = 16 tokens, contraction over D.  The order of the contraction is free: lane (c, g) (c = lane & 15, g = lane >> 4) takes the bytes
//            16 g .. 16 g + 15 of the first and of the second half of row c.
//   outputs  rows = 16 of the dims, contraction over 32 tokens.  The scores leave lane (c, g) with the tokens 4 g .. 4 g + 3 of two tiles for query c, which is
//            the right operand as it lies; the lane reads 8 bytes (dims 8 c .. 8 c + 7) of these 8 rows and transposes them in registers.
// Eight of the sixteen columns hold queries, the others the same queries again: the first eight carry the weights' leading 8 bits, the others what is left of
// them (the next 8), at no cost, so that a weight is off by at most 2^-18 of itself.  fp32 queries are split into three bf16 pieces that add up to them
// exactly.  Scores, maxima, sums and outputs are fp32.
// A wave keeps a running reference per query (moved up only where a score exceeds it by 2^8: weights are then at most 256); the waves of a block and the blocks
// of a (sequence, head) pair are joined by their references.
// ------------------------------------------------------------------------------------------------
constexpr int kCacheTile = 32;

struct CacheAttendArgs {
    const char* q;
    const uint8_t *K, *V;       // the layer's slices
    const float *ks, *vs;
    const int32_t *cu_tok, *n_tok, *tok_idx;
    int32_t max_n, T_total, n_scales, shift, n_kv, G, chunk, splits;
    int64_t logit_stride;
    float *out, *lse, *part, *ml, *lse2, *logits;
};

// Sixteen codes as bf16, in two operands.
__device__ __forceinline__ void widen16(const uint4& v, bf16x8_t* a, bf16x8_t* b) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const bf16x2_t lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[i], 1.0f, false), hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[i], 1.0f, true);
        bf16x8_t& d = i < 2 ? *a : *b;
        d[4 * (i & 1)] = lo[0];
        d[4 * (i & 1) + 1] = lo[1];
        d[4 * (i & 1) + 2] = hi[0];
        d[4 * (i & 1) + 3] = hi[1];
    }
}

__device__ __forceinline__ float max_groups(float x) {        // over the lanes with the same lane & 15
    const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    const auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

// PIECES: bf16 pieces of a query (1: bf16 queries, 3: fp32).  LISTED: rows by tok_idx, whose chunk and scales lie in LDS.  WEIGHTS: the scores are kept for
// the second launch.
template <int PIECES, bool LISTED, bool WEIGHTS, int NW>
__global__ __launch_bounds__(NW * kWave) void cache_attend_kernel(CacheAttendArgs a) {
    extern __shared__ __align__(16) char smem[];
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, c = lane & 15, g = lane >> 4, hq = c & 7;
    const int pair = blockIdx.y, b = pair / a.n_kv, h = pair % a.n_kv, split = blockIdx.x;
    int32_t first, rows;
    region(a.cu_tok, b, a.T_total, &first, &rows);
    int32_t n = min(max(a.n_tok[pair], 0), a.max_n);
    if (!LISTED) n = min(n, rows);
    const int32_t j0 = split * a.chunk, j1 = min(n, j0 + a.chunk);
    const int G = a.G;
    if (j0 >= j1 && split > 0) return;
    const uint8_t *Kh = a.K + ((int64_t)h * a.T_total + first) * kHeadDim, *Vh = a.V + ((int64_t)h * a.T_total + first) * kHeadDim;
    const float *ksh = a.ks + (int64_t)h * a.n_scales + (first >> a.shift) + b, *vsh = a.vs + (int64_t)h * a.n_scales + (first >> a.shift) + b;

    int32_t* l_idx = reinterpret_cast<int32_t*>(smem);                // [chunk]; behind them the scales
    float* l_ks = reinterpret_cast<float*>(smem) + a.chunk;
    float* l_vs = l_ks + a.chunk;
    if (LISTED) {
        const int32_t* idx = a.tok_idx + (int64_t)pair * a.max_n;
        for (int32_t j = tid; j < a.chunk; j += NW * kWave) {
            int32_t row = j0 + j < j1 ? idx[j0 + j] : -1;
            if (row < 0 || row >= rows) row = -1;
            l_idx[j] = row;
            l_ks[j] = row >= 0 ? ksh[row >> a.shift] : 0.0f;
            l_vs[j] = row >= 0 ? vsh[row >> a.shift] : 0.0f;
        }
        __syncthreads();
    }

    // the queries: columns c and c + 8 hold query c & 7 (zeros beyond G)
    bf16x8_t qf[PIECES][4];
    {
        const int64_t qrow = ((int64_t)pair * G + min(hq, G - 1)) * kHeadDim;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int d0 = (i >> 1) * 64 + g * 16 + (i & 1) * 8;
            if constexpr (PIECES == 1) {
                qf[0][i] = *reinterpret_cast<const bf16x8_t*>(a.q + (qrow + d0) * 2);
            } else {
                const float* f = reinterpret_cast<const float*>(a.q) + qrow + d0;
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    float x = f[j];
#pragma unroll
                    for (int p = 0; p < PIECES; ++p) {        // the leading 8 bits of what is left: exact, and three times 8 bits are all of them
                        const uint32_t top = __float_as_uint(x) & 0xffff0000u;
                        qf[p][i][j] = __builtin_bit_cast(__bf16, (uint16_t)(top >> 16));
                        x -= __uint_as_float(top);
                    }
                }
            }
        }
    }

    constexpr float kToLog2 = 0.08838834764831844f * 1.4426950408889634f;      // 1 / sqrt(D), base 2
    const float neg_inf = -__builtin_inff();
    float ref = neg_inf, sub = 0.0f, l = 0.0f;
    f32x4_t o[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) o[i] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};

    struct Tile { uint4 k[4]; uint2 v[8]; };
    auto row_of = [&](int32_t j) -> int32_t {                 // a row of the pool to read for entry j of the chunk
        if (LISTED) return max(l_idx[j], 0);
        return min(j0 + j, j1 - 1);
    };
    auto load = [&](Tile& t, int32_t j /* first entry of the tile, in the chunk */) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint8_t* p = Kh + (int64_t)row_of(j + 16 * i + c) * kHeadDim + 16 * g;
            t.k[2 * i] = *reinterpret_cast<const uint4*>(p);
            t.k[2 * i + 1] = *reinterpret_cast<const uint4*>(p + 64);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i)
            t.v[i] = *reinterpret_cast<const uint2*>(Vh + (int64_t)row_of(j + 16 * (i >> 2) + 4 * g + (i & 3)) * kHeadDim + 8 * c);
    };
    auto use = [&](Tile& t, int32_t j) {
        float x[8], sv[8];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            f32x4_t s = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int f = 0; f < 2; ++f) {
                bf16x8_t ka, kb;
                widen16(t.k[2 * i + f], &ka, &kb);
#pragma unroll
                for (int p = PIECES - 1; p >= 0; --p) {
                    s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ka, qf[p][2 * f], s, 0, 0, 0);
                    s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kb, qf[p][2 * f + 1], s, 0, 0, 0);
                }
            }
            if (LISTED) {
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int32_t e = j + 16 * i + 4 * g + r;
                    x[4 * i + r] = l_idx[e] >= 0 ? s[r] * (l_ks[e] * kToLog2) : neg_inf;
                    sv[4 * i + r] = l_vs[e];
                }
            } else {
                const int32_t blk = min(j0 + j + 16 * i, j1 - 1) >> a.shift;       // blocks are multiples of 16 rows
                const float sk = ksh[blk] * kToLog2, s2 = vsh[blk];
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    x[4 * i + r] = j0 + j + 16 * i + 4 * g + r < j1 ? s[r] * sk : neg_inf;
                    sv[4 * i + r] = s2;
                }
            }
        }
        if (WEIGHTS && c < G) {
            float* p = a.logits + ((int64_t)pair * G + c) * a.logit_stride + j0 + j + 4 * g;
            *reinterpret_cast<f32x4_t*>(p) = f32x4_t{x[0], x[1], x[2], x[3]};
            *reinterpret_cast<f32x4_t*>(p + 16) = f32x4_t{x[4], x[5], x[6], x[7]};
        }
        float top = fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])));
        top = max_groups(top);
        if (__any(top > ref + 8.0f)) {
            const float up = fmaxf(ref, top);
            sub = up == neg_inf ? 0.0f : up;
            const float f = __builtin_amdgcn_exp2f(ref - sub);
            ref = up;
            l *= f;
#pragma unroll
            for (int i = 0; i < 8; ++i) o[i] *= f;
        }
        bf16x8_t pf;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            x[i] = __builtin_amdgcn_exp2f(x[i] - sub);
            l += x[i];
        }
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
            const float y0 = x[i] * sv[i], y1 = x[i + 1] * sv[i + 1];
            const uint32_t lead = bf16_pair(y0, y1);
            const uint32_t rest = bf16_pair(y0 - __uint_as_float(lead << 16), y1 - __uint_as_float(lead & 0xffff0000u));
            const bf16x2_t pr = __builtin_bit_cast(bf16x2_t, c < 8 ? lead : rest);
            pf[i] = pr[0];
            pf[i + 1] = pr[1];
        }
        if (LISTED || j0 + j + kCacheTile > j1) {             // what is masked may be NaN, which no weight of zero takes away
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int32_t e = j + 16 * (i >> 2) + 4 * g + (i & 3);
                if (LISTED ? l_idx[e] < 0 : j0 + e >= j1) t.v[i] = make_uint2(0, 0);
            }
        }
        bf16x8_t vt[8];
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
#pragma unroll
            for (int d = 0; d < 4; ++d) {                     // dims 2 d and 2 d + 1 of tokens i and i + 1
                const uint32_t lo = d < 2 ? t.v[i].x : t.v[i].y, hi = d < 2 ? t.v[i + 1].x : t.v[i + 1].y;
                const uint32_t m = __builtin_amdgcn_perm(hi, lo, d & 1 ? 0x07030602u : 0x05010400u);
                const bf16x2_t e0 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(m, 1.0f, false), e1 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(m, 1.0f, true);
                vt[2 * d][i] = e0[0];
                vt[2 * d][i + 1] = e0[1];
                vt[2 * d + 1][i] = e1[0];
                vt[2 * d + 1][i + 1] = e1[1];
            }
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) o[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vt[i], pf, o[i], 0, 0, 0);
    };

    const int32_t count = j1 > j0 ? j1 - j0 : 0;
    Tile t0, t1;
    int32_t j = w * kCacheTile;
    constexpr int kStep = NW * kCacheTile;
    if (j < count) load(t0, j);
    while (j < count) {
        if (j + kStep < count) load(t1, j + kStep);
        use(t0, j);
        j += kStep;
        if (j >= count) break;
        if (j + kStep < count) load(t0, j + kStep);
        use(t1, j);
        j += kStep;
    }

    // join the waves: both halves of the columns, then all waves by their references
    l = sum_halves(sum_rows16(l));
    float* s_ref = reinterpret_cast<float*>(smem);            // [NW][8], then [NW][8] sums, then [NW][8][D]
    float* s_l = s_ref + NW * 8;
    float* s_o = s_l + NW * 8;
    if (LISTED) __syncthreads();
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) o[i][r] = dpp_add<0x128>(o[i][r]);
    if (c < 8) {
        if (g == 0) {
            s_ref[w * 8 + c] = ref;
            s_l[w * 8 + c] = l;
        }
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int i = 0; i < 8; i += 4)
                *reinterpret_cast<f32x4_t*>(s_o + ((w * 8 + c) * kHeadDim + (4 * g + r) * 8 + i)) = f32x4_t{o[i][r], o[i + 1][r], o[i + 2][r], o[i + 3][r]};
    }
    __syncthreads();
    for (int e = tid; e < G * kHeadDim; e += NW * kWave) {
        const int qg = e / kHeadDim, d = e % kHeadDim;
        float top = neg_inf;
#pragma unroll
        for (int i = 0; i < NW; ++i) top = fmaxf(top, s_ref[i * 8 + qg]);
        const float top0 = top == neg_inf ? 0.0f : top;
        float sum = 0.0f, z = 0.0f;
#pragma unroll
        for (int i = 0; i < NW; ++i) {
            const float f = __builtin_amdgcn_exp2f(s_ref[i * 8 + qg] - top0);
            z += f * s_l[i * 8 + qg];
            sum += f * s_o[(i * 8 + qg) * kHeadDim + d];
        }
        const int64_t qi = (int64_t)pair * G + qg;
        if (a.splits == 1) {
            a.out[qi * kHeadDim + d] = z == 0.0f ? 0.0f : sum / z;
            if (d == 0) {
                const float l2 = z == 0.0f ? neg_inf : top0 + __builtin_log2f(z);
                if (a.lse) a.lse[qi] = l2 * 0.6931471805599453f;
                if (WEIGHTS) a.lse2[qi] = l2;
            }
        } else {
            const int64_t pi = qi * a.splits + split;
            a.part[pi * kHeadDim + d] = sum;
            if (d == 0) *reinterpret_cast<float2*>(a.ml + 2 * pi) = make_float2(top, z);
        }
    }
}

// Joins the partial results of the blocks of a (sequence, query head): one block of D threads each.
__global__ __launch_bounds__(kHeadDim) void cache_join_kernel(CacheAttendArgs a, int listed) {
    const int64_t qi = blockIdx.x;
    const int pair = (int)(qi / a.G), b = pair / a.n_kv, d = threadIdx.x;
    int32_t first, rows;
    region(a.cu_tok, b, a.T_total, &first, &rows);
    int32_t n = min(max(a.n_tok[pair], 0), a.max_n);
    if (!listed) n = min(n, rows);
    const int splits = max(1, (n + a.chunk - 1) / a.chunk);
    const float2* ml = reinterpret_cast<const float2*>(a.ml) + qi * a.splits;
    const float* part = a.part + qi * a.splits * kHeadDim + d;
    const float neg_inf = -__builtin_inff();
    float top = neg_inf;
    for (int i = 0; i < splits; ++i) top = fmaxf(top, ml[i].x);
    const float top0 = top == neg_inf ? 0.0f : top;
    float sum = 0.0f, z = 0.0f;
    for (int i = 0; i < splits; ++i) {
        const float f = __builtin_amdgcn_exp2f(ml[i].x - top0);
        z += f * ml[i].y;
        sum += f * part[(int64_t)i * kHeadDim];
    }
    a.out[qi * kHeadDim + d] = z == 0.0f ? 0.0f : sum / z;
    if (d == 0) {
        const float l2 = z == 0.0f ? neg_inf : top0 + __builtin_log2f(z);
        if (a.lse) a.lse[qi] = l2 * 0.6931471805599453f;
        if (a.lse2) a.lse2[qi] = l2;
    }
}

// acc_out = decay * acc + the weights of the head's G queries, from the scores and the normalisers of the launches before.
constexpr int kWeightThreads = 256;
__global__ __launch_bounds__(kWeightThreads) void cache_weights_kernel(CacheAttendArgs a, const float* acc, float* acc_out, float decay) {
    const int pair = blockIdx.y, b = pair / a.n_kv, h = pair % a.n_kv;
    int32_t first, rows;
    region(a.cu_tok, b, a.T_total, &first, &rows);
    const int32_t n = min(min(max(a.n_tok[pair], 0), a.max_n), rows);
    const int32_t j = blockIdx.x * kWeightThreads + threadIdx.x;
    if (j >= n) return;
    const int64_t at = (int64_t)h * a.T_total + first + j;
    float sum = acc ? decay * acc[at] : 0.0f;
    for (int g = 0; g < a.G; ++g) {
        const float l2 = a.lse2[(int64_t)pair * a.G + g], x = a.logits[((int64_t)pair * a.G + g) * a.logit_stride + j];
        sum += l2 == -__builtin_inff() ? 0.0f : __builtin_amdgcn_exp2f(x - l2);
    }
    acc_out[at] = sum;
}

// ------------------------------------------------------------------------------------------------
// Eviction: which rows of a (layer, sequence, head) stay.  One block each.  The cut is found digit by digit (11, 11, 10 bits) in the order-preserving images of the
// weights, the kept rows are then written in order: every wave counts what it keeps of its share, and writes it behind the shares before.
// ------------------------------------------------------------------------------------------------
struct EvictArgs {
    const float* acc;
    const int32_t *cu_tok, *n_tok;
    int32_t B, n_kv, T_total, max_n, keep, sink, recent;
    int32_t *keep_idx, *n_keep;
};

__global__ __launch_bounds__(kBlockThreads) void cache_evict_kernel(EvictArgs a) {
    __shared__ uint32_t hist[2048];
    __shared__ uint32_t slot[kBlockWaves], slot2[kBlockWaves], found[2];
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    const int64_t row = blockIdx.x;                            // (layer * B + b) * Hkv + h
    const int h = (int)(row % a.n_kv), b = (int)(row / a.n_kv % a.B);
    const int64_t layer = row / a.n_kv / a.B;
    int32_t first, rows;
    region(a.cu_tok, b, a.T_total, &first, &rows);
    const int32_t n = min(min(max(a.n_tok[row], 0), a.max_n), rows);
    int32_t* out = a.keep_idx + row * max(a.keep, 1);
    if (tid == 0) a.n_keep[row] = min(n, a.keep);
    if (n <= a.keep) {
        for (int32_t j = tid; j < n; j += kBlockThreads) out[j] = j;
        return;
    }
    const float* acc = a.acc + (layer * a.n_kv + h) * (int64_t)a.T_total + first;
    const int32_t lo = a.sink, hi = n - a.recent;              // the rows that compete
    uint32_t need = (uint32_t)(a.keep - a.sink - a.recent);    // of them stay
    uint32_t prefix = 0, mask = 0;
    if (need > 0) {
#pragma unroll
        for (int pass = 0; pass < 3; ++pass) {
            const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bits = pass == 2 ? 10 : 11;
            for (int i = tid; i < 2048; i += kBlockThreads) hist[i] = 0;
            __syncthreads();
            for (int32_t j = lo + tid; j < hi; j += kBlockThreads) {
                const uint32_t key = score_key(acc[j]);
                if ((key & mask) == prefix) atomicAdd(&hist[(key >> shift) & ((1u << bits) - 1)], 1u);
            }
            __syncthreads();
            // digits from the largest down, two a thread: the one in which the count reaches `need`
            const uint32_t d0 = 2047 - 2 * tid, c0 = hist[d0], c1 = hist[d0 - 1];
            uint32_t total;
            const uint32_t upto = block_scan_u32(c0 + c1, slot, &total), before = upto - c0 - c1;
            if (before < need && need <= upto) {
                const bool second = need > before + c0;
                found[0] = d0 - (second ? 1 : 0);
                found[1] = need - before - (second ? c0 : 0);
            }
            __syncthreads();
            prefix |= found[0] << shift;
            mask |= ((1u << bits) - 1) << shift;
            need = found[1];
        }
    }
    // every row whose key is above `prefix`, and the first `need` of those equal to it; with need == 0 no row that competes
    const bool any = a.keep > a.sink + a.recent;
    const int32_t share = (n + kBlockThreads - 1) / kBlockThreads * 64, s0 = min(n, w * share), s1 = min(n, s0 + share);
    uint32_t above = 0, equal = 0;
    auto look = [&](int32_t j, bool* gt, bool* eq) {
        const bool in = j < s1, safe = j < lo || j >= hi;
        const uint32_t key = in && !safe ? score_key(acc[j]) : 0u;
        *gt = in && (safe || (any && key > prefix));
        *eq = in && !safe && any && key == prefix;
    };
    for (int32_t j = s0 + lane; j - lane < s1; j += 64) {
        bool gt, eq;
        look(j, &gt, &eq);
        above += (uint32_t)__popcll(__ballot(gt));
        equal += (uint32_t)__popcll(__ballot(eq));
    }
    if (lane == 0) {
        slot[w] = above;
        slot2[w] = equal;
    }
    __syncthreads();
    uint32_t gt_before = 0, eq_before = 0;
    for (int i = 0; i < w; ++i) {
        gt_before += slot[i];
        eq_before += slot2[i];
    }
    const unsigned long long below = (1ull << lane) - 1;
    for (int32_t j = s0 + lane; j - lane < s1; j += 64) {
        bool gt, eq;
        look(j, &gt, &eq);
        const unsigned long long bg = __ballot(gt), be = __ballot(eq);
        const uint32_t g_at = gt_before + (uint32_t)__popcll(bg & below), e_at = eq_before + (uint32_t)__popcll(be & below);
        if (gt || (eq && e_at < need)) out[g_at + min(e_at, need)] = j;
        gt_before += (uint32_t)__popcll(bg);
        eq_before += (uint32_t)__popcll(be);
    }
}

// ------------------------------------------------------------------------------------------------
// Compaction: row j of a head becomes row keep_idx[j].  Bound by HBM: the kept rows in and out.  One block takes all rows of a (layer, sequence, head, K or V) in
// ascending order, 128 at a time, reading a group before it writes it: a group's rows lie at or behind the place they go to, and those of later groups
// behind everything written, so the same buffers may be input and output.  A block's new scale is the largest of the scales its rows come with; a code of
// a smaller one is rounded again (exactly, but for what leaves the normal range).
// ------------------------------------------------------------------------------------------------
constexpr int kCompactRows = 128;

struct CompactArgs {
    const uint8_t *K, *V;
    const float *ks, *vs, *acc;
    uint8_t *K_out, *V_out;
    float *ks_out, *vs_out, *acc_out;
    const int32_t *cu_tok, *keep_idx, *n_keep;
    int32_t B, n_kv, T_total, n_scales, shift, keep;
};

__global__ __launch_bounds__(kBlockThreads) void cache_compact_kernel(CompactArgs a) {
    __shared__ int32_t s_src[kCompactRows];
    __shared__ float s_scale[kCompactRows];
    const int tid = threadIdx.x, r = tid >> 3, part = (tid & 7) * 16;
    const int64_t row = blockIdx.x;
    const int h = (int)(row % a.n_kv), b = (int)(row / a.n_kv % a.B);
    const int64_t head = row / a.n_kv / a.B * a.n_kv + h;
    const bool is_v = blockIdx.y != 0;
    int32_t first, rows;
    region(a.cu_tok, b, a.T_total, &first, &rows);
    const int32_t m = min(min(max(a.n_keep[row], 0), a.keep), rows);
    const int32_t* idx = a.keep_idx + row * a.keep;
    const int64_t pool = head * a.T_total + first, slot0 = head * a.n_scales + (first >> a.shift) + b;
    const uint8_t* src = (is_v ? a.V : a.K) + pool * kHeadDim + part;
    uint8_t* dst = (is_v ? a.V_out : a.K_out) + pool * kHeadDim + part;
    const float* sc = (is_v ? a.vs : a.ks) + slot0;
    float* sc_out = (is_v ? a.vs_out : a.ks_out) + slot0;
    const float least = __uint_as_float(27u << 23);
    const int block = 1 << a.shift;
    for (int32_t j0 = 0; j0 < m; j0 += kCompactRows) {
        const int32_t j = j0 + r;
        float w = 0.0f;
        if (tid < kCompactRows) {
            int32_t s = j0 + tid < m ? idx[j0 + tid] : -1;
            if (s < 0 || s >= rows) s = -1;
            s_src[tid] = s;
            s_scale[tid] = s >= 0 ? sc[s >> a.shift] : least;
            if (!is_v && a.acc && s >= 0) w = a.acc[pool + s];
        }
        __syncthreads();
        const int32_t from = s_src[r];
        uint4 v = from >= 0 ? *reinterpret_cast<const uint4*>(src + (int64_t)from * kHeadDim) : make_uint4(0, 0, 0, 0);
        float top = least;
        const int q0 = r & ~(block - 1);
        for (int i = 0; i < block; ++i) top = fmaxf(top, s_scale[q0 + i]);
        const float mine = s_scale[r];
        if (mine != top) {
            const float f = mine / top;
            v = make_uint4(rescale(v.x, f), rescale(v.y, f), rescale(v.z, f), rescale(v.w, f));
        }
        block_sync_after_stores();                            // the loads have arrived before any row is written
        if (j < m) {
            *reinterpret_cast<uint4*>(dst + (int64_t)j * kHeadDim) = v;
            if ((tid & 7) == 0 && r == q0) sc_out[j >> a.shift] = top;
        }
        if (!is_v && a.acc_out && tid < kCompactRows && j0 + tid < m) a.acc_out[pool + j0 + tid] = w;
    }
}

inline int64_t round_up(int64_t n, int64_t m) { return (n + m - 1) / m * m; }
inline int log2_of(int32_t n) { return 31 - __builtin_clz((unsigned)n); }

// How skv_cache_attend cuts its work: blocks of `chunk` rows per (sequence, head) pair, and where the parts of the workspace begin.
constexpr int kCacheWaves = 4;
struct AttendPlan {
    int32_t chunk, splits;
    int64_t logit_stride, ml, lse2, logits, bytes;
};
AttendPlan attend_plan(const Ctx* c, int32_t B, int32_t max_n, bool listed, bool weights) {
    AttendPlan p;
    const int64_t pairs = (int64_t)B * c->d.n_kv_heads, heads = pairs * c->G;
    const int32_t step = kCacheWaves * kCacheTile;
    int64_t splits = (4 * (int64_t)c->n_cu + pairs - 1) / pairs, most = (max_n + step - 1) / step;
    if (splits > most) splits = most;
    if (splits < 1) splits = 1;
    int64_t chunk = round_up((max_n + splits - 1) / splits, step);
    if (chunk < step) chunk = step;
    if (listed && chunk > 1024) chunk = 1024;
    p.chunk = (int32_t)chunk;
    p.splits = (int32_t)((max_n + chunk - 1) / chunk);
    if (p.splits < 1) p.splits = 1;
    p.logit_stride = round_up(max_n, kCacheTile);
    p.ml = round_up(p.splits > 1 ? heads * p.splits * kHeadDim * 4 : 0, 256);
    p.lse2 = p.ml + round_up(p.splits > 1 ? heads * p.splits * 8 : 0, 256);
    p.logits = p.lse2 + round_up(heads * 4, 256);
    p.bytes = p.logits + (weights ? round_up(heads * p.logit_stride * 4, 256) : 0);
    return p;
}

template <int PIECES, bool LISTED, bool WEIGHTS>
hipError_t attend_launch(Ctx* c, const CacheAttendArgs& a, int32_t pairs) {
    size_t lds = (size_t)kCacheWaves * 8 * (2 + kHeadDim) * 4;
    if (LISTED && (size_t)a.chunk * 12 > lds) lds = (size_t)a.chunk * 12;
    hipLaunchKernelGGL((cache_attend_kernel<PIECES, LISTED, WEIGHTS, kCacheWaves>), dim3(a.splits, pairs), dim3(kCacheWaves * kWave), lds, c->stream, a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_rotary(Ctx* c, int32_t n, const void* q, const void* k, const int32_t* pos, const double* inv_freq, int32_t rot, bool interleaved,
                         float mscale, void* q_out, void* k_out) {
    if (n == 0) return hipSuccess;
    const int EB = c->d.kv_dtype == SKV_BF16 ? 2 : 4;
    const bool vec = rot % 16 == 0;
    RotArgs a{(const char*)q, (const char*)k, (char*)q_out, (char*)k_out, pos, inv_freq, n, q ? c->d.n_q_heads : 0, k ? c->d.n_kv_heads : 0, rot / 2, 0, mscale};
    const int heads = a.n_q + a.n_k, rows = vec ? (EB == 2 ? 8 : 4) : 1;
    int groups = (heads + rows - 1) / rows;
    if (groups > 65535) groups = 65535;
    a.heads_per_wave = (heads + groups - 1) / groups;
    const dim3 grid((n + kRotWaves - 1) / kRotWaves, groups), block(kRotWaves * kWave);
    auto go = [&](auto eb, auto il) {
        constexpr int E = decltype(eb)::value;
        constexpr bool I = decltype(il)::value;
        if (vec) hipLaunchKernelGGL((rotary_kernel<E, I, true>), grid, block, 0, c->stream, a);
        else hipLaunchKernelGGL((rotary_kernel<E, I, false>), grid, block, 0, c->stream, a);
    };
    using std::integral_constant;
    if (EB == 2) interleaved ? go(integral_constant<int, 2>{}, std::true_type{}) : go(integral_constant<int, 2>{}, std::false_type{});
    else interleaved ? go(integral_constant<int, 4>{}, std::true_type{}) : go(integral_constant<int, 4>{}, std::false_type{});
    return hipGetLastError();
}

hipError_t launch_cache_append(Ctx* c, int32_t layer, int32_t B, const void* k, const void* v, int32_t n_new, const int32_t* cu_new, int32_t max_new,
                               const int32_t* cu_tok, const int32_t* n_tok, void* K, void* V, float* ks, float* vs, int32_t T_total, int32_t block, float* acc) {
    if (n_new == 0 || max_new == 0) return hipSuccess;
    const int H = c->d.n_kv_heads, n_scales = T_total / block + B;
    const int64_t pool = (int64_t)layer * H * T_total, sc = (int64_t)layer * H * n_scales;
    const AppendArgs a{(const char*)k, (const char*)v, (uint8_t*)K + pool * kHeadDim, (uint8_t*)V + pool * kHeadDim, ks + sc, vs + sc, acc ? acc + pool : nullptr,
                       cu_new, cu_tok, n_tok, n_new, max_new, T_total, n_scales, log2_of(block), H};
    const dim3 grid((unsigned)(((int64_t)max_new + block - 2) / block + 1), B * H, 2);
    auto go = [&](auto eb) {
        constexpr int E = decltype(eb)::value;
        switch (block) {
            case 16: hipLaunchKernelGGL((cache_append_kernel<E, 16>), grid, dim3(kAppendThreads), 0, c->stream, a); break;
            case 32: hipLaunchKernelGGL((cache_append_kernel<E, 32>), grid, dim3(kAppendThreads), 0, c->stream, a); break;
            case 64: hipLaunchKernelGGL((cache_append_kernel<E, 64>), grid, dim3(kAppendThreads), 0, c->stream, a); break;
            default: hipLaunchKernelGGL((cache_append_kernel<E, 128>), grid, dim3(kAppendThreads), 0, c->stream, a); break;
        }
    };
    if (c->d.kv_dtype == SKV_BF16) go(std::integral_constant<int, 2>{});
    else go(std::integral_constant<int, 4>{});
    return hipGetLastError();
}

int64_t cache_attend_work_bytes(const Ctx* c, int32_t B, int32_t max_n, bool weights) {
    const int64_t a = attend_plan(c, B, max_n, false, weights).bytes, b = attend_plan(c, B, max_n, true, false).bytes;
    return a > b ? a : b;
}

hipError_t launch_cache_attend(Ctx* c, int32_t layer, int32_t B, const void* q, const void* K, const void* V, const float* ks, const float* vs, int32_t T_total,
                               int32_t block, const int32_t* cu_tok, const int32_t* n_tok, const int32_t* tok_idx, int32_t max_n, float* out, float* lse,
                               const float* acc, float* acc_out, float decay, void* work) {
    const bool listed = tok_idx != nullptr, weights = acc_out != nullptr, wide = c->d.kv_dtype != SKV_BF16;
    const AttendPlan p = attend_plan(c, B, max_n, listed, weights);
    const int H = c->d.n_kv_heads, n_scales = T_total / block + B, pairs = B * H;
    const int64_t pool = (int64_t)layer * H * T_total, sc = (int64_t)layer * H * n_scales;
    char* ws = static_cast<char*>(work);
    const CacheAttendArgs a{(const char*)q, (const uint8_t*)K + pool * kHeadDim, (const uint8_t*)V + pool * kHeadDim, ks + sc, vs + sc, cu_tok, n_tok, tok_idx,
                            max_n, T_total, n_scales, log2_of(block), H, c->G, p.chunk, p.splits, p.logit_stride, out, lse, (float*)ws, (float*)(ws + p.ml),
                            weights ? (float*)(ws + p.lse2) : nullptr, (float*)(ws + p.logits)};
    hipError_t e;
    if (listed) e = wide ? attend_launch<3, true, false>(c, a, pairs) : attend_launch<1, true, false>(c, a, pairs);
    else if (weights) e = wide ? attend_launch<3, false, true>(c, a, pairs) : attend_launch<1, false, true>(c, a, pairs);
    else e = wide ? attend_launch<3, false, false>(c, a, pairs) : attend_launch<1, false, false>(c, a, pairs);
    if (e != hipSuccess) return e;
    if (p.splits > 1) {
        hipLaunchKernelGGL(cache_join_kernel, dim3(pairs * c->G), dim3(kHeadDim), 0, c->stream, a, listed ? 1 : 0);
        e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    if (weights && max_n > 0) {
        hipLaunchKernelGGL(cache_weights_kernel, dim3((max_n + kWeightThreads - 1) / kWeightThreads, pairs), dim3(kWeightThreads), 0, c->stream, a,
                           acc ? acc + pool : nullptr, acc_out + pool, decay);
        e = hipGetLastError();
    }
    return e;
}

hipError_t launch_cache_evict(Ctx* c, int32_t B, const float* acc, int32_t T_total, const int32_t* cu_tok, const int32_t* n_tok, int32_t max_n, int32_t keep,
                              int32_t sink, int32_t recent, int32_t* keep_idx, int32_t* n_keep) {
    const EvictArgs a{acc, cu_tok, n_tok, B, c->d.n_kv_heads, T_total, max_n, keep, sink, recent, keep_idx, n_keep};
    hipLaunchKernelGGL(cache_evict_kernel, dim3(c->d.n_layers * B * c->d.n_kv_heads), dim3(kBlockThreads), 0, c->stream, a);
    return hipGetLastError();
}

hipError_t launch_cache_compact(Ctx* c, int32_t B, const void* K, const void* V, const float* ks, const float* vs, const float* acc, int32_t T_total, int32_t block,
                                const int32_t* cu_tok, const int32_t* keep_idx, int32_t keep, const int32_t* n_keep, void* K_out, void* V_out, float* ks_out,
                                float* vs_out, float* acc_out) {
    if (keep == 0) return hipSuccess;
    const CompactArgs a{(const uint8_t*)K, (const uint8_t*)V, ks, vs, acc, (uint8_t*)K_out, (uint8_t*)V_out, ks_out, vs_out, acc_out, cu_tok, keep_idx, n_keep,
                        B, c->d.n_kv_heads, T_total, T_total / block + B, log2_of(block), keep};
    hipLaunchKernelGGL(cache_compact_kernel, dim3(c->d.n_layers * B * c->d.n_kv_heads, 2), dim3(kBlockThreads), 0, c->stream, a);
    return hipGetLastError();
}

}  // namespace skv
