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
typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));      // beginning at any word

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
// another (half layout) or in themselves (interleaved), so that a row may be turned where it lies.  32768 tokens of 40 bf16 heads: 113 us, 5.9 TB/s.
// ------------------------------------------------------------------------------------------------
constexpr int kRotWaves = 4, kRotRows = 4;

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

// VEC: rot is a multiple of 16.  Otherwise lanes hold neighbouring elements, whatever their partners are.  A wave's table of cosines and sines is its own: no barrier.
template <int EB, bool INTERLEAVED, bool VEC>
__global__ __launch_bounds__(kRotWaves * kWave) void rotary_kernel(RotArgs a) {
    __shared__ __align__(16) float2 table[kRotWaves][kHeadDim / 2];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const int heads = a.n_q + a.n_k, h0 = blockIdx.y * a.heads_per_wave, h1 = min(heads, h0 + a.heads_per_wave);
    const int64_t row_bytes = kHeadDim * EB;
    for (int64_t tok = (int64_t)blockIdx.x * kRotWaves + w; tok < a.n; tok += (int64_t)gridDim.x * kRotWaves) {
        auto row_in = [&](int h) { return h < a.n_q ? a.q + (tok * a.n_q + h) * row_bytes : a.k + (tok * a.n_k + (h - a.n_q)) * row_bytes; };
        auto row_out = [&](int h) { return h < a.n_q ? a.q_out + (tok * a.n_q + h) * row_bytes : a.k_out + (tok * a.n_k + (h - a.n_q)) * row_bytes; };
        auto angles = [&] {
            if (lane < a.half) {
                const double turns = (double)a.pos[tok] * a.inv_freq[lane] * 0.15915494309189533577;
                const float r = (float)(turns - rint(turns));
                float s, c;
                sincospif(2.0f * r, &s, &c);
                // what r's 32 bits left out, up to 2^-26 turns: the first order of its rotation (the second one is below 2^-47)
                const float rest = (float)(turns - rint(turns) - (double)r) * 6.283185307f;
                table[w][lane] = make_float2((c - s * rest) * a.mscale, (s + c * rest) * a.mscale);
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
        };
        if constexpr (VEC) {
            constexpr int E = 16 / EB, UNITS = kHeadDim / (2 * E), ROWS = kWave / UNITS;
            const int u = lane % UNITS, n_pairs = a.half / E;
            const bool turn = u < n_pairs;
            const int pa = (INTERLEAVED ? 2 * u : turn ? u : 2 * u) * 16, pb = INTERLEAVED || !turn ? pa + 16 : pa + n_pairs * 16;
            uint4 va, vb;
            auto load = [&](int h) {                          // past the last head: the last one again, which is not stored
                const char* in = row_in(min(h, heads - 1));
                va = ld_stream(in + pa);
                vb = ld_stream(in + pb);
            };
            load(h0 + lane / UNITS);                          // on its way while the angles are formed
            angles();
            float c[E], s[E];
#pragma unroll
            for (int i = 0; i < E; ++i) {
                const float2 t = turn ? table[w][u * E + i] : make_float2(1.0f, 0.0f);
                c[i] = t.x;
                s[i] = t.y;
            }
            for (int hb = h0; hb < h1; hb += ROWS) {
                const int h = hb + lane / UNITS;
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
                if (h < h1) {
                    char* out = row_out(h);
                    st_stream(out + pa, va);
                    st_stream(out + pb, vb);
                }
                if (hb + ROWS < h1) load(h + ROWS);
            }
        } else {
            // a lane has the elements 2 lane and 2 lane + 1 of kRotRows rows; partners that lie in other lanes (half layout) are read from LDS
            using Word = std::conditional_t<EB == 2, uint32_t, uint2>;
            __shared__ __align__(16) float rows[INTERLEAVED ? 1 : kRotWaves][kRotRows][kHeadDim];
            Word word[kRotRows];
            auto load = [&](int h) {                          // past the last head: the last one again, which is not stored
#pragma unroll
                for (int r = 0; r < kRotRows; ++r) word[r] = *reinterpret_cast<const Word*>(row_in(min(h + r, heads - 1)) + 2 * EB * lane);
            };
            load(h0);
            angles();
            // y = x * c + partner * s
            float c[2], s[2];
            int partner[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int e = 2 * lane + i;
                const bool turn = e < 2 * a.half, upper = INTERLEAVED ? i == 1 : e >= a.half;
                const float2 t = turn ? table[w][INTERLEAVED ? lane : upper ? e - a.half : e] : make_float2(1.0f, 0.0f);
                c[i] = t.x;
                s[i] = upper ? t.y : -t.y;
                partner[i] = !turn ? e : upper ? e - a.half : e + a.half;
            }
            for (int h = h0; h < h1; h += kRotRows) {
                float x[kRotRows][2];
#pragma unroll
                for (int r = 0; r < kRotRows; ++r) {
                    if constexpr (EB == 2) {
                        x[r][0] = __uint_as_float(word[r] << 16);
                        x[r][1] = __uint_as_float(word[r] & 0xffff0000u);
                    } else {
                        x[r][0] = __uint_as_float(word[r].x);
                        x[r][1] = __uint_as_float(word[r].y);
                    }
                    if (!INTERLEAVED) *reinterpret_cast<float2*>(&rows[w][r][2 * lane]) = make_float2(x[r][0], x[r][1]);
                }
                if (!INTERLEAVED) {
                    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
                    __builtin_amdgcn_wave_barrier();
                }
#pragma unroll
                for (int r = 0; r < kRotRows; ++r) {
                    float y[2];
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const bool turn = 2 * lane + i < 2 * a.half;
                        const float z = INTERLEAVED ? x[r][1 - i] : rows[w][r][partner[i]];
                        y[i] = turn ? x[r][i] * c[i] + z * s[i] : x[r][i];
                    }
                    if (h + r < h1) {
                        Word out;
                        if constexpr (EB == 2) {
                            out = bf16_pair(y[0], y[1]);
                            // what is copied is copied bit by bit
                            const uint32_t keep = (2 * lane < 2 * a.half ? 0u : 0xffffu) | (2 * lane + 1 < 2 * a.half ? 0u : 0xffff0000u);
                            out = (out & ~keep) | (word[r] & keep);
                        } else {
                            out = make_uint2(__float_as_uint(y[0]), __float_as_uint(y[1]));
                        }
                        *reinterpret_cast<Word*>(row_out(h + r) + 2 * EB * lane) = out;
                    }
                }
                if (!INTERLEAVED) {
                    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
                    __builtin_amdgcn_wave_barrier();
                }
                if (h + kRotRows < h1) load(h + kRotRows);
            }
        }
    }
}

// ------------------------------------------------------------------------------------------------
// Append: one block per (sequence, head, K or V, 32 to 128 rows of the scale blocks that take new rows).  Bound by HBM for prompts (the rows in, half or a quarter of
// their bytes out), by the chain of its loads for single tokens.  The block's new rows stay in registers between the search for the
// largest magnitude and the rounding.  Where rows are there already the scale can only grow; their codes are then rounded again.
// 32768 tokens of 8 bf16 heads: 35 us, 5.8 TB/s; a token of 16 sequences 5.0.
// ------------------------------------------------------------------------------------------------
constexpr int kAppendThreads = 256;
constexpr int kAppendRows = kAppendThreads / 16;          // rows at a time: 16 lanes of 8 elements
constexpr int kAppendSpan = 32;                           // rows of a launch block, at least (16384 tokens in blocks of 16: 25.0 us by 16 rows, 20.1 by 32, 20.5 by 64, 22.6 by 128)

struct AppendArgs {
    const char *k, *v;
    uint8_t *K, *V;             // the layer's slices
    float *ks, *vs, *acc;
    const int32_t *cu_new, *cu_tok, *n_tok;
    int32_t n_new, max_new, T_total, n_scales, n_kv;
};

template <int EB, int BLOCK>
__global__ __launch_bounds__(kAppendThreads) void cache_append_kernel(AppendArgs a) {
    constexpr int SPAN = BLOCK > kAppendSpan ? BLOCK : kAppendSpan, SUBS = SPAN / BLOCK;      // rows of a launch block, scale blocks among them
    constexpr int ITERS = SPAN / kAppendRows, PER = BLOCK / kAppendRows, WAVES = kAppendThreads / kWave;
    constexpr int SHIFT = BLOCK == 16 ? 4 : BLOCK == 32 ? 5 : BLOCK == 64 ? 6 : 7;
    __shared__ uint32_t most[2][SUBS][WAVES];
    const int pair = blockIdx.x, b = pair / a.n_kv, h = pair % a.n_kv;
    const bool is_v = blockIdx.z != 0;
    const int tid = threadIdx.x, col = (tid & 15) * 8, r0 = tid >> 4;
    int32_t first, rows;
    region(a.cu_tok, b, a.T_total, &first, &rows);
    const int32_t held = min(max(a.n_tok[pair], 0), rows);
    const int32_t c0 = max(a.cu_new[b], 0), c1 = min(a.cu_new[b + 1], a.n_new);
    const int32_t m = min(min(c1 > c0 ? c1 - c0 : 0, a.max_new), rows - held);
    if (m <= 0) return;
    const char* src = (is_v ? a.v : a.k) + (((int64_t)c0 * a.n_kv + h) * kHeadDim + col) * EB;
    const int64_t src_row = (int64_t)a.n_kv * kHeadDim * EB;
    float* scales = (is_v ? a.vs : a.ks) + (int64_t)h * a.n_scales + (first >> SHIFT) + b;
    uint8_t* pool = (is_v ? a.V : a.K) + ((int64_t)h * a.T_total + first) * kHeadDim + col;
    int buf = 0;
    for (int32_t t = (held >> SHIFT) + blockIdx.y * SUBS; t << SHIFT < held + m; t += gridDim.y * SUBS, buf ^= 1) {
        const int32_t base = t << SHIFT, lo = max(base, held), hi = min(base + SPAN, held + m);     // the new rows of this block
        const bool has_old = base < held;                     // in the first of its scale blocks
        const float old = has_old ? scales[t] : 0.0f;
        uint8_t* dst = pool + (int64_t)base * kHeadDim;
        uint4 x[ITERS * EB / 2];                              // rows that are not new: one that is, again (a load under a condition waits for those before it)
#pragma unroll
        for (int i = 0; i < ITERS; ++i) {
            const char* p = src + (min(max(base + r0 + i * kAppendRows, lo), hi - 1) - held) * src_row;
#pragma unroll
            for (int j = 0; j < EB / 2; ++j) x[i * (EB / 2) + j] = ld_stream(p + 16 * j);
        }
        uint32_t big[SUBS] = {};
#pragma unroll
        for (int i = 0; i < ITERS; ++i) {
            const int32_t row = base + r0 + i * kAppendRows;
            uint32_t top = 0;
#pragma unroll
            for (int e = 0; e < EB / 2; ++e) {
                float f[16 / EB];
                unpack16<EB>(x[i * (EB / 2) + e], f);
#pragma unroll
                for (int j = 0; j < 16 / EB; ++j) {
                    const uint32_t u = __float_as_uint(f[j]) & 0x7fffffffu;
                    top = max(top, u < kInfBits ? u : 0u);
                }
            }
            big[i / PER] = max(big[i / PER], row >= lo && row < hi ? top : 0u);
        }
#pragma unroll
        for (int s = 0; s < SUBS; ++s) {
#pragma unroll
            for (int d = 32; d; d >>= 1) big[s] = max(big[s], (uint32_t)__shfl_xor((int)big[s], d));
            if ((tid & 63) == 0) most[buf][s][tid >> 6] = big[s];
        }
        __syncthreads();
        float scale[SUBS];
#pragma unroll
        for (int s = 0; s < SUBS; ++s) scale[s] = scale_of(max(max(most[buf][s][0], most[buf][s][1]), max(most[buf][s][2], most[buf][s][3])));
        scale[0] = fmaxf(old, scale[0]);
        if (has_old && scale[0] > old) {
            const float f = old / scale[0];
            for (int32_t row = r0; row < held - base; row += kAppendRows) {
                uint2* p = reinterpret_cast<uint2*>(dst + (int64_t)row * kHeadDim);
                const uint2 w = *p;
                *p = make_uint2(rescale(w.x, f), rescale(w.y, f));
            }
        }
#pragma unroll
        for (int i = 0; i < ITERS; ++i) {
            const int32_t row = base + r0 + i * kAppendRows;
            const float inv = 1.0f / scale[i / PER];
            float f[8];
#pragma unroll
            for (int j = 0; j < EB / 2; ++j) unpack16<EB>(x[i * (EB / 2) + j], f + j * (16 / EB));
#pragma unroll
            for (int j = 0; j < 8; ++j) f[j] *= inv;
            const unsigned long long w = codes_of(f[0], f[1], f[2], f[3]) | (unsigned long long)codes_of(f[4], f[5], f[6], f[7]) << 32;
            if (row >= lo && row < hi) __builtin_nontemporal_store(w, reinterpret_cast<unsigned long long*>(dst + (int64_t)(row - base) * kHeadDim));
        }
#pragma unroll
        for (int s = 0; s < SUBS; ++s)
            if (tid == s && base + s * BLOCK < hi) scales[t + s] = scale[s];
        if (!is_v && a.acc)
            for (int32_t row = lo + tid; row < hi; row += kAppendThreads) a.acc[(int64_t)h * a.T_total + first + row] = 0.0f;
    }
}

// ------------------------------------------------------------------------------------------------
// Attention of one token per sequence over the cache: l_j = q . k_j s_j / sqrt(D), out = sum softmax(l)_j v_j s'_j.  Bound by HBM: 256 bytes per row and KV
// head.  The codes become bf16, which holds them exactly, and go through 16x16x32 matrix instructions as the left operand, with the G
// queries of the head as the right one:
//   scores   rows = 16 tokens, contraction over D.  The order of the contraction is free: lane (c, g) (c = lane & 15, g = lane >> 4) takes the bytes
//            16 g .. 16 g + 15 of the first and of the second half of row c.
//   outputs  rows = 16 of the dims, contraction over 32 tokens.  The scores leave lane (c, g) with the tokens 4 g .. 4 g + 3 of two tiles for query c, which is
//            the right operand as it lies; the lane reads 8 bytes (dims 8 c .. 8 c + 7) of these 8 rows and transposes them in registers.
// Eight of the sixteen columns hold queries, the others the same queries again, so that two pieces of 8 bits of the weights go through one instruction; with
// a second one for the last piece a weight keeps 24 bits.  (With two pieces results were off by 2e-6 of themselves, with three by 5e-7; the time is the same.)  fp32
// queries are split into three pieces that add up to them exactly.  Scores, maxima, sums and outputs are fp32.
// A wave keeps a running reference per query (scores are in powers of two; it is moved up only where one exceeds it by more than 8, so that weights are at most 256); the waves of a block
// and the blocks of a (sequence, head) pair are joined by their references.
// 131072 rows, 8 heads: 44 us, 6.1 TB/s, and the launch that joins.  With all of the arithmetic taken out it is the same: what counts is that the next tile is always on its way.
// ------------------------------------------------------------------------------------------------
constexpr int kCacheTile = 32, kCacheWaves = 4, kCacheStep = kCacheTile * kCacheWaves;
constexpr int kListedChunk = 1024;     // entries of a list per block, at most
constexpr int kJoinInside = 16;        // parts of a pair up to which the attention kernel joins them itself (16: 8.6 us, 9.0 by a launch of its own; 32: 11.8 and 9.2)
constexpr int kSharePairs = 1024, kShareMost = 4096;      // pairs up to which the blocks take equal shares of long batches, and of skewed ones
constexpr int kStageTiles = 8;         // tiles whose scores a wave keeps in LDS

// How the rows are dealt to blocks.  kGrid: blocks of `chunk` rows of a (sequence, head) pair.  kList: the same of its list.  kShare: the rows of all pairs in a row, in units
// of kCacheStep, in equal shares: sequences of unlike lengths keep every compute unit busy to the end.  A block that has rows of several pairs joins its waves
// for each of them.
enum CacheDeal { kGrid, kList, kShare };

struct CacheAttendArgs {
    const char* q;
    const uint8_t *K, *V;       // the layer's slices
    const float *ks, *vs;
    const int32_t *cu_tok, *n_tok, *tok_idx;
    int32_t max_n, T_total, n_scales, shift, n_kv, G, pairs, chunk, splits;
    int64_t logit_rows;         // rows of a pair in `logits`: [pair][tile][G][32]
    // Partial results by slots of G heads: part [slot][G][D] sums, ml [slot][G] (reference, normaliser).  A pair's slots lie side by side: from pair * splits on, or (kShare)
    // from block + pair on, which no two pieces share since from one piece to the next the block or the pair goes up.
    float *out, *lse, *part, *ml, *norm, *logits;      // norm [pair][G][2]: reference and 1 / normaliser of a query, for the weights
    int32_t* ends;              // kShare: [pairs][2] the first and the last block of each pair that has rows, for the launch that joins
    unsigned int* arrived;      // per pair, zero between launches; null: cache_finish_kernel joins
};

// 8 bytes that are read once.
__device__ __forceinline__ uint2 ld_stream8(const void* p) {
    typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
    const u32x2_t t = __builtin_nontemporal_load(reinterpret_cast<const u32x2_t*>(p));
    return make_uint2(t[0], t[1]);
}

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

// Rows in use of a pair.
__device__ __forceinline__ int32_t rows_in_use(const CacheAttendArgs& a, int pair, bool listed, int32_t* first, int32_t* rows) {
    region(a.cu_tok, pair / a.n_kv, a.T_total, first, rows);
    const int32_t n = min(max(a.n_tok[pair], 0), a.max_n);
    return listed ? n : min(n, *rows);
}

// What a weight is multiplied with: 1 / z, 0 where nothing is weighed.  Reference and normaliser stay apart: in one number, top0 + log2(z), the rounding of a
// reference of thousands would be a relative error of every weight of the query (a logit of 4200 in powers of two: 1e-4 of them).
__device__ __forceinline__ float share_of(float z) { return z == 0.0f ? 0.0f : 1.0f / z; }

__device__ __forceinline__ void store_out(const CacheAttendArgs& a, int64_t qi, int d, float sum, float z, float top0) {
    a.out[qi * kHeadDim + d] = z == 0.0f ? 0.0f : sum / z;
    if (d == 0) {
        const float l2 = z == 0.0f ? -__builtin_inff() : top0 + __builtin_log2f(z);
        if (a.lse) a.lse[qi] = l2 * 0.6931471805599453f;
        if (a.norm) *reinterpret_cast<float2*>(a.norm + 2 * qi) = make_float2(top0, share_of(z));
    }
}

// PIECES: bf16 pieces of a query (1: bf16 queries, 3: fp32).  kList: the chunk's rows and their scales lie in LDS.  WEIGHTS: the scores are kept for the last launch.
// Blocks of four waves that a compute unit holds, by the registers of each form.
constexpr int cache_places(int pieces, int deal, bool weights) { return pieces == 1 ? (deal == kShare || weights ? 3 : 4) : deal == kShare ? 2 : 3; }

template <int PIECES, int DEAL, bool WEIGHTS>
__global__ __launch_bounds__(kCacheWaves * kWave, cache_places(PIECES, DEAL, WEIGHTS)) void cache_attend_kernel(CacheAttendArgs a) {
    extern __shared__ __align__(16) char smem_all[];
    constexpr bool LISTED = DEAL == kList;
    constexpr int kThreads = kCacheWaves * kWave;
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), c = lane & 15, g = lane >> 4, hq = c & 7;
    const int G = a.G;
    int32_t* s_units = reinterpret_cast<int32_t*>(smem_all);          // kShare: [pairs + 1], ahead of the rest
    char* smem = smem_all + (DEAL == kShare ? (a.pairs + 4) / 4 * 16 : 0);
    int pair = blockIdx.y, slot = blockIdx.y * a.splits + blockIdx.x;
    int32_t unit = 0, unit_end = 0;
    if (DEAL == kShare) {
        __shared__ int32_t s_wave[kCacheWaves];
        constexpr int kEach = 4;
        int32_t carried = 0;                                  // units before these pairs
        int p0 = 0;
        do {
            int32_t u[kEach], sum = 0;
#pragma unroll
            for (int i = 0; i < kEach; ++i) {
                const int p = p0 + tid * kEach + i;
                int32_t f, r;
                const int32_t m = rows_in_use(a, min(p, a.pairs - 1), false, &f, &r);
                u[i] = p < a.pairs ? (m + kCacheStep - 1) / kCacheStep : 0;
                sum += u[i];
            }
            const int32_t upto = (int32_t)wave_scan_u32((uint32_t)sum);
            if (lane == 63) s_wave[w] = upto;
            __syncthreads();
            int32_t before = carried + upto - sum;
#pragma unroll
            for (int i = 0; i < kCacheWaves; ++i) {
                before += i < w ? s_wave[i] : 0;
                carried += s_wave[i];
            }
#pragma unroll
            for (int i = 0; i < kEach; ++i) {
                const int p = p0 + tid * kEach + i;
                before += u[i];
                if (p < a.pairs) s_units[p + 1] = before;
            }
            p0 += kEach * kThreads;
            if (p0 < a.pairs) __syncthreads();
        } while (p0 < a.pairs);
        if (tid == 0) s_units[0] = 0;
        __syncthreads();
        const int32_t all = s_units[a.pairs], n_blocks = min((int32_t)gridDim.x, all);
        if ((int32_t)blockIdx.x >= n_blocks) return;
        unit = (int32_t)((int64_t)all * blockIdx.x / n_blocks);
        unit_end = (int32_t)((int64_t)all * (blockIdx.x + 1) / n_blocks);
        int lo = 0, hi = a.pairs;                             // the last pair that begins at or before `unit`, of those that begin there the one with rows
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (s_units[mid] <= unit) lo = mid;
            else hi = mid;
        }
        pair = __builtin_amdgcn_readfirstlane(lo);
        unit = __builtin_amdgcn_readfirstlane(unit);
        unit_end = __builtin_amdgcn_readfirstlane(unit_end);
    }

    for (;;) {                                                // kShare: the pieces of the block's share; otherwise once
    const int b = pair / a.n_kv, h = pair % a.n_kv;
    const int32_t begin = DEAL == kShare ? __builtin_amdgcn_readfirstlane(s_units[pair]) : 0, stop = DEAL == kShare ? min(unit_end, (int32_t)__builtin_amdgcn_readfirstlane(s_units[pair + 1])) : 0;
    const int32_t j0 = DEAL == kShare ? (unit - begin) * kCacheStep : (int32_t)blockIdx.x * a.chunk;
    if (DEAL == kShare) {
        slot = blockIdx.x + pair;
        if (tid == 0 && unit == begin) a.ends[2 * pair] = blockIdx.x;
        if (tid == 0 && unit_end >= s_units[pair + 1]) a.ends[2 * pair + 1] = blockIdx.x;
    }

    // a list's entries are asked for first: rows and scales wait for them
    constexpr int kEntries = LISTED ? kListedChunk / kThreads : 1;
    int32_t entry[kEntries];
    if (LISTED) {
        const int32_t* idx = a.tok_idx + (int64_t)pair * a.max_n;
#pragma unroll
        for (int i = 0; i < kEntries; ++i) entry[i] = idx[min(j0 + tid + i * kThreads, a.max_n - 1)];
    }
    // the queries: columns c and c + 8 hold query c & 7 (the last one again beyond G)
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
                        x = p == 0 && __builtin_fabsf(x) == __builtin_inff() ? 0.0f : x - __uint_as_float(top);      // nothing is left of an infinity (NaN stays: its first piece may be one)
                    }
                }
            }
        }
    }
    int32_t first, rows;
    const int32_t n = rows_in_use(a, pair, LISTED, &first, &rows);
    const int32_t j1 = DEAL == kShare ? min(n, (stop - begin) * kCacheStep) : min(n, j0 + a.chunk), count = j1 > j0 ? j1 - j0 : 0;       // entries of this piece
    if (DEAL != kShare && count == 0 && blockIdx.x > 0) return;
    // rows: the piece's first row, with 32-bit offsets from it; a list: the sequence's first row
    const int64_t row0 = (int64_t)h * a.T_total + first + (LISTED ? 0 : j0);
    const uint8_t *Kh = a.K + row0 * kHeadDim, *Vh = a.V + row0 * kHeadDim;
    const float *ksh = a.ks + (int64_t)h * a.n_scales + (first >> a.shift) + b, *vsh = a.vs + (int64_t)h * a.n_scales + (first >> a.shift) + b;

    int32_t* l_idx = reinterpret_cast<int32_t*>(smem);                // [chunk]; behind them the scales
    float* l_ks = reinterpret_cast<float*>(smem) + a.chunk;
    float* l_vs = l_ks + a.chunk;
    // WEIGHTS: the wave's scores of up to kStageTiles tiles, [tile][G][32].  A store to memory for every tile would be waited for with the next tile's loads.
    float* l_x = reinterpret_cast<float*>(smem) + w * G * kStageTiles * kCacheTile;
    float e_ks[kEntries], e_vs[kEntries];
    if (LISTED) {
#pragma unroll
        for (int i = 0; i < kEntries; ++i) {
            const int32_t j = tid + i * kThreads;
            if (j >= count || entry[i] < 0 || entry[i] >= rows) entry[i] = -1;
            if (j < a.chunk) l_idx[j] = entry[i];
            e_ks[i] = ksh[max(entry[i], 0) >> a.shift];
            e_vs[i] = vsh[max(entry[i], 0) >> a.shift];
        }
        __syncthreads();
    }

    constexpr float kToLog2 = 0.08838834764831844f * 1.4426950408889634f;      // 1 / sqrt(D), base 2
    const float neg_inf = -__builtin_inff();
    float ref = neg_inf, sub = 0.0f, l = 0.0f;
    f32x4_t o[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) o[i] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
    uint4 kt[4];                                              // the tile's codes: K, then V
    uint2 vv[8];
    float sk[2], sv2[2];                                      // rows: the scales of the tile's two groups of 16 (blocks are multiples of 16)

    // A tile's scales are asked for with its keys: loads return in order, so that scales asked for later would be waited for with everything before them.
    // Values come by non-temporal loads (2.4 M rows in plain ones 130 us, in these 124), keys by plain ones: a load takes half of a line, and the other one may be lost between
    // non-temporal ones (32 lists of 2048 rows 33 us, with plain ones 28).
    auto load_k = [&](int32_t j /* first entry of the tile, in the piece */) {
        if (LISTED) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const uint8_t* p = Kh + (int64_t)max(l_idx[min(j + 16 * i + c, a.chunk - 1)], 0) * kHeadDim + 16 * g;
                kt[2 * i] = *reinterpret_cast<const uint4*>(p);
                kt[2 * i + 1] = *reinterpret_cast<const uint4*>(p + 64);
            }
            return;
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int32_t blk = min(j0 + j + 16 * i, j1 - 1) >> a.shift;
            sk[i] = ksh[blk];
            sv2[i] = vsh[blk];
        }
        const uint8_t* base = Kh + (uint32_t)j * kHeadDim;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint32_t off = (uint32_t)min(16 * i + c, count - 1 - j) * kHeadDim + 16 * g;
            kt[2 * i] = *reinterpret_cast<const uint4*>(base + off);
            kt[2 * i + 1] = *reinterpret_cast<const uint4*>(base + off + 64);
        }
    };
    auto load_v = [&](int32_t j) {
        const uint8_t* base = LISTED ? Vh : Vh + (uint32_t)j * kHeadDim;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int e = 16 * (i >> 2) + 4 * g + (i & 3);
            if (LISTED) vv[i] = ld_stream8(base + (int64_t)max(l_idx[min(j + e, a.chunk - 1)], 0) * kHeadDim + 8 * c);
            else vv[i] = ld_stream8(base + (uint32_t)(min(e, count - 1 - j) * kHeadDim + 8 * c));
        }
    };
    // WEIGHTS: the staged tiles, the first of them at entry j, to memory
    auto flush = [&](int32_t j) {
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        float* to = a.logits + ((int64_t)pair * a.logit_rows + j0 + j) * G;
        for (int e = lane * 4; e < kStageTiles * G * kCacheTile; e += kWave * 4) {
            const int tile = e / (G * kCacheTile);            // a power of two
            if (j + tile * kCacheStep < count)
                *reinterpret_cast<f32x4_t*>(to + (int64_t)tile * kCacheStep * G + (e & (G * kCacheTile - 1))) = *reinterpret_cast<const f32x4_t*>(l_x + e);
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    };

    int32_t j = w * kCacheTile, staged = j;
    if (j < count) {
        load_k(j);
        load_v(j);
    }
    if (LISTED) {                                             // the scales, while the first rows are on their way
#pragma unroll
        for (int i = 0; i < kEntries; ++i) {
            const int32_t e = tid + i * kThreads;
            if (e < a.chunk) {
                l_ks[e] = entry[i] >= 0 ? e_ks[i] * kToLog2 : 0.0f;           // of no row: nothing that was read in its place
                l_vs[e] = entry[i] >= 0 ? e_vs[i] : 0.0f;
            }
        }
        __syncthreads();
    }
    for (; j < count; j += kCacheStep) {
        float x[8], sv[8];
        const bool tail = LISTED || j + kCacheTile > count;   // some of its entries may be none
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            f32x4_t s = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int f = 0; f < 2; ++f) {
                bf16x8_t ka, kb;
                widen16(kt[2 * i + f], &ka, &kb);
#pragma unroll
                for (int p = PIECES - 1; p >= 0; --p) {
                    s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ka, qf[p][2 * f], s, 0, 0, 0);
                    s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kb, qf[p][2 * f + 1], s, 0, 0, 0);
                }
            }
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int32_t e = j + 16 * i + 4 * g + r;
                x[4 * i + r] = s[r] * (LISTED ? l_ks[e] : sk[i] * kToLog2);
                sv[4 * i + r] = LISTED ? l_vs[e] : sv2[i];
            }
        }
        if (tail) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int32_t e = j + 16 * (i >> 2) + 4 * g + (i & 3);
                if (LISTED ? l_idx[e] < 0 : e >= count) x[i] = neg_inf;
            }
        }
        // The next tile's keys, while the rest of this one is computed, and its values behind the last use of these.  Past the last tile that is one row again: loads
        // under a condition would make the compiler wait for the values where it waits for the keys.
        const int32_t next = min(j + kCacheStep, count - 1);
        load_k(next);
        if (WEIGHTS) {
            const int at = (j - staged) / kCacheStep;
            if (c < G) {
                float* p = l_x + (at * G + c) * kCacheTile + 4 * g;
                *reinterpret_cast<f32x4_t*>(p) = f32x4_t{x[0], x[1], x[2], x[3]};
                *reinterpret_cast<f32x4_t*>(p + 16) = f32x4_t{x[4], x[5], x[6], x[7]};
            }
            if (at == kStageTiles - 1 || j + kCacheStep >= count) {
                flush(staged);
                staged = j + kCacheStep;
            }
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
        // the weights (times the rows' scales) in three pieces of 8 bits: the first columns carry the leading and the last one, the others the middle one
        bf16x8_t pf, pl;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            x[i] = __builtin_amdgcn_exp2f(x[i] - sub);
            l += x[i];
        }
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
            const float y0 = x[i] * sv[i], y1 = x[i + 1] * sv[i + 1];
            const uint32_t lead = bf16_pair(y0, y1);
            const float r0 = y0 - __uint_as_float(lead << 16), r1 = y1 - __uint_as_float(lead & 0xffff0000u);
            const uint32_t mid = bf16_pair(r0, r1), low = bf16_pair(r0 - __uint_as_float(mid << 16), r1 - __uint_as_float(mid & 0xffff0000u));
            const bf16x2_t a2 = __builtin_bit_cast(bf16x2_t, c < 8 ? lead : mid), b2 = __builtin_bit_cast(bf16x2_t, c < 8 ? low : 0u);
            pf[i] = a2[0];
            pf[i + 1] = a2[1];
            pl[i] = b2[0];
            pl[i + 1] = b2[1];
        }
        if (tail) {                                           // what is masked may be NaN, which no weight of zero takes away
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int32_t e = j + 16 * (i >> 2) + 4 * g + (i & 3);
                if (LISTED ? l_idx[e] < 0 : e >= count) vv[i] = make_uint2(0, 0);
            }
        }
#pragma unroll
        for (int d = 0; d < 4; ++d) {                         // dims 2 d and 2 d + 1 of the lane's 8 rows
            bf16x8_t va, vb;
#pragma unroll
            for (int i = 0; i < 8; i += 2) {
                const uint32_t lo = d < 2 ? vv[i].x : vv[i].y, hi = d < 2 ? vv[i + 1].x : vv[i + 1].y;
                const uint32_t m = __builtin_amdgcn_perm(hi, lo, d & 1 ? 0x07030602u : 0x05010400u);
                const bf16x2_t e0 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(m, 1.0f, false), e1 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(m, 1.0f, true);
                va[i] = e0[0];
                va[i + 1] = e0[1];
                vb[i] = e1[0];
                vb[i + 1] = e1[1];
            }
            o[2 * d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(va, pl, o[2 * d], 0, 0, 0);
            o[2 * d + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vb, pl, o[2 * d + 1], 0, 0, 0);
            o[2 * d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(va, pf, o[2 * d], 0, 0, 0);
            o[2 * d + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vb, pf, o[2 * d + 1], 0, 0, 0);
        }
        load_v(next);
    }

    // join the waves: both halves of the columns, then all waves by their references
    l = sum_halves(sum_rows16(l));
    float* s_ref = reinterpret_cast<float*>(smem);            // [waves][8], then [waves][8] sums, then [waves][8][D]
    float* s_l = s_ref + kCacheWaves * 8;
    float* s_o = s_l + kCacheWaves * 8;
    if (LISTED || WEIGHTS) __syncthreads();
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
    for (int e = tid; e < G * kHeadDim; e += kThreads) {
        const int qg = e / kHeadDim, d = e % kHeadDim;
        float top = neg_inf;
#pragma unroll
        for (int i = 0; i < kCacheWaves; ++i) top = fmaxf(top, s_ref[i * 8 + qg]);
        const float top0 = top == neg_inf ? 0.0f : top;
        float sum = 0.0f, z = 0.0f;
#pragma unroll
        for (int i = 0; i < kCacheWaves; ++i) {
            const float f = __builtin_amdgcn_exp2f(s_ref[i * 8 + qg] - top0);
            z += f * s_l[i * 8 + qg];
            sum += f * s_o[(i * 8 + qg) * kHeadDim + d];
        }
        if (DEAL != kShare && a.splits == 1) {
            store_out(a, (int64_t)pair * G + qg, d, sum, z, top0);
            continue;
        }
        const int64_t pi = (int64_t)slot * G + qg;
        if (DEAL != kShare && a.arrived) {
            st_agent(a.part + pi * kHeadDim + d, sum);
            if (d == 0) st_agent64(reinterpret_cast<float2*>(a.ml) + pi, top, z);
        } else {
            a.part[pi * kHeadDim + d] = sum;
            if (d == 0) *reinterpret_cast<float2*>(a.ml + 2 * pi) = make_float2(top, z);
        }
    }
    if (DEAL == kShare) {
        if (stop >= unit_end) return;
        unit = stop;
        for (++pair; __builtin_amdgcn_readfirstlane(s_units[pair + 1]) <= unit; ++pair) {}      // `unit` belongs to a pair, since it is below the last one's end
        __syncthreads();
        continue;
    }
    if (!a.arrived) return;

    // few parts: the block that arrives last joins them, head by head in a fixed order
    __shared__ int s_last;
    const int parts = max(1, (n + a.chunk - 1) / a.chunk);
    block_sync_after_stores();
    if (tid == 0) {
        const bool last = __hip_atomic_fetch_add(a.arrived + pair, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (unsigned)parts - 1;
        if (last) st_agent(a.arrived + pair, 0u);
        s_last = last;
    }
    __syncthreads();
    if (!s_last) return;
    // Everything is asked for at once: the references (through LDS, for all) and the sums of the two dims of up to two heads that a thread adds up.
    float2* s_ml = reinterpret_cast<float2*>(smem);           // [parts][G], at most 8 * kJoinInside = the threads
    constexpr int kItems = 8 * (kHeadDim / 2) / kThreads;
    const int64_t pi0 = (int64_t)pair * a.splits * G;
    const unsigned long long m_own = ld_agent64(a.ml + 2 * (pi0 + min(tid, G * parts - 1)));
    unsigned long long v[kItems][kJoinInside];
    auto sums = [&](int k) {                                  // of the thread's item k
        const int e = min(tid + k * kThreads, G * (kHeadDim / 2) - 1);
        return a.part + (pi0 + e / (kHeadDim / 2)) * kHeadDim + e % (kHeadDim / 2) * 2;
    };
#pragma unroll
    for (int k = 0; k < kItems; ++k)
        if (k * kThreads < G * (kHeadDim / 2)) {
#pragma unroll
            for (int i = 0; i < kJoinInside; ++i) v[k][i] = ld_agent64(sums(k) + (int64_t)min(i, parts - 1) * G * kHeadDim);
        }
    if (tid < G * parts) s_ml[tid] = make_float2(lo_f(m_own), hi_f(m_own));
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kItems; ++k) {
        const int e = tid + k * kThreads, qg = e / (kHeadDim / 2), d = e % (kHeadDim / 2) * 2;
        if (e >= G * (kHeadDim / 2)) break;
        float top = neg_inf, z = 0.0f, s0 = 0.0f, s1 = 0.0f;
        for (int i = 0; i < parts; ++i) top = fmaxf(top, s_ml[i * G + qg].x);
        const float top0 = top == neg_inf ? 0.0f : top;
        auto add = [&](int i, unsigned long long p) {
            const float2 m = s_ml[i * G + qg];
            const float f = __builtin_amdgcn_exp2f(m.x - top0);
            z += f * m.y;
            s0 += f * lo_f(p);
            s1 += f * hi_f(p);
        };
#pragma unroll
        for (int i = 0; i < kJoinInside; ++i)
            if (i < parts) add(i, v[k][i]);
        const int64_t qi = (int64_t)pair * G + qg;
        store_out(a, qi, d, s0, z, top0);
        store_out(a, qi, d + 1, s1, z, top0);
    }
    return;
    }
}

// What is left behind the attention launch, in one: blocks that join the partial results of a (sequence, query head), and blocks that add up the weights of 1024 rows of a
// pair.  Neither waits for the other: the normalisers are as few numbers as there are parts, and whoever needs them takes them from there.
constexpr int kFinishThreads = 256, kWeightRows = 4;          // rows a thread

struct FinishArgs {
    int32_t listed, share;      // whether the attention launch was kList, kShare
    int32_t joins;              // blocks of a pair that join: its heads (0: joined already)
    const float* acc;
    float *acc_out, decay;
};

// The slots of a pair's parts.
__device__ __forceinline__ int parts_of(const CacheAttendArgs& a, const FinishArgs& f, int pair, int64_t* slot) {
    int32_t first, rows;
    const int32_t n = rows_in_use(a, pair, f.listed != 0, &first, &rows);
    if (f.share) {
        const int32_t k0 = a.ends[2 * pair], k1 = a.ends[2 * pair + 1];
        *slot = n > 0 ? k0 + pair : 0;
        return n > 0 ? k1 - k0 + 1 : 0;
    }
    *slot = (int64_t)pair * a.splits;
    return max(1, (n + a.chunk - 1) / a.chunk);
}

// The largest reference and the normaliser relative to it (0 where that is -inf) of parts ml[0], ml[G], ..., by one wave.
__device__ __forceinline__ float2 normaliser(const float2* ml, int parts, int G, int lane) {
    const float neg_inf = -__builtin_inff();
    const float2 own = lane < parts ? ml[(int64_t)lane * G] : make_float2(neg_inf, 0.0f);      // mostly all there are
    float top = own.x;
    for (int i = lane + kWave; i < parts; i += kWave) top = fmaxf(top, ml[(int64_t)i * G].x);
#pragma unroll
    for (int m = 32; m; m >>= 1) top = fmaxf(top, __shfl_xor(top, m));
    const float top0 = top == neg_inf ? 0.0f : top;
    float z = __builtin_amdgcn_exp2f(own.x - top0) * own.y;
    for (int i = lane + kWave; i < parts; i += kWave) {
        const float2 v = ml[(int64_t)i * G];
        z += __builtin_amdgcn_exp2f(v.x - top0) * v.y;
    }
#pragma unroll
    for (int m = 32; m; m >>= 1) z += __shfl_xor(z, m);
    return make_float2(top0, z);
}

// Eight parts of a head at a time.
__device__ __forceinline__ void join_head(const CacheAttendArgs& a, const FinishArgs& f, int pair, int qg, float* s_o) {
    constexpr int ROWS = kFinishThreads / (kHeadDim / 4);
    const int tid = threadIdx.x, r = tid / (kHeadDim / 4), d = tid % (kHeadDim / 4) * 4;
    int64_t slot;
    const int parts = parts_of(a, f, pair, &slot);
    const float2* ml = reinterpret_cast<const float2*>(a.ml) + slot * a.G + qg;
    const float* part = a.part + (slot * a.G + qg) * kHeadDim + d;
    const float2 n = normaliser(ml, parts, a.G, tid & 63);    // every wave for itself
    f32x4_t sum = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 4
    for (int i = r; i < parts; i += ROWS) sum += __builtin_amdgcn_exp2f(ml[(int64_t)i * a.G].x - n.x) * *reinterpret_cast<const f32x4_t*>(part + (int64_t)i * a.G * kHeadDim);
    *reinterpret_cast<f32x4_t*>(s_o + r * kHeadDim + d) = sum;
    __syncthreads();
    if (tid < kHeadDim) {
        float v = 0.0f;
#pragma unroll
        for (int i = 0; i < ROWS; ++i) v += s_o[i * kHeadDim + tid];
        store_out(a, (int64_t)pair * a.G + qg, tid, v, n.y, n.x);
    }
}

// G: query heads of a KV head whose weights are added up: acc_out = decay * acc + their sum; 0: none.
template <int G>
__global__ __launch_bounds__(kFinishThreads) void cache_finish_kernel(CacheAttendArgs a, FinishArgs f) {
    __shared__ __align__(16) float s_o[kFinishThreads * 4];
    const int pair = blockIdx.y, tid = threadIdx.x;
    if ((int)blockIdx.x < f.joins) {
        join_head(a, f, pair, blockIdx.x, s_o);
        return;
    }
    if constexpr (G > 0) {
        const int b = pair / a.n_kv, h = pair % a.n_kv;
        int32_t first, rows;
        region(a.cu_tok, b, a.T_total, &first, &rows);
        const int32_t n = min(min(max(a.n_tok[pair], 0), a.max_n), rows), j0 = (int32_t)(blockIdx.x - f.joins) * kFinishThreads * kWeightRows;
        if (j0 >= n) return;
        const int32_t j = min(j0 + tid * kWeightRows, n - 1) / kWeightRows * kWeightRows;      // past the end: the last rows again, which are not stored
        const int64_t at = (int64_t)h * a.T_total + first + j;
        f32x4_t x[G];                                         // scores of 4 rows: 16-byte loads; the weights begin anywhere
        float2 norm[G];
        float sum[kWeightRows];
#pragma unroll
        for (int g = 0; g < G; ++g)
            x[g] = __builtin_nontemporal_load(reinterpret_cast<const f32x4_t*>(a.logits + ((int64_t)pair * a.logit_rows + j / kCacheTile * kCacheTile) * G + g * kCacheTile + j % kCacheTile));
        const bool whole = j + kWeightRows <= n;
        f32x4_any weights = {0.0f, 0.0f, 0.0f, 0.0f};
        if (f.acc) {
            if (whole) {
                weights = *reinterpret_cast<const f32x4_any*>(f.acc + at);
            } else {
#pragma unroll
                for (int r = 0; r < kWeightRows; ++r) weights[r] = f.acc[at + min(r, n - 1 - j)];
            }
        }
#pragma unroll
        for (int r = 0; r < kWeightRows; ++r) sum[r] = f.acc ? f.decay * weights[r] : 0.0f;
        if (f.joins) {
            int64_t slot;
            const int parts = parts_of(a, f, pair, &slot);
            for (int g = tid >> 6; g < G; g += kFinishThreads / kWave) {
                const float2 v = normaliser(reinterpret_cast<const float2*>(a.ml) + slot * G + g, parts, G, tid & 63);
                if ((tid & 63) == 0) reinterpret_cast<float2*>(s_o)[g] = make_float2(v.x, share_of(v.y));
            }
            __syncthreads();
        }
#pragma unroll
        for (int g = 0; g < G; ++g) norm[g] = f.joins ? reinterpret_cast<const float2*>(s_o)[g] : reinterpret_cast<const float2*>(a.norm)[(int64_t)pair * G + g];
#pragma unroll
        for (int g = 0; g < G; ++g)
#pragma unroll
            for (int r = 0; r < kWeightRows; ++r) sum[r] += __builtin_amdgcn_exp2f(x[g][r] - norm[g].x) * norm[g].y;
        if (j0 + tid * kWeightRows < n) {
            if (whole) {
                *reinterpret_cast<f32x4_any*>(f.acc_out + at) = f32x4_any{sum[0], sum[1], sum[2], sum[3]};
            } else {
#pragma unroll
                for (int r = 0; r < kWeightRows; ++r)
                    if (j + r < n) f.acc_out[at + r] = sum[r];
            }
        }
    }
}

// ------------------------------------------------------------------------------------------------
// Eviction: which rows of a (layer, sequence, head) stay.  The cut is found digit by digit (11, 11, 10 bits) in the order-preserving images of the weights; every wave has a share of
// neighbouring rows, counts what it keeps of them and writes it behind the shares before, in order.  The images stay in registers (KEYS * 1024 rows a block), so that
// the weights are read once; the time goes into the five passes over them (32768 rows: 3 us to load, 5 for images and the first digit, 2 for each other one, 5 to count and write).
// Counters: two of each digit, taken by lane, since gathered weights crowd into few digits (half of the rows may have the same one) and lanes that
// add to one counter queue for it.
// SLICED: longer heads, by several blocks each in four launches.  Launch i < 3 counts the i-th digit, the last one writes; what lies between two launches are the counts of every
// slice, from which each block finds the next digit of the cut, and in the end its place in the list, by itself.  (131072 rows, 8 heads: 32 us; one block a head that reads them five times: 144.)
// ------------------------------------------------------------------------------------------------
struct EvictArgs {
    const float* acc;
    const int32_t *cu_tok, *n_tok;
    int32_t B, n_kv, T_total, max_n, keep, sink, recent;
    int32_t *keep_idx, *n_keep;
    int64_t row0;               // the first head of this launch
    // SLICED
    int32_t launch;
    uint32_t* counts;           // [row of this launch][slice][kEvictSliceWords]: counts of the three digits
};
constexpr int kEvictDigits = 2048, kEvictCopies = 2;

template <int THREADS, int KEYS, bool SLICED>
__global__ __launch_bounds__(THREADS) void cache_evict_kernel(EvictArgs a) {
    __shared__ __align__(16) uint32_t hist[kEvictDigits * kEvictCopies];
    constexpr int WAVES = THREADS / kWave, EACH = kEvictDigits / THREADS;      // digits a thread
    __shared__ uint32_t slot[WAVES], slot2[WAVES], found[2], s_above, s_equal;
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int64_t row = a.row0 + (SLICED ? blockIdx.y : blockIdx.x);           // (layer * B + b) * Hkv + h
    const int slice = SLICED ? blockIdx.x : 0;
    const int h = (int)(row % a.n_kv), b = (int)(row / a.n_kv % a.B);
    const int64_t layer = row / a.n_kv / a.B;
    int32_t first, rows;
    region(a.cu_tok, b, a.T_total, &first, &rows);
    const int32_t n = min(min(max(a.n_tok[row], 0), a.max_n), rows);
    int32_t* out = a.keep_idx + row * max(a.keep, 1);
    if (tid == 0 && slice == 0 && (!SLICED || a.launch == 3)) a.n_keep[row] = min(n, a.keep);
    constexpr int32_t kSlice = KEYS * THREADS;
    const int32_t begin = SLICED ? slice * kSlice : 0, end = SLICED ? min(n - begin, kSlice) + begin : n;
    if (begin >= end) return;
    if (n <= a.keep) {
        if (!SLICED || a.launch == 3)
            for (int32_t j = begin + tid; j < end; j += THREADS) out[j] = j;
        return;
    }
    if (a.keep == 0) return;
    const float* acc = a.acc + (layer * a.n_kv + h) * (int64_t)a.T_total + first;
    const int32_t share = (end - begin + THREADS - 1) / THREADS * 64, s0 = min(end, begin + w * share), s1 = min(end, s0 + share);
    const int copy = lane & (kEvictCopies - 1);
    // the images: rows that stay whatever they weigh above all others, lanes without a row below them (where NaN is, too)
    auto image = [&](int32_t j0 /* of the wave's first lane */, float f) -> uint32_t {
        uint32_t key = score_key(f);
        if (j0 < a.sink || j0 + 64 > min(n - a.recent, s1)) {
            const int32_t j = j0 + lane;
            key = j >= s1 ? 0u : j < a.sink || j >= n - a.recent ? 0xffffffffu : key;
        }
        return key;
    };
    uint32_t keys[KEYS];
#pragma unroll
    for (int i = 0; i < KEYS; ++i) keys[i] = __float_as_uint(acc[min(s0 + i * 64 + lane, n - 1)]);   // a load under a condition would wait for the one before
    for (int i = tid; i < kEvictDigits * kEvictCopies / 4; i += THREADS) *reinterpret_cast<uint4*>(hist + 4 * i) = make_uint4(0, 0, 0, 0);
    if (tid == 0) s_above = s_equal = 0;
    __syncthreads();
    // f(i) for the wave's groups of 64 rows
    auto each = [&](auto f) {
#pragma unroll
        for (int i = 0; i < KEYS; ++i)
            if (s0 + i * 64 < s1) f(i);
    };
    const int slices = (n + kSlice - 1) / kSlice;
    uint32_t* counts = SLICED ? a.counts + (int64_t)blockIdx.y * gridDim.x * kEvictSliceWords : nullptr;
    const uint32_t d0 = kEvictDigits - EACH * (tid + 1);      // the thread's digits, d0 the lowest of them: the first threads have the largest
    auto place = [](uint32_t d) { return d % EACH * THREADS + d / EACH; };          // counters of a thread's digits, so that the threads' lie side by side
    uint32_t need = (uint32_t)a.keep, prefix = 0;
    bool imaged = false;
    // SLICED, between the launches: in the first slice's words the cut so far and what is still needed (of each digit, two words), in every slice's the rows above it in slices before
    uint32_t *known = counts + 3 * kEvictDigits, *own = counts + (int64_t)slice * kEvictSliceWords + 3 * kEvictDigits + 4;
    if (SLICED && a.launch >= 2) {
        prefix = known[2 * (a.launch - 2)];
        need = known[2 * (a.launch - 2) + 1];
        if (tid == 0) s_above = *own;
    }
#pragma unroll
    for (int pass = 0; pass < 3; ++pass) {
        if (SLICED && pass < a.launch - 1) continue;
        const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0;
        const uint32_t digits = pass == 2 ? 1024u : 2048u;
        uint32_t c[EACH] = {}, before_slice[EACH] = {};       // counts of the thread's digits, and of them those in slices before
        if (SLICED && pass < a.launch) {
            constexpr int kAhead = 8;                         // slices on their way
            const uint32_t* p = counts + pass * kEvictDigits + d0;
            for (int s = 0; s < slices; s += kAhead) {
                uint32_t v[kAhead][EACH];
#pragma unroll
                for (int i = 0; i < kAhead; ++i)
#pragma unroll
                    for (int k = 0; k < EACH; ++k) v[i][k] = p[(int64_t)min(s + i, slices - 1) * kEvictSliceWords + k];
#pragma unroll
                for (int i = 0; i < kAhead; ++i)
#pragma unroll
                    for (int k = 0; k < EACH; ++k) {
                        c[k] += s + i < slices ? v[i][k] : 0u;
                        before_slice[k] += s + i < slices && s + i < slice ? v[i][k] : 0u;
                    }
            }
        } else {
            each([&](int i) {
                if (!imaged) keys[i] = image(s0 + i * 64, __uint_as_float(keys[i]));
                const uint32_t key = keys[i];
                const uint32_t d = (key >> shift) & (digits - 1);
                if (pass == 0 || (key >> (pass == 1 ? 21 : 10)) == prefix) atomicAdd(&hist[place(d) * kEvictCopies + copy], 1u);
            });
            imaged = true;
            __syncthreads();
#pragma unroll
            for (int k = 0; k < EACH; ++k) {
                uint2* p = reinterpret_cast<uint2*>(hist + place(d0 + k) * kEvictCopies);
                const uint2 v = *p;
                *p = make_uint2(0, 0);                        // for the next pass
                c[k] = v.x + v.y;
                if (SLICED) counts[(int64_t)slice * kEvictSliceWords + pass * kEvictDigits + d0 + k] = c[k];
            }
            if (SLICED) return;
        }
        // the digit in which the count, from the largest one down, reaches `need`
        uint32_t sum = 0;
#pragma unroll
        for (int k = 0; k < EACH; ++k) sum += c[k];
        const uint32_t upto_wave = wave_scan_u32(sum);
        if (lane == 63) slot[w] = upto_wave;
        __syncthreads();
        const uint32_t waves_to = wave_scan_u32(lane < WAVES ? slot[lane] : 0u);
        uint32_t before = upto_wave - sum + (w ? (uint32_t)__builtin_amdgcn_readlane((int)waves_to, w - 1) : 0u);
        if (before < need && need <= before + sum) {
#pragma unroll
            for (int k = EACH - 1; k >= 0; --k) {
                if (before < need && need <= before + c[k]) {
                    found[0] = d0 + k;
                    found[1] = need - before;
                }
                before += c[k];
            }
        }
        __syncthreads();
        if (SLICED) {
            const uint32_t digit = found[0];
            uint32_t mine = 0;
#pragma unroll
            for (int k = 0; k < EACH; ++k) {
                mine += d0 + k > digit ? before_slice[k] : 0u;
                if (pass == 2 && d0 + k == digit) s_equal = before_slice[k];
            }
            if (mine) atomicAdd(&s_above, mine);
        }
        prefix = (prefix << (pass == 2 ? 10 : 11)) | found[0];
        need = found[1];
        if (SLICED) {
            __syncthreads();
            if (tid == 0 && a.launch < 3) {
                *own = s_above;
                if (slice == 0) {
                    known[2 * pass] = prefix;
                    known[2 * pass + 1] = need;
                }
            }
        }
    }
    if (!imaged) each([&](int i) { keys[i] = image(s0 + i * 64, __uint_as_float(keys[i])); });
    // every row whose image is above `prefix`, and the first `need` of those equal to it: bits of a word a lane
    uint32_t kept_rows = 0, equal_rows = 0;
    each([&](int i) {
        kept_rows |= keys[i] > prefix ? 1u << i : 0u;
        equal_rows |= keys[i] == prefix ? 1u << i : 0u;
    });
    if (prefix == 0) equal_rows &= s0 + lane < s1 ? (2u << ((s1 - 1 - s0 - lane) >> 6)) - 1 : 0u;       // NaN: lanes without a row look the same
    const uint32_t above = __builtin_amdgcn_readlane((int)wave_scan_u32((uint32_t)__popc(kept_rows)), 63);
    const uint32_t equal = __builtin_amdgcn_readlane((int)wave_scan_u32((uint32_t)__popc(equal_rows)), 63);
    if (lane == 0) {
        slot[w] = above;
        slot2[w] = equal;
    }
    __syncthreads();
    uint32_t above_before = lane < w ? slot[lane] : 0u, eq_before = lane < w ? slot2[lane] : 0u;
#pragma unroll
    for (int m = 1; m < WAVES; m <<= 1) {
        above_before += (uint32_t)__shfl_xor((int)above_before, m);
        eq_before += (uint32_t)__shfl_xor((int)eq_before, m);
    }
    uint32_t at = __builtin_amdgcn_readfirstlane((int)above_before), eq = __builtin_amdgcn_readfirstlane((int)eq_before);
    if (SLICED) {
        at += s_above;
        eq += s_equal;
    }
    at += min(eq, need);
    if (eq < need && equal > 0) {
        if (eq + equal <= need) {
            kept_rows |= equal_rows;
        } else {                                              // the lowest ones that are still wanted
#pragma unroll 1
            for (int i = 0; i < KEYS && eq < need; ++i) {
                unsigned long long be = __ballot((equal_rows >> i) & 1);
                const uint32_t many = (uint32_t)__popcll(be);
                for (uint32_t k = need - eq; k < many && be; ++k) be &= ~(1ull << (63 - __builtin_clzll(be)));
                eq += many;
                kept_rows |= (uint32_t)(be >> lane & 1) << i;
            }
        }
    }
#pragma unroll
    for (int i = 0; i < KEYS; ++i) {
        const bool mine = (kept_rows >> i) & 1;
        const unsigned long long kept = __ballot(mine);
        if (mine) out[at + __builtin_amdgcn_mbcnt_hi((uint32_t)(kept >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)kept, 0u))] = s0 + i * 64 + lane;
        at += (uint32_t)__popcll(kept);
    }
}

// ------------------------------------------------------------------------------------------------
// Compaction: row j of a head becomes row keep_idx[j].  Bound by HBM: the kept rows in and out.  A block's new scale is the largest of the scales its rows come
// with; a code of a smaller one is rounded again (exactly, but for what leaves the normal range).
// A launch block takes `span` rows of one (layer, sequence, head, K or V) in ascending order, 128 at a time, eight lanes a row.  Where the outputs are the inputs `span` is all
// of them: a group's rows lie at or behind the place they go to, those of later groups behind everything written, and every group is read before it is
// written, so nothing is lost.  The rows of the next group and the list of the one behind are on their way while a group is written: a chain of three loads would
// otherwise be waited for every 16 KB.  128 heads, 8192 of 16384 rows: 106 us, 5.2 TB/s; in place 116.
// ------------------------------------------------------------------------------------------------
constexpr int kCompactRows = 128;

struct CompactArgs {
    const uint8_t *K, *V;
    const float *ks, *vs, *acc;
    uint8_t *K_out, *V_out;
    float *ks_out, *vs_out, *acc_out;
    const int32_t *cu_tok, *keep_idx, *n_keep;
    int32_t B, n_kv, T_total, n_scales, shift, keep, span;
    int64_t row0;               // the first head of this launch
};

__global__ __launch_bounds__(kBlockThreads) void cache_compact_kernel(CompactArgs a) {
    __shared__ __align__(16) float s_top[2][kBlockWaves];     // largest scale of a wave's 8 rows
    const int tid = threadIdx.x, w = tid >> 6, r = tid >> 3, part = (tid & 7) * 16;
    const int64_t row = a.row0 + blockIdx.x;
    const int h = (int)(row % a.n_kv), b = (int)(row / a.n_kv % a.B);
    const int64_t head = row / a.n_kv / a.B * a.n_kv + h;
    const bool is_v = blockIdx.y != 0;
    int32_t first, rows;
    region(a.cu_tok, b, a.T_total, &first, &rows);
    const int32_t m = min(min(max(a.n_keep[row], 0), a.keep), rows);
    const int32_t begin = (int32_t)min((int64_t)blockIdx.z * a.span, (int64_t)m), end = a.span < m - begin ? begin + a.span : m;
    if (begin >= end) return;
    const int32_t* idx = a.keep_idx + row * a.keep;
    const int64_t pool = head * a.T_total + first, slot0 = head * a.n_scales + (first >> a.shift) + b;
    const uint8_t* src = (is_v ? a.V : a.K) + pool * kHeadDim + part;
    uint8_t* dst = (is_v ? a.V_out : a.K_out) + pool * kHeadDim + part;
    const float* sc = (is_v ? a.vs : a.ks) + slot0;
    float* sc_out = (is_v ? a.vs_out : a.ks_out) + slot0;
    const float least = __uint_as_float(27u << 23);
    const int waves = (1 << a.shift) / 8, w0 = w & ~(waves - 1);      // waves of a scale block, the first of this one's
    const bool weigh = !is_v && a.acc && (tid & 7) == 0;

    // entry j of the list, -1 behind its end or where it is none of the rows; loads are unconditional (one under a condition waits for those before it)
    auto entry = [&](int32_t j) {
        const int32_t s = idx[min(j, end - 1)];
        return j < end && s >= 0 && s < rows ? s : -1;
    };
    struct Group { int32_t from; uint4 v; float scale, weight; };
    auto load = [&](Group& g, int32_t from) {
        const int32_t s = max(from, 0);
        g.from = from;
        g.v = ld_stream(src + (int64_t)s * kHeadDim);
        g.scale = sc[s >> a.shift];
        g.weight = weigh ? a.acc[pool + s] : 0.0f;
    };
    Group now, next;
    load(now, entry(begin + r));
    int32_t from = entry(begin + kCompactRows + r);
    int buf = 0;
    for (int32_t j0 = begin; j0 < end; j0 += kCompactRows, buf ^= 1) {
        const bool more = j0 + kCompactRows < end;
        if (more) {
            load(next, from);
            from = entry(j0 + 2 * kCompactRows + r);
        }
        const float mine = now.from >= 0 ? now.scale : least;
        float top = mine;
        top = fmaxf(top, __shfl_xor(top, 8));
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        if ((tid & 63) == 0) s_top[buf][w] = top;
        uint4 v = now.from >= 0 ? now.v : make_uint4(0, 0, 0, 0);
        float weight = now.from >= 0 ? now.weight : 0.0f;
        asm volatile("" : "+v"(v.x), "+v"(v.y), "+v"(v.z), "+v"(v.w), "+v"(weight));       // this group's loads have arrived before any of it is written
        __syncthreads();
        for (int i = 0; i < waves; ++i) top = fmaxf(top, s_top[buf][w0 + i]);
        if (mine != top) {
            const float f = mine / top;
            v = make_uint4(rescale(v.x, f), rescale(v.y, f), rescale(v.z, f), rescale(v.w, f));
        }
        const int32_t j = j0 + r;
        if (j < end) {
            st_stream(dst + (int64_t)j * kHeadDim, v);
            if (weigh) a.acc_out[pool + j] = weight;
            if ((tid & 7) == 0 && (j & ((1 << a.shift) - 1)) == 0) sc_out[j >> a.shift] = top;
        }
        now = next;
    }
}

inline int64_t round_up(int64_t n, int64_t m) { return (n + m - 1) / m * m; }
inline int log2_of(int32_t n) { return 31 - __builtin_clz((unsigned)n); }

// How skv_cache_attend deals its work, and where the parts of the workspace begin.
// Rows a block (of one a compute unit) above which a batch is dealt in equal shares: of 16 sequences of 1024 to 4096 rows, 8 heads (2048) take 25.2 us by chunks and 25.1 in shares, of 2048
// to 8192 rows 41 and 34; 64 sequences of up to 1024 rows (2048) 24 and 27, up to 16384 254 and 211.  With weights half as many: 16 x 4096 rows 37 by chunks and 31 in shares, 64 x
// 1024 rows 35 and 31, 16 x 2048 (1024) 21 and 26.  And rows a chunk of a batch that is dealt in those, at least.
// More pairs than kSharePairs take blocks of their own, which are then many and long enough (256 sequences of 1024 rows, 8 heads: 79 us by chunks, 101 in shares; 512 of up to 2048 198 and
// 246), unless the longest sequence would keep its block busy for longer than the chip takes for all rows (255 of 1024 rows and one of 131072, no weights: 925 and 159).
constexpr int kCacheShared = 2048, kCacheRagged = 512;
constexpr int kGridChunk = 1 << 24;        // rows of a chunk whose bytes a 32-bit offset reaches
bool skewed(const Ctx* c, int32_t max_n, int32_t T_total) { return (int64_t)max_n * c->n_cu > (int64_t)c->d.n_kv_heads * T_total; }
struct AttendLayout {
    int64_t logit_rows, ml, norm, ends, logits, bytes;
};
AttendLayout attend_layout(const Ctx* c, int64_t pairs, int64_t slots, int32_t max_n, bool weights) {
    AttendLayout w;
    const int64_t heads = pairs * c->G;
    w.logit_rows = round_up(max_n, kCacheTile);
    w.ml = round_up(slots * c->G * kHeadDim * 4, 256);
    w.norm = w.ml + round_up(slots * c->G * 8, 256);
    w.ends = w.norm + round_up(heads * 8, 256);
    w.logits = w.ends + round_up(pairs * 8, 256);
    w.bytes = w.logits + (weights ? round_up(heads * w.logit_rows * 4, 256) : 0);
    return w;
}
struct AttendPlan {
    int deal;
    int32_t chunk, splits, blocks;         // kShare: blocks of the launch
    AttendLayout work;
};
AttendPlan attend_plan(const Ctx* c, int32_t B, int32_t max_n, bool listed, bool weights, bool skewed) {
    AttendPlan p;
    const int64_t pairs = (int64_t)B * c->d.n_kv_heads, rows = pairs * max_n;
    // One block a compute unit: with more a block's beginning and end (queries, counts, joining its waves) are paid more often than its waits are hidden (8 heads x 16384 rows
    // 13.5 us with one, 13.8 with two, 14.9 with four; 64 lists of 2048 rows 13.9, 14.5, 17.6; 131072 rows 50, 50, 53).
    int64_t chunk = round_up((rows + c->n_cu - 1) / c->n_cu, kCacheStep);
    if (chunk < kCacheStep) chunk = kCacheStep;
    p.deal = listed ? kList : B > 1 && (pairs <= kSharePairs || (skewed && pairs <= kShareMost)) && chunk > (weights ? kCacheShared / 2 : kCacheShared) ? kShare : kGrid;
    if (p.deal == kGrid && B > 1 && chunk > kCacheRagged) {               // sequences of unlike lengths: several rounds of shorter blocks
        chunk = round_up((rows + 4 * (int64_t)c->n_cu - 1) / (4 * (int64_t)c->n_cu), kCacheStep);
        if (chunk < kCacheRagged) chunk = kCacheRagged;
    }
    if (chunk > (listed ? kListedChunk : kGridChunk)) chunk = listed ? kListedChunk : kGridChunk;
    p.chunk = (int32_t)chunk;
    p.splits = (int32_t)((max_n + chunk - 1) / chunk);
    if (p.splits < 1) p.splits = 1;
    p.blocks = cache_places(c->d.kv_dtype == SKV_BF16 ? 1 : 3, kShare, weights) * c->n_cu;
    p.work = attend_layout(c, pairs, p.deal == kShare ? p.blocks + pairs : p.splits > 1 ? pairs * p.splits : 0, max_n, weights);
    return p;
}

template <int PIECES, int DEAL, bool WEIGHTS>
hipError_t attend_launch(Ctx* c, const CacheAttendArgs& a, int32_t blocks) {
    size_t lds = (size_t)kCacheWaves * 8 * (2 + kHeadDim) * 4;                             // joining the waves
    if (DEAL == kList && (size_t)a.chunk * 12 > lds) lds = (size_t)a.chunk * 12;
    if (WEIGHTS && (size_t)kCacheWaves * a.G * kStageTiles * kCacheTile * 4 > lds) lds = (size_t)kCacheWaves * a.G * kStageTiles * kCacheTile * 4;
    if (DEAL == kShare) lds += (size_t)(a.pairs + 4) / 4 * 16;
    const dim3 grid = DEAL == kShare ? dim3(blocks) : dim3(a.splits, a.pairs);
    hipLaunchKernelGGL((cache_attend_kernel<PIECES, DEAL, WEIGHTS>), grid, dim3(kCacheWaves * kWave), lds, c->stream, a);
    return hipGetLastError();
}

// go(first head, heads) for all heads, by blocks of up to kBlockThreads threads each: a launch may have 2^32 - 1 threads in a dimension.
constexpr int64_t kHeadsAtOnce = 1 << 21;
template <typename Go>
hipError_t by_heads(int64_t heads, const Go& go) {
    for (int64_t row0 = 0; row0 < heads; row0 += kHeadsAtOnce) {
        go(row0, (unsigned)(heads - row0 < kHeadsAtOnce ? heads - row0 : kHeadsAtOnce));
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace

hipError_t launch_rotary(Ctx* c, int32_t n, const void* q, const void* k, const int32_t* pos, const double* inv_freq, int32_t rot, bool interleaved,
                         float mscale, void* q_out, void* k_out) {
    if (n == 0) return hipSuccess;
    const int EB = c->d.kv_dtype == SKV_BF16 ? 2 : 4;
    const bool vec = rot % 16 == 0;
    RotArgs a{(const char*)q, (const char*)k, (char*)q_out, (char*)k_out, pos, inv_freq, n, q ? c->d.n_q_heads : 0, k ? c->d.n_kv_heads : 0, rot / 2, 0, mscale};
    const int heads = a.n_q + a.n_k, rows = vec && EB == 2 ? 8 : 4;
    // Few tokens: as few heads a wave as one load takes, for a short chain.  Many: all heads of a token, so that its angles are formed once (32768 tokens of 40 bf16 heads: 110 us with
    // one wave a token, 115 with two, 136 with five).  Between: as many waves as the chip has places for, 32 a compute unit.
    int groups = (heads + rows - 1) / rows;
    const int64_t most = (32 * (int64_t)c->n_cu + n - 1) / n;
    if (groups > most) groups = (int)most;
    if (groups > 65535) groups = 65535;
    a.heads_per_wave = (int)round_up((heads + groups - 1) / groups, rows);
    groups = (heads + a.heads_per_wave - 1) / a.heads_per_wave;
    const int64_t blocks = ((int64_t)n + kRotWaves - 1) / kRotWaves;
    const dim3 grid((unsigned)(blocks < 1 << 22 ? blocks : 1 << 22), groups), block(kRotWaves * kWave);
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
                       cu_new, cu_tok, n_tok, n_new, max_new, T_total, n_scales, H};
    // pairs fastest: a token's heads lie side by side in the input, and the blocks that read them run at the same time
    const int span = block > kAppendSpan ? block : kAppendSpan;
    // a sequence's first scale block may hold up to block - 1 rows already
    const int64_t blocks = ((int64_t)max_new + block - 1 + span - 1) / span;
    const dim3 grid(B * H, (unsigned)(blocks < 65535 ? blocks : 65535), 2);
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

// Enough for every plan of up to B sequences and max_n rows, and no less for more of either: plans do not grow steadily (chunks are rounded up, shares need fewer parts than
// chunks, lists take chunks of their own), and a buffer made for a cache's largest length has to do for every length on the way there.  Parts: pairs * ceil(max_n / chunk) <=
// pairs + rows / chunk.  A chunk has 128 rows at least, and as many as n_cu (B > 1: 4 n_cu) blocks would need, unless that is cut to kListedChunk or more.  Shares take fewer than 4 n_cu
// blocks, and only where there are more than 1024 rows a compute unit.
int64_t cache_attend_work_bytes(const Ctx* c, int32_t B, int32_t max_n, bool weights) {
    const int64_t pairs = (int64_t)B * c->d.n_kv_heads, rows = pairs * max_n, dealt = (B > 1 ? 4 : 1) * (int64_t)c->n_cu;
    int64_t parts = rows / kCacheStep < dealt ? rows / kCacheStep : dealt;
    if (rows / kListedChunk > parts) parts = rows / kListedChunk;
    return attend_layout(c, pairs, pairs + parts, max_n, weights).bytes;
}

hipError_t launch_cache_attend(Ctx* c, int32_t layer, int32_t B, const void* q, const void* K, const void* V, const float* ks, const float* vs, int32_t T_total,
                               int32_t block, const int32_t* cu_tok, const int32_t* n_tok, const int32_t* tok_idx, int32_t max_n, float* out, float* lse,
                               const float* acc, float* acc_out, float decay, void* work) {
    const bool listed = tok_idx != nullptr && max_n > 0, weights = acc_out != nullptr, wide = c->d.kv_dtype != SKV_BF16;
    const AttendPlan p = attend_plan(c, B, max_n, listed, weights, skewed(c, max_n, T_total));
    const int H = c->d.n_kv_heads, n_scales = T_total / block + B, pairs = B * H;
    const int64_t pool = (int64_t)layer * H * T_total, sc = (int64_t)layer * H * n_scales;
    const bool share = p.deal == kShare, joined = share || p.splits > kJoinInside;
    char* ws = static_cast<char*>(work);
    const CacheAttendArgs a{(const char*)q, (const uint8_t*)K + pool * kHeadDim, (const uint8_t*)V + pool * kHeadDim, ks + sc, vs + sc, cu_tok, n_tok, tok_idx,
                            max_n, T_total, n_scales, log2_of(block), H, c->G, pairs, p.chunk, p.splits, p.work.logit_rows, out, lse, (float*)ws,
                            (float*)(ws + p.work.ml), weights ? (float*)(ws + p.work.norm) : nullptr, (float*)(ws + p.work.logits), (int32_t*)(ws + p.work.ends),
                            !joined && p.splits > 1 ? c->att_counter : nullptr};
    hipError_t e;
    if (listed) e = wide ? attend_launch<3, kList, false>(c, a, 0) : attend_launch<1, kList, false>(c, a, 0);
    else if (share && weights) e = wide ? attend_launch<3, kShare, true>(c, a, p.blocks) : attend_launch<1, kShare, true>(c, a, p.blocks);
    else if (share) e = wide ? attend_launch<3, kShare, false>(c, a, p.blocks) : attend_launch<1, kShare, false>(c, a, p.blocks);
    else if (weights) e = wide ? attend_launch<3, kGrid, true>(c, a, 0) : attend_launch<1, kGrid, true>(c, a, 0);
    else e = wide ? attend_launch<3, kGrid, false>(c, a, 0) : attend_launch<1, kGrid, false>(c, a, 0);
    if (e != hipSuccess) return e;
    const bool weigh = weights && max_n > 0;
    if (!joined && !weigh) return hipSuccess;
    const int per = kFinishThreads * kWeightRows;
    const FinishArgs f{listed ? 1 : 0, share ? 1 : 0, joined ? c->G : 0, acc ? acc + pool : nullptr, weigh ? acc_out + pool : nullptr, decay};
    const dim3 grid(f.joins + (weigh ? (max_n + per - 1) / per : 0), pairs), threads(kFinishThreads);
    switch (weigh ? c->G : 0) {
        case 0: hipLaunchKernelGGL(cache_finish_kernel<0>, grid, threads, 0, c->stream, a, f); break;
        case 1: hipLaunchKernelGGL(cache_finish_kernel<1>, grid, threads, 0, c->stream, a, f); break;
        case 2: hipLaunchKernelGGL(cache_finish_kernel<2>, grid, threads, 0, c->stream, a, f); break;
        case 4: hipLaunchKernelGGL(cache_finish_kernel<4>, grid, threads, 0, c->stream, a, f); break;
        default: hipLaunchKernelGGL(cache_finish_kernel<8>, grid, threads, 0, c->stream, a, f); break;
    }
    return hipGetLastError();
}

hipError_t launch_cache_evict(Ctx* c, int32_t B, const float* acc, int32_t T_total, const int32_t* cu_tok, const int32_t* n_tok, int32_t max_n, int32_t keep,
                              int32_t sink, int32_t recent, int32_t* keep_idx, int32_t* n_keep) {
    EvictArgs a{acc, cu_tok, n_tok, B, c->d.n_kv_heads, T_total, max_n, keep, sink, recent, keep_idx, n_keep, 0, 0, c->evict_counts};
    const int64_t heads = (int64_t)c->d.n_layers * B * c->d.n_kv_heads;
    // as few threads a head as hold its images with eight each, then more images (a load of a row that is none costs as much as one of a row)
    auto whole = [&](auto threads, auto keys) {
        constexpr int N = decltype(threads)::value, K = decltype(keys)::value;
        return by_heads(heads, [&](int64_t row0, unsigned here) {
            a.row0 = row0;
            hipLaunchKernelGGL((cache_evict_kernel<N, K, false>), dim3(here), dim3(N), 0, c->stream, a);
        });
    };
    using std::integral_constant;
    constexpr integral_constant<int, 8> k8{};
    if (max_n <= 8 * 256) return whole(integral_constant<int, 256>{}, k8);
    if (max_n <= 8 * 512) return whole(integral_constant<int, 512>{}, k8);
    if (max_n <= 8 * 1024) return whole(integral_constant<int, 1024>{}, k8);
    if (max_n <= 16 * 1024) return whole(integral_constant<int, 1024>{}, integral_constant<int, 16>{});
    if (max_n <= kEvictSlice) return whole(integral_constant<int, 1024>{}, integral_constant<int, kEvictSlice / 1024>{});
    // short slices where all of them have room and a place on the chip at once, long ones otherwise, as many heads at a time as there is room for
    auto go = [&](auto keys) {
        constexpr int K = decltype(keys)::value;
        const int slices = (int)(((int64_t)max_n + K * kBlockThreads - 1) / (K * kBlockThreads)), at_once = evict_slices(c->d) / slices;
        for (a.row0 = 0; a.row0 < heads; a.row0 += at_once) {
            const unsigned here = (unsigned)(heads - a.row0 < at_once ? heads - a.row0 : at_once);
            for (a.launch = 0; a.launch < 4; ++a.launch) {
                hipLaunchKernelGGL((cache_evict_kernel<kBlockThreads, K, true>), dim3(slices, here), dim3(kBlockThreads), 0, c->stream, a);
                const hipError_t e = hipGetLastError();
                if (e != hipSuccess) return e;
            }
        }
        return hipSuccess;
    };
    const int64_t few = heads * (((int64_t)max_n + 8 * kBlockThreads - 1) / (8 * kBlockThreads));
    return few <= evict_slices(c->d) && few <= c->n_cu ? go(k8) : go(integral_constant<int, kEvictSlice / kBlockThreads>{});
}

hipError_t launch_cache_compact(Ctx* c, int32_t B, const void* K, const void* V, const float* ks, const float* vs, const float* acc, int32_t T_total, int32_t block,
                                const int32_t* cu_tok, const int32_t* keep_idx, int32_t keep, const int32_t* n_keep, void* K_out, void* V_out, float* ks_out,
                                float* vs_out, float* acc_out) {
    if (keep == 0) return hipSuccess;
    const int64_t heads = (int64_t)c->d.n_layers * B * c->d.n_kv_heads;
    // other outputs: rows cut over four blocks a compute unit, two of them at once, in groups of 128 (8 layers x 8 heads, 2048 of 4096 rows: 18.9 us with one, 17.7 with two, 18.5 with
    // four, 21.7 with eight; 16 x 8 x 8192: 117, 108, 107, 105)
    const int64_t most = keep < T_total ? keep : T_total;     // rows of a list that can be used, however long it is
    int64_t span = most;
    if (K != K_out) {
        const int64_t cuts = (4 * (int64_t)c->n_cu + 2 * heads - 1) / (2 * heads);
        span = round_up((most + cuts - 1) / cuts, kCompactRows);
    }
    const unsigned spans = (unsigned)((most + span - 1) / span);
    if (span > most) span = most;                             // in 32 bits again
    CompactArgs a{(const uint8_t*)K, (const uint8_t*)V, ks, vs, acc, (uint8_t*)K_out, (uint8_t*)V_out, ks_out, vs_out, acc_out, cu_tok, keep_idx, n_keep,
                  B, c->d.n_kv_heads, T_total, T_total / block + B, log2_of(block), keep, (int32_t)span, 0};
    return by_heads(heads, [&](int64_t row0, unsigned here) {
        a.row0 = row0;
        hipLaunchKernelGGL(cache_compact_kernel, dim3(here, 2, spans), dim3(kBlockThreads), 0, c->stream, a);
    });
}

}  // namespace skv
