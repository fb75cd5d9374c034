// Attention of one new token per sequence over a paged cache on gfx950.
//
// A work-group takes up to 16 query heads that share a head of keys, and a span of a
// sequence's positions; its waves take 64 positions at a time.  Scores are products
// of 16 keys and 16 queries, S^T = K Q^T, in which a lane's accumulators are 4 keys
// 4 (lane / 16) .. of query lane % 16: maxima and sums are taken there, and 8 of
// them from two tiles of keys are at once the operand of the second product, O^T =
// V^T P^T, whose depth is those 32 keys.  Products are 16 wide whatever the number of
// heads: matrix instructions are not what bounds it.  8-bit elements become bf16
// numbers, which they are, by an instruction for two; a key's factor 2^e multiplies
// its score, a value's its probability.
//
// Bound by how long reads take: pages are looked up and read a round ahead, with 1.1 to
// 1.4 waves a SIMD that wait 56 to 63 % of their time.  64 x 1600 tokens of 4 heads of
// 64 bf16 reals: 23.4 us, 4.5 TB/s (read when they were needed: 31); 4 sequences of up
// to 65536 of 2 heads in 8 bits: 14 us and 4 for the join.  One lane to a key and
// head, on the vector units, took 22207 us for the latter.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "cache_tile.h"

namespace quan {
namespace {

constexpr int kWaves = 8, kThreads = 64 * kWaves;
constexpr int kChunk = 64;             // positions that a wave takes at a time
constexpr int kRound = kWaves * kChunk;  // and a work-group
constexpr int kQueries = 16;           // of a work-group
constexpr int kBiasLds = 8192;         // biases held in LDS

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef unsigned u32x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ f32x4 mma16(const bf16x8 &a, const bf16x8 &b, const f32x4 &c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

// 8 elements in 8 bits (two dwords) as bf16.
__device__ __forceinline__ bf16x8 widen(unsigned lo, unsigned hi)
{
    const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, false);
    const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, true);
    const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, false);
    const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, true);
    return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// A value in the three lanes l ^ 16, l ^ 32, l ^ 48 too.
__device__ __forceinline__ float quarters_max(float x)
{
    const auto w = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return half_max(fmaxf(__uint_as_float(w[0]), __uint_as_float(w[1])));
}
__device__ __forceinline__ float quarters_sum(float x)
{
    const auto w = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return half_sum(__uint_as_float(w[0]) + __uint_as_float(w[1]));
}

// fp32 numbers as bf16 parts, each what the ones before leave.
template <int PARTS> __device__ __forceinline__ void split(f32x8 v, bf16x8 (&p)[PARTS])
{
#pragma unroll
    for (int i = 0; i < PARTS; ++i) {
        p[i] = __builtin_convertvector(v, bf16x8);
        if (i + 1 < PARTS)
            v -= __builtin_convertvector(p[i], f32x8);
    }
}

struct Token {
    CacheAttention a;
    // of heads (kv_heads x group_blocks); spans at most; partial results [span][head][D],
    // [span][head][2], D the head's reals rounded up to 32, 64 or 128; or NULL: a
    // work-group takes all of a sequence
    int units, group_blocks, group, spans;
    float *part, *part_stats;
};

// How the positions of all sequences are dealt out: spans of `len`, a whole number
// of rounds, so many that they are at most `spans`.
__device__ __forceinline__ int length_of(const CacheAttention &a, int seq)
{
    return a.kv_len != nullptr ? min(max(a.kv_len[seq], 0), a.cache.capacity()) : a.cache.capacity();
}
__device__ __forceinline__ int span_length(const Token &t)
{
    const int lane = threadIdx.x & 63;
    int64_t total = 0;
    for (int i = lane; i < t.a.n; i += 64)
        total += length_of(t.a, i);
#pragma unroll
    for (int l = 1; l < 64; l *= 2)
        total += __shfl_xor(total, l, 64);
    const int64_t per = int64_t(t.spans - t.a.n) * kRound;  // (> 0)
    // (a sequence's last span is at least one position: no more than n beyond total / len)
    return int(max(int64_t(1), (total + per - 1) / per)) * kRound;
}
// First span of each of 64 sequences from i0 on (a lane each), and of the next 64.
struct Spans {
    int first, count, next;
};
__device__ __forceinline__ Spans spans_from(const Token &t, int i0, int first, int len)
{
    const int lane = threadIdx.x & 63, seq = i0 + lane;
    const int count = seq < t.a.n ? (length_of(t.a, seq) + len - 1) / len : 0;
    int upto = count;
#pragma unroll
    for (int l = 1; l < 64; l *= 2) {
        const int v = __shfl_up(upto, l, 64);
        upto += lane >= l ? v : 0;
    }
    return {first + upto - count, count, first + __shfl(upto, 63, 64)};
}
struct Share {
    int seq, begin, end;  // positions; seq < 0: none
};
__device__ __forceinline__ Share share_of(const Token &t, int span)
{
    if (t.part == nullptr)
        return {span, 0, length_of(t.a, span)};
    const int len = span_length(t), lane = threadIdx.x & 63;
    int first = 0;
    for (int i0 = 0; i0 < t.a.n; i0 += 64) {
        const Spans s = spans_from(t, i0, first, len);
        const auto here = __ballot(span >= s.first && span < s.first + s.count);
        if (here) {
            const int l = __builtin_ctzll(here), seq = i0 + l;
            const int begin = (span - __shfl(s.first, l, 64)) * len;
            return {seq, begin, min(begin + len, length_of(t.a, seq))};
        }
        first = s.next;
    }
    return {-1, 0, 0};
}

// A real of a head's output from its sum over the keys.
template <typename T> __device__ __forceinline__ void finish(const CacheAttention &a, int seq, int head, int real, float v, float sum)
{
    const int dq = a.cache.dq;
    if (real >= 4 * dq)
        return;
    v *= sum > 0.0f || sum != sum ? 1.0f / sum : 0.0f;
    T *to = static_cast<T *>(const_cast<void *>(a.out.data)) + seq * a.out.s_n + int64_t(head) * dq;
    to[(real / dq) * a.out.s_p + real % dq] = T(v);
}

// What a form's chunk of 64 positions takes: bytes of a row that a lane reads of
// keys at a time (16, of narrow 8-bit rows 8) and of values (its sixteenth).
template <CacheForm F, int D> struct Rows {
    static constexpr int kBytes = D * cache_elem_size(F);
    static constexpr int kLoad = kBytes < 64 ? 8 : 16, kLoads = kBytes / (4 * kLoad);  // a key's four lanes
    static constexpr int kElems = kLoad / cache_elem_size(F);                          // of a load
    static constexpr int kValue = kBytes / 16;                                         // bytes of a value's row per lane
    // 16-key tiles at a time, so that what is read fits the registers
    static constexpr int kTiles = kBytes > 256 ? 2 : 4;
};
template <int BYTES> struct Word;
template <> struct Word<2> { typedef unsigned short type; };
template <> struct Word<4> { typedef unsigned type; };
template <> struct Word<8> { typedef unsigned type __attribute__((ext_vector_type(2))); };
template <> struct Word<16> { typedef unsigned type __attribute__((ext_vector_type(4))); };
template <> struct Word<32> { typedef unsigned type __attribute__((ext_vector_type(8))); };

// BYTES of a row from `at` on; what is behind its end is any of its own.
template <int BYTES> __device__ __forceinline__ typename Word<BYTES>::type load_value(const unsigned char *row, int at, int end)
{
    typedef typename Word<BYTES>::type word;
    if constexpr (BYTES == 32) {
        typedef typename Word<16>::type half;
        const half a = *reinterpret_cast<const half *>(row + (at < end ? at : 0));
        const half b = *reinterpret_cast<const half *>(row + (at + 16 < end ? at + 16 : 0));
        return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
    } else {
        // (a row is whole 16 bytes)
        return *reinterpret_cast<const word *>(row + (at < end ? at : 0));
    }
}

// BIAS 0: none, 1: the work-group's rows of the table lie in LDS, 2: in memory.
template <typename T, CacheForm F, int D, int BIAS>
__global__ void __launch_bounds__(kThreads, sizeof(T) == 2 && D < 128 ? 4 : 2) cache_attention_kernel(Token t)
{
    typedef Rows<F, D> R;
    constexpr bool E4M3 = F == CacheForm::E4M3, FP32 = F == CacheForm::F32;
    constexpr int PQ = FP32 ? 1 : sizeof(T) == 2 ? 1 : 3, PP = sizeof(T) == 2 ? 2 : 3;  // bf16 parts of q and P
    constexpr int kMine = D / 16;  // reals of a value's row per lane
    constexpr int TILES = R::kTiles, SUB = TILES * 16;
    extern __shared__ __attribute__((aligned(16))) unsigned char lds_raw[];

    const CacheAttention &a = t.a;
    const Cache &c = a.cache;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, i = lane & 15, q = lane >> 4;
    const int unit = blockIdx.x % t.units, span = blockIdx.x / t.units;
    const int kv_head = unit / t.group_blocks, g0 = unit % t.group_blocks * kQueries;
    const int head0 = kv_head * t.group + g0, heads = min(kQueries, t.group - g0);
    const Share share = share_of(t, span);
    if (share.seq < 0)
        return;
    const int seq = share.seq;

    int *rows = reinterpret_cast<int *>(lds_raw) + wave * 4 * kChunk;
    float *key_by = reinterpret_cast<float *>(rows + kChunk), *value_by = key_by + kChunk;
    int *buckets = rows + 3 * kChunk;
    float *bias = reinterpret_cast<float *>(lds_raw) + kWaves * 4 * kChunk;  // [heads][ny nx]
    const int nb = a.bias.ny * a.bias.nx;
    const float *table = a.bias.table + int64_t(head0) * nb;
    if (BIAS == 1) {
        for (int e = threadIdx.x; e < heads * nb; e += kThreads)
            bias[e] = in_log2(table[e]);
        __syncthreads();
    }
    int pos_y = 0, pos_x = 0;
    if (BIAS != 0 && a.pos != nullptr) {
        pos_y = query_pos(a.pos[2 * seq]);
        pos_x = query_pos(a.pos[2 * seq + 1]);
    }

    // the query that the lane holds, as the products' operand: of load l its elements
    // are the reals (4 l + q) kElems ..
    constexpr int kReals = R::kLoads * R::kElems;
    bf16x8 qf[FP32 ? 1 : PQ][FP32 ? 1 : kReals / 8];
    float qs[FP32 ? kReals : 1];
    {
        const T *row = static_cast<const T *>(a.q.data) + seq * a.q.s_n + int64_t(head0 + min(i, heads - 1)) * c.dq;
        const bool whole = a.q.vec;  // (and dq a multiple of 8)
        constexpr int kAt = R::kElems < 8 ? R::kElems : 8;
#pragma unroll
        for (int l = 0; l < R::kLoads; ++l)
#pragma unroll
            for (int e0 = 0; e0 < R::kElems; e0 += kAt) {
                const int real = (4 * l + q) * R::kElems + e0;
                f32x8 v = 0.0f;
                if (kAt == 8 && whole) {
                    const bool here = real < 4 * c.dq;
                    const int comp = here ? real / c.dq : 0;
                    v = to_f32(load_chunk<T>(row + comp * a.q.s_p + (here ? real - comp * c.dq : 0), here ? 8 : 0, true));
                } else {
#pragma unroll
                    for (int e = 0; e < kAt; ++e) {
                        const bool here = real + e < 4 * c.dq;
                        const int comp = here ? (real + e) / c.dq : 0;
                        const float x = float(row[comp * a.q.s_p + (here ? real + e - comp * c.dq : 0)]);
                        v[e] = here ? x : 0.0f;
                    }
                }
                if constexpr (FP32) {
#pragma unroll
                    for (int e = 0; e < kAt; ++e)
                        qs[l * R::kElems + e0 + e] = v[e];
                } else {
                    bf16x8 p[PQ];
                    split<PQ>(v, p);
#pragma unroll
                    for (int s = 0; s < PQ; ++s)
                        qf[s][(l * R::kElems + e0) / 8] = p[s];
                }
            }
    }

    f32x4 o[kMine];
#pragma unroll
    for (int m = 0; m < kMine; ++m)
        o[m] = 0.0f;
    float top = -INFINITY, sum = 0.0f;
    const float scale = a.scale * kLog2e;
    const int page_rows = c.page_tokens;
    const bool partial = c.row_bytes != R::kBytes;  // the rows are shorter than D reals
    const int chunks = c.row_bytes / 16;

    // a position's page is read a round ahead, a position's factors with its rows
    const int32_t *pages = c.table + int64_t(seq) * c.table_pages;
    auto page_of = [&](int j) { return j < share.end ? pages[fast_div(j, c.by_page)] : -1; };
    int page = page_of(share.begin + wave * kChunk + lane);
    for (int j0 = share.begin + wave * kChunk; j0 < share.end; j0 += kRound) {
        // the chunk's rows, a position per lane
        const int j = j0 + lane;
        const bool here = page >= 0 && page < c.pages;
        const int row = here ? (page * c.heads + kv_head) * page_rows + j - fast_div(j, c.by_page) * page_rows : 0;
        const auto ok = __ballot(here);
        page = page_of(j + kRound);
        rows[lane] = row;
        unsigned key_exp = 0, value_exp = 0;
        if (E4M3) {
            key_exp = c.key_exp[row];
            value_exp = c.value_exp[row];
        }
        if (BIAS != 0) {
            const int y = fast_div(j, a.by_width), x = j - y * a.width;
            const int dy = min(max(y - pos_y, -a.bias.ry), a.bias.ry), dx = min(max(x - pos_x, -a.bias.rx), a.bias.rx);
            const int iy = a.bias.by != nullptr ? min(max(a.bias.by[dy + a.bias.ry], 0), a.bias.ny - 1) : 0;
            const int ix = a.bias.bx != nullptr ? min(max(a.bias.bx[dx + a.bias.rx], 0), a.bias.nx - 1) : 0;
            buckets[lane] = iy * a.bias.nx + ix;
        }
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");

#pragma unroll
        for (int sub = 0; sub < kChunk; sub += SUB) {
            if (sub > 0 && j0 + sub >= share.end)
                break;
            // keys: lane (i, q) reads its loads of key i of each tile
            typedef typename Word<R::kLoad>::type key_word;
            key_word kw[TILES][R::kLoads];
#pragma unroll
            for (int tile = 0; tile < TILES; ++tile) {
                const unsigned char *p = c.keys + int64_t(rows[sub + 16 * tile + i]) * c.row_bytes;
#pragma unroll
                for (int l = 0; l < R::kLoads; ++l) {
                    int at = (4 * l + q) * R::kLoad;
                    if (partial && at >= c.row_bytes)
                        at = 0;
                    kw[tile][l] = *reinterpret_cast<const key_word *>(p + at);
                }
            }
            // values: its sixteenth of 8 rows of each pair of tiles
            typedef typename Word<R::kValue>::type value_word;
            value_word vw[TILES / 2][8];
#pragma unroll
            for (int u = 0; u < TILES / 2; ++u)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const i32x4 r4 = *reinterpret_cast<const i32x4 *>(rows + sub + 32 * u + 16 * h + 4 * q);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        vw[u][4 * h + e] = load_value<R::kValue>(c.values + int64_t(r4[e]) * c.row_bytes, i * R::kValue,
                                                                partial ? c.row_bytes : R::kBytes);
                    }
                }
            if (E4M3 && sub == 0) {
                key_by[lane] = here ? scale * factor_of(key_exp) : 0.0f;
                value_by[lane] = here ? factor_of(value_exp) : 0.0f;
                __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
                __builtin_amdgcn_wave_barrier();
                __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
            }
            if (partial && !E4M3) {
                // (an 8-bit row that is not finite is so as a whole)
#pragma unroll
                for (int tile = 0; tile < TILES; ++tile)
#pragma unroll
                    for (int l = 0; l < R::kLoads; ++l)
                        if (4 * l + q >= chunks)
                            kw[tile][l] = key_word{};
            }
            f32x4 s[TILES];
#pragma unroll
            for (int tile = 0; tile < TILES; ++tile) {
                s[tile] = 0.0f;
#pragma unroll
                for (int l = 0; l < R::kLoads; ++l) {
                    if constexpr (FP32) {
                        const f32x4 k = __builtin_bit_cast(f32x4, kw[tile][l]);
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            s[tile] = __builtin_amdgcn_mfma_f32_16x16x4f32(k[e], qs[4 * l + e], s[tile], 0, 0, 0);
                    } else {
                        constexpr int kFrags = R::kElems / 8;
#pragma unroll
                        for (int f = 0; f < kFrags; ++f) {
                            bf16x8 k;
                            if constexpr (E4M3)
                                k = widen(kw[tile][l][2 * f], kw[tile][l][2 * f + 1]);
                            else
                                k = __builtin_bit_cast(bf16x8, kw[tile][l]);
#pragma unroll
                            for (int p = PQ - 1; p >= 0; --p)  // (the least first)
                                s[tile] = mma16(k, qf[p][l * kFrags + f], s[tile]);
                        }
                    }
                }
                if (E4M3)
                    s[tile] *= *reinterpret_cast<const f32x4 *>(key_by + sub + 16 * tile + 4 * q);
                else
                    s[tile] *= scale;
                if (BIAS != 0) {
                    const i32x4 b = *reinterpret_cast<const i32x4 *>(buckets + sub + 16 * tile + 4 * q);
                    const int64_t of = int64_t(min(i, heads - 1)) * nb;
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        s[tile][e] += BIAS == 1 ? bias[int(of) + b[e]] : in_log2(table[of + b[e]]);
                }
            }
            if (~ok != 0) {
#pragma unroll
                for (int tile = 0; tile < TILES; ++tile) {
                    const unsigned mine = unsigned(ok >> (sub + 16 * tile + 4 * q));
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        s[tile][e] = mine >> e & 1 ? s[tile][e] : -INFINITY;
                        vw[tile / 2][4 * (tile % 2) + e] = mine >> e & 1 ? vw[tile / 2][4 * (tile % 2) + e] : value_word{};
                    }
                }
            }
            float most = s[0][0];
#pragma unroll
            for (int tile = 0; tile < TILES; ++tile)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    most = fmaxf(most, s[tile][e]);
            const float now = fmaxf(top, quarters_max(most)), base = now == -INFINITY ? 0.0f : now;
            const float back = exp2_fast(top - base);
            top = now;
            sum *= back;
#pragma unroll
            for (int m = 0; m < kMine; ++m)
                o[m] *= back;
#pragma unroll
            for (int u = 0; u < TILES / 2; ++u) {
                f32x8 p;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    p[e] = exp2_fast(s[2 * u + e / 4][e % 4] - base);
                    sum += p[e];
                }
                if (E4M3) {
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const f32x4 by = *reinterpret_cast<const f32x4 *>(value_by + sub + 32 * u + 16 * h + 4 * q);
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            p[4 * h + e] *= by[e];
                    }
                }
                if constexpr (FP32) {
#pragma unroll
                    for (int e = 0; e < 8; ++e)
#pragma unroll
                        for (int m = 0; m < kMine; ++m) {
                            const float v = __uint_as_float(vw[u][e][m]);
                            o[m] = __builtin_amdgcn_mfma_f32_16x16x4f32(v, p[e], o[m], 0, 0, 0);
                        }
                } else {
                    bf16x8 pf[PP];
                    if constexpr (F == CacheForm::BF16) {  // (whose values may be infinite)
                        pf[0] = cut(p);
                        pf[1] = __builtin_convertvector(p, bf16x8);
                    } else {
                        split<PP>(p, pf);
                    }
#pragma unroll
                    for (int m = 0; m < kMine; ++m) {
                        // element m of the 8 rows
                        bf16x8 v;
                        if constexpr (E4M3) {
                            unsigned w[8];
#pragma unroll
                            for (int e = 0; e < 8; ++e) {
                                if constexpr (R::kValue <= 4)
                                    w[e] = vw[u][e];
                                else
                                    w[e] = vw[u][e][m / 4];
                            }
                            const unsigned b = m % 4;
                            const unsigned pick = (4 + b) << 8 | b;  // byte b of two words: of the second, the first
                            const unsigned w01 = __builtin_amdgcn_perm(w[1], w[0], pick), w23 = __builtin_amdgcn_perm(w[3], w[2], pick);
                            const unsigned w45 = __builtin_amdgcn_perm(w[5], w[4], pick), w67 = __builtin_amdgcn_perm(w[7], w[6], pick);
                            v = widen(__builtin_amdgcn_perm(w23, w01, 0x05040100), __builtin_amdgcn_perm(w67, w45, 0x05040100));
                        } else {
                            u32x2 w[4];
                            unsigned d[4];
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                if constexpr (R::kValue <= 4)
                                    w[e] = u32x2{unsigned(vw[u][2 * e]), unsigned(vw[u][2 * e + 1])};
                                else
                                    w[e] = u32x2{unsigned(vw[u][2 * e][m / 2]), unsigned(vw[u][2 * e + 1][m / 2])};
                                d[e] = __builtin_amdgcn_perm(w[e][1], w[e][0], m % 2 ? 0x07060302 : 0x05040100);
                            }
                            typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
                            v = __builtin_bit_cast(bf16x8, u32x4{d[0], d[1], d[2], d[3]});
                        }
#pragma unroll
                        for (int p2 = PP - 1; p2 >= 0; --p2)
                            o[m] = mma16(v, pf[p2], o[m]);
                    }
                }
            }
        }
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();  // the chunk's rows have been read
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    }
    sum = quarters_sum(sum);

    // the waves' results joined: o[m][r] is real (4 q + r) D / 16 + m of query i
    __syncthreads();
    float *acc = reinterpret_cast<float *>(lds_raw), *stats = acc + kWaves * heads * D;
    if (i < heads) {
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int m = 0; m < kMine; ++m)
                acc[(wave * heads + i) * D + (4 * q + r) * kMine + m] = o[m][r];
        if (q == 0) {
            stats[2 * (wave * heads + i)] = top;
            stats[2 * (wave * heads + i) + 1] = sum;
        }
    }
    __syncthreads();
    for (int e = threadIdx.x; e < heads * D; e += kThreads) {
        const int head = e / D, real = e % D;
        float m = -INFINITY, total = 0.0f, value = 0.0f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w)
            m = fmaxf(m, stats[2 * (w * heads + head)]);
        const float base = m == -INFINITY ? 0.0f : m;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            const float by = exp2_fast(stats[2 * (w * heads + head)] - base);
            total = fmaf(by, stats[2 * (w * heads + head) + 1], total);
            value = fmaf(by, acc[(w * heads + head) * D + real], value);
        }
        if (t.part == nullptr) {
            finish<T>(a, seq, head0 + head, real, value, total);
            continue;
        }
        const int64_t at = int64_t(span) * a.heads + head0 + head;
        t.part[at * D + real] = value;
        if (real == 0) {
            t.part_stats[2 * at] = m;
            t.part_stats[2 * at + 1] = total;
        }
    }
}

// The spans' partial results joined: a work-group per sequence and head, its lanes in
// sets of D / 4 (4 reals each) that take the spans in turn and meet in LDS.
template <typename T, int D> __global__ void __launch_bounds__(256) cache_join_kernel(Token t)
{
    constexpr int kLanes = D / 4, kSets = 256 / kLanes;
    __shared__ float acc[kSets * D], stats[2 * kSets];
    const CacheAttention &a = t.a;
    const int seq = blockIdx.x / a.heads, head = blockIdx.x % a.heads;
    const int len = span_length(t);
    int first = 0, count = 0;
    for (int i0 = 0, next = 0; i0 <= seq; i0 += 64) {
        const Spans s = spans_from(t, i0, next, len);
        first = __shfl(s.first, seq & 63, 64);
        count = __shfl(s.count, seq & 63, 64);
        next = s.next;
    }
    const int set = threadIdx.x / kLanes, d = 4 * (threadIdx.x % kLanes);
    float top = -INFINITY, sum = 0.0f;
    f32x4 o = 0.0f;
#pragma unroll 4
    for (int s = set; s < count; s += kSets) {
        const int64_t at = int64_t(first + s) * a.heads + head;
        const float m = t.part_stats[2 * at], l = t.part_stats[2 * at + 1];
        const f32x4 v = *reinterpret_cast<const f32x4 *>(t.part + at * D + d);
        const float now = fmaxf(top, m), base = now == -INFINITY ? 0.0f : now;
        const float back = exp2_fast(top - base), w = exp2_fast(m - base);
        top = now;
        sum = sum * back + l * w;
        o = o * back + v * w;
    }
    *reinterpret_cast<f32x4 *>(acc + set * D + d) = o;
    if (d == 0) {
        stats[2 * set] = top;
        stats[2 * set + 1] = sum;
    }
    __syncthreads();
    const int real = threadIdx.x;
    if (real >= D)
        return;
    top = -INFINITY;
    for (int s = 0; s < kSets; ++s)
        top = fmaxf(top, stats[2 * s]);
    const float base = top == -INFINITY ? 0.0f : top;
    float value = 0.0f, total = 0.0f;
    for (int s = 0; s < kSets; ++s) {
        const float w = exp2_fast(stats[2 * s] - base);
        total = fmaf(w, stats[2 * s + 1], total);
        value = fmaf(w, acc[s * D + real], value);
    }
    finish<T>(a, seq, head, real, value, total);
}

int padded_reals(int dq)
{
    return 4 * padded_dq(dq);
}

// may_split: there is memory for partial results.
Token plan(const CacheAttention &a, bool may_split)
{
    Token t{};
    t.a = a;
    t.group = a.heads / a.cache.heads;
    t.group_blocks = (t.group + kQueries - 1) / kQueries;
    t.units = a.cache.heads * t.group_blocks;
    // spans beyond one for each sequence, where there is not a work-group for each
    // compute unit: so many that there is (4 x 65536 tokens: 18.9 us, 20.8 with two, 22.3
    // with four)
    const int64_t groups = int64_t(a.n) * t.units;
    if (may_split && groups < 256 && a.cache.capacity() > kRound) {
        const int64_t rounds = (int64_t(a.cache.capacity()) + kRound - 1) / kRound * a.n;
        t.spans = int(std::min<int64_t>(a.n + (256 + t.units - 1) / t.units, a.n + rounds));
    }
    return t;
}
size_t part_bytes(const Token &t)
{
    return size_t(t.spans) * t.a.heads * (padded_reals(t.a.cache.dq) + 2) * sizeof(float);
}

template <typename T, CacheForm F, int D> hipError_t launch(const Token &t, hipStream_t s)
{
    const CacheAttention &a = t.a;
    const unsigned grid = unsigned(t.units) * unsigned(t.part != nullptr ? t.spans : a.n);
    const int heads = std::min(t.group, kQueries), nb = a.bias.ny * a.bias.nx;
    const bool held = a.bias.table != nullptr && int64_t(heads) * nb <= kBiasLds;
    const size_t lds = std::max(size_t(kWaves * 4 * kChunk + (held ? heads * nb : 0)) * 4,
                                size_t(kWaves) * heads * (D + 2) * sizeof(float));
    if (a.bias.table == nullptr)
        cache_attention_kernel<T, F, D, 0><<<grid, kThreads, lds, s>>>(t);
    else if (held)
        cache_attention_kernel<T, F, D, 1><<<grid, kThreads, lds, s>>>(t);
    else
        cache_attention_kernel<T, F, D, 2><<<grid, kThreads, lds, s>>>(t);
    if (hipError_t e = hipGetLastError())
        return e;
    if (t.part != nullptr)
        cache_join_kernel<T, D><<<unsigned(a.n) * unsigned(a.heads), 256, 0, s>>>(t);
    return hipGetLastError();
}
template <typename T, CacheForm F> hipError_t launch_dq(const Token &t, hipStream_t s)
{
    switch (padded_reals(t.a.cache.dq)) {
    case 32:
        return launch<T, F, 32>(t, s);
    case 64:
        return launch<T, F, 64>(t, s);
    default:
        return launch<T, F, 128>(t, s);
    }
}

}  // namespace

size_t cache_attention_extra_bytes(const CacheAttention &a, DType)
{
    return part_bytes(plan(a, true));
}

hipError_t cache_attention_run(const CacheAttention &a, DType dt, void *extra, hipStream_t s)
{
    Token t = plan(a, extra != nullptr);
    if (t.spans > 0) {
        t.part = static_cast<float *>(extra);
        t.part_stats = t.part + size_t(t.spans) * a.heads * padded_reals(a.cache.dq);
    }
    switch (a.cache.form) {
    case CacheForm::BF16:
        return launch_dq<__bf16, CacheForm::BF16>(t, s);
    case CacheForm::F32:
        return launch_dq<float, CacheForm::F32>(t, s);
    default:
        return dt == DType::BF16 ? launch_dq<__bf16, CacheForm::E4M3>(t, s) : launch_dq<float, CacheForm::E4M3>(t, s);
    }
}

}  // namespace quan
