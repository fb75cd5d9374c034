// A paged cache of keys and values on gfx950: new tokens into its pages, in 8 bits
// with a power of two per row or as they are, and back.
//
// A work-group takes some tokens and finds their slots first, and where they lie in the
// maps, a thread for each.  Then a lane takes 8 reals of a row (a token's head of k or
// v) and neighbouring lanes, as many as a power of two, the row, neighbouring rows being
// a token's heads, which lie side by side in the maps; a lane has 4 rows in flight.  The
// largest magnitude of a row is found in its lanes' registers.
//
// Bound by HBM and, writing 8 bits, by the vector instructions on the way (45 % busy;
// 2.2 waves a SIMD, waiting 54 % of their time): 16 x 1600 tokens of 8 heads of 64 bf16
// reals written in 19.2 us, 8 sequences of up to 6400 tokens of 4 heads of 128 read in
// 16.2, 79 MB each, of which a large copy takes 14.5 us; with one row in flight 28.6
// and 24.4.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "cache_tile.h"

namespace quan {
namespace {

constexpr int kThreads = 256;
constexpr int kFirsts = 2048;  // entries of `first` that a work-group holds in LDS
constexpr int kTokens = 64;    // most tokens of a work-group
constexpr int kAhead = 4;      // rows of a set of lanes in flight

struct Copy {
    CacheCopy c;
    FastDiv by_heads, by_tokens;
    int64_t pixels;
    int tokens, lanes;  // of a work-group; of a row, a power of two
};
constexpr int kNoSequence = -2, kNoSlot = -1;

// The largest of neighbouring lanes' numbers, 1, 2, 4, 8 or 16 of them (an 8-bit row has
// 16 at most).
__device__ __forceinline__ unsigned lanes_max(unsigned x, int lanes)
{
    const auto step = [&](unsigned y, int of) { x = lanes > of ? max(x, y) : x; };
    step(__builtin_amdgcn_update_dpp(0, int(x), 0xB1, 0xf, 0xf, false), 1);   // lane ^ 1
    step(__builtin_amdgcn_update_dpp(0, int(x), 0x4E, 0xf, 0xf, false), 2);   // lane ^ 2
    step(__builtin_amdgcn_update_dpp(0, int(x), 0x141, 0xf, 0xf, false), 4);  // 7 - lane of 8
    step(__builtin_amdgcn_update_dpp(0, int(x), 0x140, 0xf, 0xf, false), 8);  // 15 - lane of 16
    return x;
}

// The sequence of pixel `token` of a packed map: the last that starts at or
// before it.
__device__ __forceinline__ int find_sequence(const int32_t *first, int count, int token)
{
    int low = 0, high = count;  // first[low] <= token < first[high] where they are in order
    while (high - low > 1) {
        const int mid = (low + high) >> 1;
        if (first[mid] <= token)
            low = mid;
        else
            high = mid;
    }
    return low;
}

// 8 reals of a map's row for the head at x, from real `at` on (fewer at the head's
// end): where they are, and whether, goes to fn(real, its distance from x).
template <typename Do> __device__ __forceinline__ void for_reals(const AttnMap &m, int dq, int at, Do &&fn)
{
    int comp = at / dq, ch = at - comp * dq;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        fn(e, at + e < 4 * dq ? comp * m.s_p + ch : -1);
        if (++ch == dq) {
            ch = 0;
            ++comp;
        }
    }
}

template <typename T, CacheForm F, bool READ>
__global__ void __launch_bounds__(kThreads) cache_copy_kernel(Copy p)
{
    constexpr bool E4M3 = F == CacheForm::E4M3;
    typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
    __shared__ int firsts[kFirsts], slots[kTokens];
    __shared__ T *maps[kTokens][2];  // where a token's keys and values lie
    const CacheCopy &c = p.c;
    const Cache &cache = c.cache;
    const int32_t *first = c.seq.first;
    const int pixel0 = int(blockIdx.x) * p.tokens, count = int(min(int64_t(p.tokens), p.pixels - pixel0));
    const bool held = c.seq.count < kFirsts;
    if (first != nullptr && held) {
        for (int i = threadIdx.x; i <= c.seq.count; i += kThreads)
            firsts[i] = first[i];
        __syncthreads();
    }
    // the row of head 0 at a token's slot
    if (int(threadIdx.x) < count) {
        const int pixel = pixel0 + int(threadIdx.x);
        int seq, position, slot = kNoSlot;
        bool some = true;
        if (first == nullptr) {
            seq = fast_div(pixel, p.by_tokens);
            position = pixel - seq * c.seq.tokens;
        } else {
            seq = held ? find_sequence(firsts, c.seq.count, pixel) : find_sequence(first, c.seq.count, pixel);
            const Tokens t = held ? tokens_of(c.seq, firsts, seq) : tokens_of(c.seq, first, seq);
            position = pixel - t.at;
            some = position >= 0 && position < t.len;
        }
        if (some) {
            // (a start near the type's end wraps to below 0)
            position = int(unsigned(position) + unsigned(c.start != nullptr ? c.start[seq] : 0));
            const int end = c.kv_len != nullptr ? min(c.kv_len[seq], cache.capacity()) : cache.capacity();
            if (position >= 0 && position < end) {
                const Slot s = slot_of(cache, seq, position);
                if (s.row >= 0)
                    slot = s.row + s.slot;
            }
        }
        slots[threadIdx.x] = some ? slot : kNoSequence;
        const int img = first == nullptr ? seq : 0, in_map = pixel - img * c.seq.tokens;
        for (int side = 0; side < 2; ++side) {
            const AttnMap &m = side ? c.v : c.k;
            maps[threadIdx.x][side] = static_cast<T *>(const_cast<void *>(m.data)) + img * m.s_n + in_map * m.s_t;
        }
    }
    __syncthreads();

    const int lane = threadIdx.x & (p.lanes - 1), per = kThreads / p.lanes;
    const int rows = count * 2 * cache.heads, real = 8 * lane;
    const bool here = real < 4 * cache.dq;
    const int comp = here ? real / cache.dq : 0, ch = here ? real - comp * cache.dq : 0;
    const int64_t in_k = comp * c.k.s_p + ch, in_v = comp * c.v.s_p + ch;  // the lane's reals of a token's head
    const bool whole = c.k.vec && c.v.vec && cache.dq % 8 == 0;  // 8 reals lie side by side, aligned
    // bytes of the lane's 8 elements in a row, and how many of them it has
    constexpr int kBytes = 8 * cache_elem_size(F);
    const int at_byte = lane * kBytes;
    const auto row_at = [&](int i) { return uint64_t(unsigned(i)) * unsigned(cache.row_bytes) + at_byte; };
    for (int r0 = threadIdx.x / p.lanes; r0 < rows; r0 += per * kAhead) {
        T *x[kAhead];
        int at[kAhead];  // (a cache has fewer than 2^31 rows)
        bool value[kAhead];
        int slot[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int row = min(r0 + u * per, rows - 1);
            const int side = fast_div(row, p.by_heads), head = row - side * cache.heads;  // token * 2 + (1 for v)
            value[u] = side & 1;
            slot[u] = r0 + u * per < rows ? slots[side >> 1] : kNoSequence;
            at[u] = max(slot[u], 0) + head * cache.page_tokens;
            x[u] = maps[side >> 1][side & 1] + head * cache.dq;
        }
        f32x8 v[kAhead];
        if constexpr (READ) {
            unsigned byte[kAhead];
            typedef typename Elem<T>::frag frag;
            u32x2 d[kAhead];
            frag f[kAhead];
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                byte[u] = 127;
                d[u] = u32x2{};
                f[u] = frag{};
                if (slot[u] < 0)
                    continue;
                const unsigned char *row = (value[u] ? cache.values : cache.keys) + row_at(at[u]);
                if constexpr (E4M3) {
                    if (at_byte < cache.row_bytes)
                        d[u] = *reinterpret_cast<const u32x2 *>(row);
                    byte[u] = (value[u] ? cache.value_exp : cache.key_exp)[at[u]];
                } else if (at_byte + kBytes <= cache.row_bytes) {
                    f[u] = *reinterpret_cast<const frag *>(row);
                } else if (at_byte < cache.row_bytes) {  // (half of 8 fp32 elements)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        f[u][e] = reinterpret_cast<const T *>(row)[e];
                }
            }
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                if constexpr (E4M3) {
                    const f32x4 a = from_e4m3(d[u][0]), b = from_e4m3(d[u][1]);
                    v[u] = __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7) * factor_of(byte[u]);
                } else {
                    v[u] = to_f32(f[u]);
                }
                if (slot[u] == kNoSequence)
                    continue;
                if (whole) {
                    store_chunk<T>(x[u] + (value[u] ? in_v : in_k), v[u], here ? 8 : 0, true);
                } else {
                    for_reals(value[u] ? c.v : c.k, cache.dq, real, [&](int e, int64_t off) {
                        if (off >= 0)
                            x[u][off] = T(v[u][e]);
                    });
                }
            }
        } else {
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                if (whole) {
                    v[u] = to_f32(load_chunk<T>(x[u] + (value[u] ? in_v : in_k), here ? 8 : 0, true));
                } else {
                    for_reals(value[u] ? c.v : c.k, cache.dq, real, [&](int e, int64_t off) {
                        const float t = float(x[u][off >= 0 ? off : 0]);
                        v[u][e] = off >= 0 ? t : 0.0f;
                    });
                }
            }
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                unsigned char *row = (value[u] ? cache.values : cache.keys) + row_at(at[u]);
                if constexpr (E4M3) {
                    unsigned top = 0;
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        top = max(top, __float_as_uint(v[u][e]) & 0x7fffffffu);
                    top = lanes_max(top, p.lanes);
                    const unsigned byte = factor_byte(top);
                    const float by = inverse_of(byte), most = byte == kLastByte ? 240.0f : 448.0f;
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        v[u][e] = __builtin_amdgcn_fmed3f(v[u][e] * by, -most, most);
                    u32x2 d = {unsigned(to_e4m3(v[u][0], v[u][1], v[u][2], v[u][3])),
                               unsigned(to_e4m3(v[u][4], v[u][5], v[u][6], v[u][7]))};
                    if (byte == 255u)
                        d = 0x7f7f7f7fu;
                    if (slot[u] < 0)
                        continue;
                    if (at_byte < cache.row_bytes)
                        *reinterpret_cast<u32x2 *>(row) = d;
                    if (lane == 0)
                        (value[u] ? cache.value_exp : cache.key_exp)[at[u]] = uint8_t(byte);
                } else if (slot[u] >= 0) {
                    if (at_byte + kBytes <= cache.row_bytes)
                        store_chunk<T>(reinterpret_cast<T *>(row), v[u], 8, true);
                    else if (at_byte < cache.row_bytes)
                        store_quad(reinterpret_cast<T *>(row), f32x4{v[u][0], v[u][1], v[u][2], v[u][3]}, 4, true);
                }
            }
        }
    }
}

Copy copy_plan(const CacheCopy &c)
{
    Copy p;
    p.c = c;
    p.by_heads = FastDiv(c.cache.heads);
    p.by_tokens = FastDiv(c.seq.tokens);
    p.pixels = int64_t(c.seq.first != nullptr ? 1 : c.seq.count) * c.seq.tokens;
    p.lanes = 1;
    while (p.lanes * 8 * cache_elem_size(c.cache.form) < c.cache.row_bytes)
        p.lanes *= 2;
    // so many tokens that each lane has kAhead rows, or twice as many where that leaves
    // four work-groups to a compute unit (16 x 1600 tokens of 8 heads written: 22.3 us
    // against 23.2, 24.2 with four times as many; 25600 of 4 heads read: 19.1, 19.7, 20.1)
    const int rows = kAhead * kThreads / p.lanes;
    p.tokens = std::max(1, std::min(kTokens, rows / (2 * c.cache.heads)));
    if (2 * p.tokens <= kTokens && p.pixels / (2 * p.tokens) >= 1024)
        p.tokens *= 2;
    // (few tokens: over the chip)
    p.tokens = int(std::min<int64_t>(p.tokens, (p.pixels + 255) / 256));
    return p;
}

template <bool READ> hipError_t copy_run(const CacheCopy &c, DType dt, hipStream_t s)
{
    const Copy p = copy_plan(c);
    const unsigned grid = unsigned((p.pixels + p.tokens - 1) / p.tokens);
    switch (c.cache.form) {
    case CacheForm::BF16:
        cache_copy_kernel<__bf16, CacheForm::BF16, READ><<<grid, kThreads, 0, s>>>(p);
        break;
    case CacheForm::F32:
        cache_copy_kernel<float, CacheForm::F32, READ><<<grid, kThreads, 0, s>>>(p);
        break;
    default:
        if (dt == DType::BF16)
            cache_copy_kernel<__bf16, CacheForm::E4M3, READ><<<grid, kThreads, 0, s>>>(p);
        else
            cache_copy_kernel<float, CacheForm::E4M3, READ><<<grid, kThreads, 0, s>>>(p);
    }
    return hipGetLastError();
}

}  // namespace

int64_t cache_copy_groups(const CacheCopy &c)
{
    const Copy p = copy_plan(c);
    return (p.pixels + p.tokens - 1) / p.tokens;
}

hipError_t cache_write_run(const CacheCopy &c, DType dt, hipStream_t stream)
{
    return copy_run<false>(c, dt, stream);
}

hipError_t cache_read_run(const CacheCopy &c, DType dt, hipStream_t stream)
{
    return copy_run<true>(c, dt, stream);
}

}  // namespace quan
