// A paged cache of keys and values on gfx950: new tokens into its pages, in 8 bits
// with a power of two per row or as they are, and back.
//
// A row (a token's head of k or v) is taken by as many neighbouring lanes as it has
// 16-byte chunks, rounded up to a power of two; the rows of a token's heads lie side
// by side in the maps, so that neighbouring sets of lanes read neighbouring reals.
// The largest magnitude of a row is found in its lanes' registers.  Bound by the way
// of the maps and pages from and to memory.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "cache_tile.h"

namespace quan {
namespace {

constexpr int kThreads = 256;
constexpr int kFirsts = 2048;  // entries of `first` that a work-group holds in LDS

struct Copy {
    CacheCopy c;
    FastDiv by_heads, by_tokens;
    int rows, lanes;  // tokens x 2 heads; lanes of a row, a power of two
    int images;
};

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

// EPL reals of a head's row from real `at` on; components lie s_p apart.
template <typename T, int EPL, typename Do> __device__ __forceinline__ void for_reals(const AttnMap &m, int dq, int at, Do &&fn)
{
    int comp = at / dq, ch = at - comp * dq;
#pragma unroll
    for (int e = 0; e < EPL; ++e) {
        fn(e, at + e < 4 * dq, comp * m.s_p + ch);
        if (++ch == dq) {
            ch = 0;
            ++comp;
        }
    }
}

template <typename T, CacheForm F, bool READ>
__global__ void __launch_bounds__(kThreads) cache_copy_kernel(Copy p)
{
    constexpr int EPL = chunk_elems(F);
    constexpr bool E4M3 = F == CacheForm::E4M3;
    __shared__ int firsts[kFirsts];
    const CacheCopy &c = p.c;
    const Cache &cache = c.cache;
    const int32_t *first = c.seq.first;
    if (first != nullptr && c.seq.count < kFirsts) {
        for (int i = threadIdx.x; i <= c.seq.count; i += kThreads)
            firsts[i] = first[i];
        __syncthreads();
    }
    const int lane = threadIdx.x & (p.lanes - 1), per = kThreads / p.lanes;
    const int step = int(gridDim.x) * per;
    const int real = lane * EPL;
    const bool has = lane * 16 < cache.row_bytes;
    for (int64_t r = int64_t(blockIdx.x) * per + threadIdx.x / p.lanes; r < p.rows; r += step) {
        const int row = int(r);
        const int side = fast_div(row, p.by_heads), head = row - side * cache.heads;  // token * 2 + (1 for v)
        const int pixel = side >> 1;
        const bool value = side & 1;
        int seq, token, img, position;
        if (first == nullptr) {
            img = seq = fast_div(pixel, p.by_tokens);
            token = position = pixel - seq * c.seq.tokens;
        } else {
            const bool held = c.seq.count < kFirsts;
            seq = held ? find_sequence(firsts, c.seq.count, pixel) : find_sequence(first, c.seq.count, pixel);
            const Tokens t = held ? tokens_of(c.seq, firsts, seq) : tokens_of(c.seq, first, seq);
            img = 0;
            token = pixel;
            position = pixel - t.at;
            if (position < 0 || position >= t.len)
                continue;  // of no sequence
        }
        // (a start near the type's end wraps to below 0)
        position = int(unsigned(position) + unsigned(c.start != nullptr ? c.start[seq] : 0));
        const int end = c.kv_len != nullptr ? min(c.kv_len[seq], cache.capacity()) : cache.capacity();
        int64_t at = -1;
        if (position >= 0 && position < end) {
            const Slot s = slot_of(cache, seq, position);
            if (s.row >= 0)
                at = int64_t(s.row) + head * cache.page_tokens + s.slot;
        }
        const AttnMap &m = value ? c.v : c.k;
        T *x = static_cast<T *>(const_cast<void *>(m.data)) + img * m.s_n + token * m.s_t + int64_t(head) * cache.dq;
        unsigned char *chunk = (value ? cache.values : cache.keys) + at * cache.row_bytes + lane * 16;
        uint8_t *exponent = (value ? cache.value_exp : cache.key_exp) + at;
        // chunks of 8 reals (4 in fp32 rows) in one component, aligned
        const bool whole = m.vec && cache.dq % (EPL < 8 ? 4 : 8) == 0;
        if (READ) {
            float v[EPL];
#pragma unroll
            for (int e = 0; e < EPL; ++e)
                v[e] = 0.0f;
            if (at >= 0 && has) {
                if constexpr (E4M3) {
                    const i32x4 d = *reinterpret_cast<const i32x4 *>(chunk);
                    const float by = factor_of(*exponent);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const f32x4 t = from_e4m3(d[e]);
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            v[4 * e + i] = t[i] * by;
                    }
                } else if constexpr (F == CacheForm::BF16) {
                    const f32x8 t = to_f32(*reinterpret_cast<const bf16x8 *>(chunk));
#pragma unroll
                    for (int e = 0; e < EPL; ++e)
                        v[e] = t[e];
                } else {
                    const f32x4 t = *reinterpret_cast<const f32x4 *>(chunk);
#pragma unroll
                    for (int e = 0; e < EPL; ++e)
                        v[e] = t[e];
                }
            }
            if (whole) {
#pragma unroll
                for (int i = 0; i < EPL; i += EPL < 8 ? 4 : 8) {
                    const int comp = (real + i) / cache.dq;
                    T *to = x + comp * m.s_p + (real + i - comp * cache.dq);
                    if (real + i >= 4 * cache.dq)
                        continue;
#pragma unroll
                    for (int q = 0; q < (EPL < 8 ? 4 : 8); q += 4)
                        store_quad(to + q, f32x4{v[i + q], v[i + q + 1], v[i + q + 2], v[i + q + 3]}, 4, true);
                }
            } else {
                for_reals<T, EPL>(m, cache.dq, real, [&](int e, bool here, int64_t off) {
                    if (here)
                        x[off] = T(v[e]);
                });
            }
            continue;
        }
        float v[EPL];
        if (whole) {
#pragma unroll
            for (int i = 0; i < EPL; i += EPL < 8 ? 4 : 8) {
                const bool here = real + i < 4 * cache.dq;
                const int comp = here ? (real + i) / cache.dq : 0;
                const T *from = x + comp * m.s_p + (here ? real + i - comp * cache.dq : 0);
                if constexpr (EPL < 8) {
                    const f32x4 t = *reinterpret_cast<const f32x4 *>(from);
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        v[i + e] = here ? t[e] : 0.0f;
                } else {
                    const f32x8 t = to_f32(load_chunk<T>(from, here ? 8 : 0, true));
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        v[i + e] = t[e];
                }
            }
        } else {
            for_reals<T, EPL>(m, cache.dq, real, [&](int e, bool here, int64_t off) {
                const float t = float(x[here ? off : 0]);
                v[e] = here ? t : 0.0f;
            });
        }
        if constexpr (E4M3) {
            unsigned top = 0;
#pragma unroll
            for (int e = 0; e < EPL; ++e)
                top = max(top, __float_as_uint(v[e]) & 0x7fffffffu);
            for (int l = 1; l < p.lanes; l *= 2)
                top = max(top, unsigned(__shfl_xor(int(top), l, 64)));
            const unsigned byte = factor_byte(top);
            const float by = inverse_of(byte), most = byte == kLastByte ? 240.0f : 448.0f;
#pragma unroll
            for (int e = 0; e < EPL; ++e)
                v[e] = fminf(fmaxf(v[e] * by, -most), most);
            i32x4 d;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                d[e] = byte == 255u ? 0x7f7f7f7f : to_e4m3(v[4 * e], v[4 * e + 1], v[4 * e + 2], v[4 * e + 3]);
            if (at >= 0 && has) {
                *reinterpret_cast<i32x4 *>(chunk) = d;
                if (lane == 0)
                    *exponent = uint8_t(byte);
            }
        } else if (at >= 0 && has) {
            if constexpr (F == CacheForm::BF16) {
                f32x8 t;
#pragma unroll
                for (int e = 0; e < EPL; ++e)
                    t[e] = v[e];
                *reinterpret_cast<bf16x8 *>(chunk) = to_frag<__bf16>(t);
            } else {
                *reinterpret_cast<f32x4 *>(chunk) = f32x4{v[0], v[1], v[2], v[3]};
            }
        }
    }
}

template <bool READ> hipError_t copy_run(const CacheCopy &c, DType dt, hipStream_t s)
{
    Copy p;
    p.c = c;
    p.images = c.seq.first != nullptr ? 1 : c.seq.count;
    p.by_heads = FastDiv(c.cache.heads);
    p.by_tokens = FastDiv(c.seq.tokens);
    p.rows = p.images * c.seq.tokens * 2 * c.cache.heads;
    p.lanes = 1;
    while (p.lanes * 16 < c.cache.row_bytes)
        p.lanes *= 2;
    const int per = kThreads / p.lanes;
    const unsigned grid = unsigned(std::min<int64_t>((int64_t(p.rows) + per - 1) / per, 1 << 20));
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

hipError_t cache_write_run(const CacheCopy &c, DType dt, hipStream_t stream)
{
    return copy_run<false>(c, dt, stream);
}

hipError_t cache_read_run(const CacheCopy &c, DType dt, hipStream_t stream)
{
    return copy_run<true>(c, dt, stream);
}

}  // namespace quan
