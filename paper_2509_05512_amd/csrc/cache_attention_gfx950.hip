// Attention of one new token per sequence over a paged cache on gfx950.
//
// A work-group takes a query head of a sequence; its waves take the keys in turn,
// two reals of a row in each lane, with a softmax of their own each, and are joined
// in LDS.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "cache_tile.h"

namespace quan {
namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64;

template <CacheForm F> __device__ __forceinline__ float element(const unsigned char *row, int i)
{
    if (F == CacheForm::E4M3)
        return from_e4m3(row[i])[0];
    if (F == CacheForm::BF16)
        return float(reinterpret_cast<const __bf16 *>(row)[i]);
    return reinterpret_cast<const float *>(row)[i];
}

__device__ __forceinline__ float wave_sum(float x)
{
    for (int l = 1; l < 64; l *= 2)
        x += __shfl_xor(x, l, 64);
    return x;
}

template <typename T, CacheForm F> __global__ void __launch_bounds__(kThreads) cache_attention_kernel(CacheAttention a)
{
    const Cache &c = a.cache;
    const int head = blockIdx.x % a.heads, seq = blockIdx.x / a.heads, kv_head = head / (a.heads / c.heads);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, d = 4 * c.dq;
    const int len = a.kv_len != nullptr ? min(max(a.kv_len[seq], 0), c.capacity()) : c.capacity();
    const T *q_row = static_cast<const T *>(a.q.data) + seq * a.q.s_n + int64_t(head) * c.dq;
    float q[2], o[2] = {0.0f, 0.0f};
#pragma unroll
    for (int e = 0; e < 2; ++e) {
        const int i = 2 * lane + e;
        q[e] = i < d ? float(q_row[(i / c.dq) * a.q.s_p + i % c.dq]) * a.scale * kLog2e : 0.0f;
    }
    float top = -INFINITY, sum = 0.0f;
    const int y = a.pos != nullptr ? query_pos(a.pos[2 * seq]) : 0, x = a.pos != nullptr ? query_pos(a.pos[2 * seq + 1]) : 0;
    for (int j = wave; j < len; j += kWaves) {
        const Slot s = slot_of(c, seq, j);
        if (s.row < 0)
            continue;
        const int64_t row = int64_t(s.row) + kv_head * c.page_tokens + s.slot;
        const unsigned char *k = c.keys + row * c.row_bytes, *v = c.values + row * c.row_bytes;
        float score = 0.0f, value[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int i = 2 * lane + e;
            score += i < d ? q[e] * element<F>(k, i) : 0.0f;
            value[e] = i < d ? element<F>(v, i) : 0.0f;
        }
        score = wave_sum(score);
        if (F == CacheForm::E4M3) {
            score *= factor_of(c.key_exp[row]);
            value[0] *= factor_of(c.value_exp[row]);
            value[1] *= factor_of(c.value_exp[row]);
        }
        if (a.bias.table != nullptr) {
            const int at_y = fast_div(j, a.by_width), at_x = j - at_y * a.width;
            const int dy = min(max(at_y - y, -a.bias.ry), a.bias.ry), dx = min(max(at_x - x, -a.bias.rx), a.bias.rx);
            const int iy = a.bias.by != nullptr ? min(max(a.bias.by[dy + a.bias.ry], 0), a.bias.ny - 1) : 0;
            const int ix = a.bias.bx != nullptr ? min(max(a.bias.bx[dx + a.bias.rx], 0), a.bias.nx - 1) : 0;
            score += in_log2(a.bias.table[(int64_t(head) * a.bias.ny + iy) * a.bias.nx + ix]);
        }
        const float now = fmaxf(top, score), m = now == -INFINITY ? 0.0f : now;
        const float back = exp2_fast(top - m), p = exp2_fast(score - m);
        top = now;
        sum = fmaf(sum, back, p);
#pragma unroll
        for (int e = 0; e < 2; ++e)
            o[e] = fmaf(o[e], back, p * value[e]);
    }
    __shared__ float acc[kWaves][128], stats[kWaves][2];
    acc[wave][2 * lane] = o[0];
    acc[wave][2 * lane + 1] = o[1];
    if (lane == 0) {
        stats[wave][0] = top;
        stats[wave][1] = sum;
    }
    __syncthreads();
    const int i = threadIdx.x;
    if (i >= d)
        return;
    float m = -INFINITY, total = 0.0f, out = 0.0f;
    for (int w = 0; w < kWaves; ++w)
        m = fmaxf(m, stats[w][0]);
    m = m == -INFINITY ? 0.0f : m;
    for (int w = 0; w < kWaves; ++w) {
        const float by = exp2_fast(stats[w][0] - m);
        total = fmaf(by, stats[w][1], total);
        out = fmaf(by, acc[w][i], out);
    }
    out *= total > 0.0f || total != total ? 1.0f / total : 0.0f;
    T *to = static_cast<T *>(const_cast<void *>(a.out.data)) + seq * a.out.s_n + int64_t(head) * c.dq;
    to[(i / c.dq) * a.out.s_p + i % c.dq] = T(out);
}

}  // namespace

size_t cache_attention_extra_bytes(const CacheAttention &, DType)
{
    return 0;
}

hipError_t cache_attention_run(const CacheAttention &a, DType dt, void *, hipStream_t s)
{
    const unsigned grid = unsigned(a.n) * unsigned(a.heads);
    if (a.cache.form == CacheForm::BF16)
        cache_attention_kernel<__bf16, CacheForm::BF16><<<grid, kThreads, 0, s>>>(a);
    else if (a.cache.form == CacheForm::F32)
        cache_attention_kernel<float, CacheForm::F32><<<grid, kThreads, 0, s>>>(a);
    else if (dt == DType::BF16)
        cache_attention_kernel<__bf16, CacheForm::E4M3><<<grid, kThreads, 0, s>>>(a);
    else
        cache_attention_kernel<float, CacheForm::E4M3><<<grid, kThreads, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace quan
