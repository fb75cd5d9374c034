// Internal launch interface of the operators on sequences of pixels: a paged
// cache of keys and values, attention of one new token over it, and causal
// attention of packed sequences.  Host-only declarations; every argument has
// been validated by the caller before one of these runs.
#pragma once

#include "quan_block.h"

namespace quan {

// Where the tokens of the sequences lie in a map of images of `tokens` pixels
// each: sequence i is image i, or with `first` (device, [count + 1]) pixels
// first[i] .. first[i + 1] - 1 of the one image.
struct Sequences {
    const int32_t *first;
    int count, tokens;
};

enum class CacheForm : int { F32 = 0, BF16 = 1, E4M3 = 2 };
constexpr int cache_elem_size(CacheForm f) { return f == CacheForm::F32 ? 4 : f == CacheForm::BF16 ? 2 : 1; }
// Bytes of a row: a head's 4 dq reals, component-major, up to whole 16 bytes.
constexpr int cache_row_bytes(int dq, CacheForm f) { return (4 * dq * cache_elem_size(f) + 15) / 16 * 16; }

// Row r of a page's head h is row (page * heads + h) * page_tokens + r of keys,
// values and the exponents' bytes.
struct Cache {
    unsigned char *keys, *values;
    uint8_t *key_exp, *value_exp;  // E4M3: e + 127 of a row's factor 2^e
    const int32_t *table;          // [sequences][table_pages]; entries outside 0..pages-1: no page
    CacheForm form;
    int pages, page_tokens, heads, dq, sequences, table_pages, row_bytes;
    FastDiv by_page;  // page_tokens
    constexpr int capacity() const { return table_pages * page_tokens; }
};

// Tokens of maps k, v to positions start[i] + j of their sequence, and back.
// Positions at or behind kv_len[i] (NULL: the table's end) are left alone, and
// read as zeros.
struct CacheCopy {
    Cache cache;
    Sequences seq;
    AttnMap k, v;
    const int32_t *start, *kv_len;  // [sequences]; NULL: 0, the table's end
};
int64_t cache_copy_groups(const CacheCopy &c);  // work-groups of 256 lanes
hipError_t cache_write_run(const CacheCopy &c, DType dt, hipStream_t stream);
hipError_t cache_read_run(const CacheCopy &c, DType dt, hipStream_t stream);

// One query per sequence against the positions below kv_len (NULL: all that the
// table has).  The bias's offsets are those from place pos = (y, x) of the query
// to place (j / width, j % width) of position j.
struct CacheAttention {
    Cache cache;
    AttnMap q, out;
    AttnBias bias;
    const int32_t *kv_len, *pos;
    int n, heads, width;
    FastDiv by_width;
    float scale;
};
size_t cache_attention_extra_bytes(const CacheAttention &a, DType dt);
hipError_t cache_attention_run(const CacheAttention &a, DType dt, void *extra, hipStream_t stream);

// Queries of a sequence are the last of its keys' tokens: with `causal` query i
// of lq sees keys j <= i + lk - lq.
struct PackedCall {
    AttnMap q, k, v;
    Sequences qs, ks;
    int images, heads, kv_heads, dq;  // images of the maps: 1 with qs.first
    bool causal;
    float scale;
    constexpr int64_t q_tokens() const { return int64_t(images) * qs.tokens; }
    constexpr int64_t k_tokens() const { return int64_t(images) * ks.tokens; }
};
// stats [heads][q_tokens][2] or NULL; rest (bf16) the remainder of out to 16 more
// bits, dense like it, or NULL.
size_t packed_forward_work_bytes(const PackedCall &c, DType dt);
size_t packed_forward_extra_bytes(const PackedCall &c, DType dt);
hipError_t packed_forward_run(const PackedCall &c, DType dt, const AttnMap &out, void *rest, float *stats, void *work,
                              void *extra, hipStream_t stream);
struct PackedGradients {
    AttnMap out, dout, dq, dk, dv;
    const void *rest;
    const float *stats;
};
// A dense map like q's.
inline AttnMap packed_dense(const PackedCall &c, const void *data)
{
    const int64_t all = int64_t(c.heads) * c.dq;
    return {data, c.qs.tokens * 4 * all, 4 * all, all, c.dq % 8 == 0, c.dq};
}
size_t packed_backward_work_bytes(const PackedCall &c, DType dt, const PackedGradients &g);
hipError_t packed_backward_run(const PackedCall &c, DType dt, const PackedGradients &g, void *work, hipStream_t stream);
// Maps that do not lie in whole aligned chunks are copied first (see AttnPack):
// bytes of a copy, and one more map of a launch, which `m` is afterwards.
size_t packed_copy_bytes(int64_t tokens, int heads, int dq, DType dt);
void packed_copy_add(AttnPack &pack, AttnMap &m, int images, int tokens, int heads, int dq, DType dt, unsigned char *&at);
// Blocks of `size` tokens that the sequences have at most (see locate() in
// packed_tile.h).
inline int64_t packed_blocks(const Sequences &s, int size = 128)
{
    return s.first != nullptr ? int64_t(s.tokens) / size + s.count
                              : int64_t(s.count) * ((int64_t(s.tokens) + size - 1) / size);
}

}  // namespace quan
