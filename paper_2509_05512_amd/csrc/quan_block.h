// Internal launch interface of the attention block's operators (norms with
// gate, residual scale and dropout; attention between the pixels of a map).
// Host-only declarations; every argument has been validated by the caller
// before one of these runs.
#pragma once

#include <hip/hip_runtime_api.h>
#include <stddef.h>
#include <stdint.h>

#include "quan_launch.h"

namespace quan {

// launch(args, work, extra, stream) as one call on the stream, with `bytes` of
// the block's workspace, and `extra_bytes` of another or NULL where that cannot
// be had (or no bytes are asked for).  Returns a QUAN_* code.
int run_on_stream(void *stream, size_t bytes, size_t extra_bytes,
                  hipError_t (*launch)(void *, void *, void *, hipStream_t), void *args, const char *what);

// Dropout's mask: element j of pixel m's row of 4C reals is kept where the 16
// bits j % 8 of Philox 4x32-7 (J. Salmon, M. Moraes, R. Dror, D. Shaw,
// "Parallel random numbers: as easy as 1, 2, 3", SC 2011) for counter (j / 8,
// m, offset) and key seed reach `cut`; rng holds {seed, offset} in device
// memory.  Kept elements are multiplied by `factor`.
struct Drop {
    const uint64_t *rng;
    unsigned cut;  // 0: no dropout
    float factor;
};

// Rows of 4c reals, one per pixel, of n images with hw pixels each.
struct RowsGeom {
    int64_t n, hw;
    int c;
};
constexpr int kRowsMaxChannels = 1024;

// out = x + scale gate drop(z), z = y or gamma y / rms(y); h = next_gamma out
// / rms(out) (next_gamma NULL: no h).  y NULL: h of x alone, no out.
struct ResidualForward {
    const void *x, *y;
    const float *gamma, *scale, *next_gamma;  // [4][c] or NULL
    const void *gate;                         // [n][4][c] or NULL
    void *out, *h;
};
hipError_t residual_forward_run(const RowsGeom &g, DType dt, const ResidualForward &a, const Drop &drop, float eps,
                                hipStream_t stream);

// The gradients of the above.  G = dout + the norm's gradient of dh at `out`
// goes to dx; its dropped, gated and scaled part through the norm of y to dy.
// y NULL: dx alone (dout may be NULL).  `work` must hold
// residual_backward_work_bytes(...) bytes.
struct ResidualBackward {
    const void *y, *dout, *out, *dh;
    const float *gamma, *scale, *next_gamma;
    const void *gate;
    void *dx, *dy, *dgate;
    float *dgamma, *dscale, *dnext_gamma;
};
size_t residual_backward_work_bytes(const RowsGeom &g, const ResidualBackward &a);
hipError_t residual_backward_run(const RowsGeom &g, DType dt, const ResidualBackward &a, const Drop &drop, float eps,
                                 void *work, hipStream_t stream);

hipError_t dropout_run(const RowsGeom &g, DType dt, const void *x, void *out, const Drop &drop, hipStream_t stream);

// Attention between the pixels of maps, heads of dq quaternion channels:
//   s_ij = scale Re<q_i, k_j> + table[head][by][bx],  P = softmax over the
//   image's keys j < kv_len,  out_i = sum_j P_ij v_j;  rows without a key: 0.
// A map: element (n, head, token, component, channel) at n s_n + head s_h +
// token s_t + component s_p + channel.
struct AttnMap {
    const void *data;
    int64_t s_n, s_t, s_p;
    bool vec;     // 16-byte aligned everywhere
    int64_t s_h;  // the head's channels: dq
};
// The bias.  by, bx: buckets of the offsets -r..r of key - (query + pos) per
// axis, offsets beyond them taking the end's (by NULL: one bucket).
struct AttnBias {
    const float *table;  // [heads][ny * nx], NULL: no bias
    const int32_t *by, *bx;
    int ny, nx, ry, rx;
};
struct AttnGeom {
    int n, heads, kv_heads, dq;
    int hq, wq, hk, wk;
    float scale;
    constexpr int lq() const { return hq * wq; }
    constexpr int lk() const { return hk * wk; }
};
constexpr int kAttnMaxDq = 32;       // quaternion channels of a head
constexpr int kAttnMaxWidth = 1792;  // of maps with more than one row, with a bias
constexpr int kAttnMaxBuckets = 1024;  // per axis
struct AttnCall {
    AttnGeom g;
    AttnMap q, k, v;
    AttnBias bias;
    const int32_t *kv_len;  // [n] or NULL
    const int32_t *pos;     // [n][2] (y, x) of query 0 in the keys' map, or NULL
};
// Heads are read as 16-byte chunks of whole rows of D = 4 * padded_dq reals;
// maps that do not lie so (unaligned slices, other dq) are copied first, head by
// head ([n][head][token][D], zeros in the added channels; of keys those that the
// image has).
constexpr int padded_dq(int dq) { return dq <= 8 ? 8 : dq <= 16 ? 16 : 32; }
struct AttnPack {
    static constexpr int kMaps = 6;
    AttnMap src[kMaps];
    const int32_t *kv_len[kMaps];  // [n], NULL: all tokens
    int heads[kMaps], tokens[kMaps];
    FastDiv by_heads[kMaps];
    void *dst[kMaps];
    int maps;
};
hipError_t attention_pack_run(const AttnPack &p, int n, int dq, DType dt, hipStream_t stream);

// out, and where given its remainder to 16 more bits (dense [n][lq][4][c]) and
// stats [n][heads][lq][2]: the row's maximum in units of log 2 and the sum of
// 2^(score - maximum).  `work` holds the copies that the call needs, `extra`
// (or NULL) partial results of a call with few queries.
// _fits: whether a tile's offsets fit in LDS (without a bias, and for maps as
// wide as each other, always).
bool attention_forward_fits(const AttnCall &a, DType dt);
size_t attention_forward_work_bytes(const AttnCall &a, DType dt);
size_t attention_forward_extra_bytes(const AttnCall &a, DType dt);
hipError_t attention_forward_run(const AttnCall &a, DType dt, const AttnMap &out, void *rest, float *stats, void *work,
                                 void *extra, hipStream_t stream);
// dtable [heads][ny * nx] or NULL.
struct AttnGradients {
    AttnMap out, dout, dq, dk, dv;
    const void *rest;
    const float *stats;
    float *dtable;
};
bool attention_backward_fits(const AttnCall &a, DType dt, const AttnGradients &g);
size_t attention_backward_work_bytes(const AttnCall &a, DType dt, const AttnGradients &g);
hipError_t attention_backward_run(const AttnCall &a, DType dt, const AttnGradients &g, void *work, hipStream_t stream);

}  // namespace quan
