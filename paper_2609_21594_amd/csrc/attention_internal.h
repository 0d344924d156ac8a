// Internal interface between the attention entry points (attention_api.hip)
// and their gfx950 kernels (attention_kernels.hip).  Not installed.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "muon_internal.h"

namespace muon {

// A [batch, tokens, heads, head_dim] array: strides in bytes, head_dim
// contiguous.
struct Heads {
  char* p;
  int64_t batch, token, head;
};

// Sequences of a call.  Dense: `batch` sequences of q_tokens and k_tokens,
// each cut to q_len[b] / k_len[b] where given.  Packed (q_off given): n_seq
// sequences one behind the other on one token axis, sequence s being
// [off[s], off[s + 1]).  The device values are clamped to the token axes
// before use, so that no value reaches an address outside them.
struct Seqs {
  int64_t batch;
  int32_t q_tokens, k_tokens, n_seq;
  const int32_t *q_off, *k_off, *q_len, *k_len;
};

struct AttnArgs {
  Heads q, k, v, out, res, dout, dq, dk, dv;
  Seqs seqs;
  int32_t q_heads, kv_heads, group, dim;
  int32_t causal, window;
  int32_t fill;              // packed: rows that no sequence holds get zeros (lse: -inf)
  float scale, scale2;       // scale2 = scale * log2(e)
  float* lse;                // [batch][q_heads][q_tokens], natural logarithm
  float* max_logits;         // [q_heads] or null
  // forward, split over the keys: per split and row the unnormalised output
  // (fp32) and its maximum and sum
  int32_t splits;
  float* part_o;             // [splits][rows][dim]
  float2* part_ml;           // [splits][rows]
  // backward: per row log2(sum exp) (+inf where nothing is visible), dout . out,
  // and (fp32) what the probabilities are multiplied with
  float *lse2, *delta, *norm;
  // backward, the heads of a group in kv_parts parts with workgroups of their
  // own: where more than one, the parts' fp32 gradients,
  // [batch * k_tokens][kv_heads][kv_parts][dim]
  int32_t kv_parts;
  float *part_dk, *part_dv;
  // fp32: the planes of the arrays that tiles are staged from (k_split)
  char *split_q, *split_k, *split_v, *split_do;
  // what the tiles are staged from, and bytes between a row's planes (set by
  // the launch)
  Heads sq, sk, sv, sdo;
  int32_t plane;
};
// Bytes of the planes of an fp32 array of `rows` rows.
inline size_t split_bytes(int64_t rows, int dim) { return size_t(rows) * size_t((dim + 7) / 8) * 48; }

hipError_t run_attention_forward(AttnArgs a, int dtype, hipStream_t st, LaunchTimer* timer);
hipError_t run_attention_backward(AttnArgs a, int dtype, hipStream_t st, LaunchTimer* timer);
// Over how many parts of the key axis the forward pass of this request is
// spread (1: none), and in how many parts its backward pass takes the query
// heads that share keys.
int forward_splits(const Seqs& s, int q_heads, int kv_heads, int dim, bool causal, int window);
int backward_parts(const Seqs& s, int q_heads, int kv_heads, bool causal, int window);

constexpr int kRotaryMax = 4;
struct RotaryTensor {
  Heads x, y;
  int32_t heads;
  int32_t vec;               // 16-byte accesses
};
struct RotaryArgs {
  RotaryTensor t[kRotaryMax];
  int32_t n;
  int64_t batch, tokens;
  const void* positions;     // null: 0, 1, .. along the tokens
  int32_t positions64;       // int64 (else int32)
  int64_t pos_batch, pos_token;  // strides in elements
  int64_t first;             // added to every position
  const double* freqs;       // dim_rot / 2, radians a position
  int32_t dim, rot, interleaved;
  float scale, sign;
};
hipError_t run_rotary(const RotaryArgs& a, int dtype, hipStream_t st, LaunchTimer* timer);

constexpr int kClipMax = 32;
struct ClipEntry {
  char *wq, *wk;
  int64_t ldq, ldk;          // bytes
  float* logits;
  int32_t q_heads, kv_heads, dim, cols;
  int32_t vec;
  float threshold;
};
struct ClipArgs {
  ClipEntry e[kClipMax];
  int32_t first[kClipMax + 1];  // first workgroup of each entry
  int32_t n;
  int32_t rows;                 // rows of a workgroup, kClipRows at most
};
hipError_t run_qk_clip(const ClipArgs& a, int dtype, hipStream_t st, LaunchTimer* timer);
hipError_t run_reset_logits(const ClipArgs& a, hipStream_t st);
// Rows of its entry one workgroup of the clip takes: 16 where that still makes
// 1024 workgroups, else 4, one a wave (on an MI355X 32 layers of 4096 + 1024
// rows of 4096 bf16 take 113 us with 16 rows, 130 with 8; one of 1024 rows of
// 768 fp32 7.6 us with 16, 4.6 with 4).
constexpr int kClipRows = 16, kClipRowsFew = 4;

}  // namespace muon
