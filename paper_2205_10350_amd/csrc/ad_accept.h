// Acceptance of drafted tokens under sampled decoding (ad_accept_sampled.hip).
#pragma once

#include "ad_internal.h"

namespace ad {

struct AcceptArgs {
  const void* logits;            // [rows, vocab], rows `stride` elements apart
  size_t stride;
  const int* draft;              // [rows]
  const float* probs;            // [rows, vocab], rows probs_stride apart; null: drafted tokens are certain
  size_t probs_stride;
  const float* temperature;      // [n_seq]; null: 1
  const float *accept_u, *pick_u;   // [rows], [n_seq]
  const int* row_start;          // [n_seq + 1]
  int vocab, n_seq, rows, max_rows;
  int* n_accept;                 // [n_seq], may be null
  int* tokens;                   // [rows]
  int keep;                      // 1: rows without a decided token keep what `tokens` holds
  // the launcher's: per row and piece of the vocabulary, per sequence and piece
  int pieces, rest;              // rest: the deciding rows' sums are taken apart (rest_sum)
  double* piece_sum;
  float* piece_max;
  double* rest_sum;
  struct AcceptRowInfo* row_info;   // [rows]
};
struct AcceptRowInfo { double z; float m; int stands; };
// The inputs of a verify call, host-visible and by sequence, as packed rows in device memory: draft, u [n_seq, k_max], v, t [n_seq] -> rows of
// row_start (draft_out, u_out) and copies (v_out, t_out)
void launch_accept_inputs(const int* draft, const float* u, const float* v, const float* t, int k_max, const int* row_start, int n_seq, int* draft_out,
                          float* u_out, float* v_out, float* t_out, hipStream_t s);
size_t accept_bytes(int n_seq, int rows, int vocab);
// Whether a launch looks the rows up in the table instead of taking max_rows of every sequence (by sequence: at most 65,535)
inline bool accept_packed(int n_seq, int rows, int max_rows) { return (size_t)n_seq * max_rows > 4 * (size_t)rows; }
void launch_accept_sampled(int dtype, AcceptArgs a, void* ws, hipStream_t s);
void launch_accept_nothing(const AcceptArgs& a, hipStream_t s);   // a.rows == 0: counts of 0

}  // namespace ad
