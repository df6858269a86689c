// What distillation adds to the loss's products (sq_ce.hip), by the kernels of
// sq_distill.hip.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "sq_launch.h"

namespace sq {

// What rounding to bf16 took from a logit's gradient, kept of the entries of a token
// that lost the most (id < 0: none).
constexpr int kDistillLost = 8;
struct DistillLost {
  int id;
  float lost;
};

// One piece's logit gradients in bf16: columns of rows [v0, v0 + n) of the head, in
// `groups` matrices [T, width] one after another, whose last begins `shift` columns
// inside the one before it; the rows from `main` on in fp32, 8 per token.
struct DistillPiece {
  uint16_t* d;
  int64_t v0;
  int n, width, groups, shift;
  float* dtail;
  int64_t main;
  const int* rows;          // compact row -> token, or null (row = token)
  const int* count;         // live rows, or null (T)
  int T, V;
  DistillLost* lost;        // [T, kDistillLost] by compact row, of all pieces: written with one of them, else null
};

// y[t] = V where token t has an entry that counts, else -1.
int distill_live_launch(const Distill& k, int T, int V, int* y, hipStream_t s);
// The same, and k.picked: the logits of the entries that count times f, zeros for the
// others.
int distill_pick_launch(const Distill& k, int head, int T, int V, int H, const void* X, const void* W, const uint8_t* scales,
                        float f, int* y, hipStream_t s);
// loss and lse from the tiles' (max, sum) pairs and k.picked.
int distill_loss_launch(const Distill& k, const float2* part, const int* rows, const int* count, const int* y, int T, int V,
                        int tiles, float* loss, float* lse, hipStream_t s);
// dloss (p - q) at the entries of a piece, over the dloss p that stands there.
int distill_put_launch(const Distill& k, const DistillPiece& piece, const float* lse, const float* dloss, hipStream_t s);

}  // namespace sq
