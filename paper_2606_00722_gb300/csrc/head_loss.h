// What the kernels of the head's loss share: the plan of one piece of a call
// (sizes, operands, workspace) and their launchers.
#pragma once
#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/epic.h"

namespace epic {

constexpr int kRowTile = 256;   // rows of a workspace come in whole tiles
constexpr int kRecCols = 128;   // tokens whose exponentials one record sums
// Rows of one target whose gradient at it is kept in 32 bits for the head's gradient (an int4).  With none, 1, 2 and 4 the head's
// gradient of a step in bf16 is off by 0.0027, 0.0020, 0.0017 and 0.0017 of itself (500 rows, 1,000 tokens drawn alike), and by
// 0.0027, 0.0022, 0.0021 and 0.0020 with targets as frequent as words (2,048 rows, 32,768 tokens); a step of 500 x 256 x 1,000 takes
// 32, 33, 35 and 37 us, large ones the same within 2 %.
constexpr int kListed = 4;
constexpr int kMostParts = 64;  // of a gradient's sum

// Few tiles with long sums are cut into parts, whose sums meet in a second kernel: of gradients of hidden states over the
// tokens, of the head's over the positions.  1: not cut; 0: no such gradient.
struct GradSplit {
  int hidden_parts, head_parts;
  int tile_cost;        // what a tile costs beside its sum, in steps of it
  float *hidden, *head; // [parts][cap][ldp], [parts][tokens][ldp]
  long long tokens;     // V in whole tiles
};

// A piece: up to `cap` positions of the call.  Those that count stand in order, packed, in rows 0..*count-1 of the
// workspace; rows from there to the end of the tile are zeros in hc, hs and e.
struct HeadPlan {
  int rows, cap;            // positions of this piece; rows of room (a multiple of kRowTile)
  int d, V, nrec;
  long long ldh, lde, ldw;  // elements from row to row of hc and hs, of e, of the head
  const void* head;         // [V][ldw]
  int* count;               // rows that count
  int* again;               // != 0: e holds gradients of logits; see below
  float* post;              // power of two that gradients of logits in e are multiplied with
  int* counts;              // of 256 positions each, and the largest factor among them
  float* tops;
  int* src;                 // [cap] position in the piece
  long long* to;            // [cap] where the row's gradient begins, from the first position's
  int* tgt;                 // [cap] target token
  float *g;                 // [cap] what the row's gradient is multiplied with (weight, gradient from above)
  float *zt;                // [cap] logit of the target
  // Either e = 2^(z log2 e - ref), ref a whole number; a gradient of a logit is coef e, and hs = coef h.
  float *ref, *coef;        // [cap]
  // Or, where the logsumexp is known, e = known_mul 2^(z log2 e - known_ref), gradients of logits / *post.
  float *known_ref, *known_mul;  // [cap]
  // The gradient at the target, minus the sum of the others' (so that little is lost where they are few), is most of a row's.
  // Of the first kListed rows of a target it is 0 in e, kept in 32 bits, and multiplied with the target's row of the head, and
  // with the hidden state, as sums leave.  More rows of one target have it in e: in the gradient of the head their roundings even
  // out, and in a row's own, which has no other as large, what the rounding took is added in the same way.
  float *at_target;         // [cap] that: all of it, or what the rounding took
  float *e_target;          // [cap] what e holds there, as gradients of logits
  int4* list;               // [V] the first rows with that target, or -1; NULL without gradients
  float2* rec;              // [nrec][cap] (whole reference, sum of exponentials relative to it), target left out
  void *hc, *hs;            // [cap][ldh] hidden states; the same times coef, or NULL
  void* e;                  // [cap][lde]
  float* acc;               // [V][ldp] or NULL: gradient of the head so far, of calls in several pieces
  long long ldp;            // elements from row to row of acc and of parts, a multiple of 32
  GradSplit split;
};

// How a piece's gradient of the head meets the pieces before it
enum HeadSum { kOnly = 0, kFirst = 1, kMiddle = 2, kLast = 3 };

// Where gradients of hidden states [B][n][d] go; a packed row's begins `to` elements behind
struct HiddenGrad {
  void* grad;
  long long stride_b, stride_n;
};

// Logits of the packed rows.  sums: records and target logits.  probs: e, with a known logsumexp or not.  only_again: nothing
// unless *again; then with e_target at the targets.
struct LogitsPass {
  bool sums, probs, known, only_again;
};

// How boxes of the operands are copied, the same for all of a call's kernels and pieces: 64 columns by 64 rows, those that go
// out by 32 rows
struct HeadMaps {
  CUtensorMap hc, hs, head, e, e_out, grad_out, hidden_parts, head_parts;
  bool boxes;  // rows of grad_out start at multiples of 16 bytes and end there (a box's end is cut in whole 16 bytes)
};
// grads: they are wanted; grad_head: or NULL
epic_status make_head_maps(HeadMaps& maps, const HeadPlan& p, int dtype, bool grads, void* grad_head, long long stride);

epic_status launch_head_logits(const HeadPlan& p, const HeadMaps& maps, int dtype, const LogitsPass& pass, cudaStream_t st);
// Gradients of hidden states, grad[to] = coef e W (out.grad NULL: none), and of the head, grad_head [V][stride] = e^T hs with the
// pieces before (NULL: none); of gradients of logits in e, post e W and post e^T hc.
epic_status launch_head_grads(const HeadPlan& p, const HeadMaps& maps, int dtype, const HiddenGrad& out, void* grad_head,
                              long long stride, HeadSum sum, cudaStream_t st);

GradSplit split_grads(int rows, int d, int V);

}  // namespace epic
