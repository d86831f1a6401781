// Descriptors of the operators that work on a caller's tensors without a network: scores of classes, their gradient, and
// the norm of gradients, clipping by it and the update with clipped gradients.  Plain data only.
#pragma once
#include <stddef.h>
#include <stdint.h>

#ifndef CNN_GLOBAL
#define CNN_GLOBAL
#endif

namespace cnn355 {

enum ElementType : int { ELEMENT_F32 = 0, ELEMENT_BF16 = 1, ELEMENT_F16 = 2 };   // CNN_TYPE_* of the C ABI
constexpr size_t element_bytes(int type) { return type == ELEMENT_F32 ? 4 : 2; }

// ---- scores of classes ------------------------------------------------------------------------
constexpr int SCORE_TOP = 64;      // best classes at most: one a lane
constexpr int SCORE_TILE = 1024;   // classes that a wavefront looks at together, 16 a lane
constexpr int SCORE_PARTS = 256;   // workgroups that share a row at most

struct ScoreJob {
  const CNN_GLOBAL void* x;         // [rows] of [classes], `stride` elements apart
  const CNN_GLOBAL int* labels;     // [rows], or null; outside [0, classes): the row has none
  CNN_GLOBAL float* log_probs;      // [rows], or null
  CNN_GLOBAL float* entropy;        // [rows], or null
  CNN_GLOBAL float* normaliser;     // [rows][2], or null
  CNN_GLOBAL int* top;              // [rows][n_top], or null
  CNN_GLOBAL float* top_log_probs;  // [rows][n_top], or null
  CNN_GLOBAL unsigned long long* part_best;  // [rows][parts][n_top]   (parts > 1)
  CNN_GLOBAL float* part_sums;               // [rows][parts][4]
  long long rows, stride;
  int classes, type, n_top;
  int parts, part_tiles;            // workgroups that share a row, tiles of each
};

struct ScoreGradJob {
  const CNN_GLOBAL void* x;
  CNN_GLOBAL void* grad;            // [rows] of [classes], `grad_stride` elements apart
  const CNN_GLOBAL int* labels;
  const CNN_GLOBAL float* normaliser;
  const CNN_GLOBAL float* entropy;
  const CNN_GLOBAL float* g_log_probs;
  const CNN_GLOBAL float* g_entropy;
  long long rows, stride, grad_stride;
  int classes, type;
};

// ---- many tensors -------------------------------------------------------------------------------
constexpr int LIST_MOST = 128;     // tensors of one launch: the descriptor travels as a kernel argument (below 4 KB)
constexpr int LIST_CHUNK = 8192;   // elements that a workgroup takes at a time
constexpr int LIST_SUMS = 1024;    // workgroups of a call that leave a sum, at most, and one a launch more

struct TensorJob {
  const CNN_GLOBAL void* from[LIST_MOST];   // gradients
  CNN_GLOBAL void* to[LIST_MOST];           // what is written: clipped gradients, or weights (float)
  unsigned long long n[LIST_MOST];          // elements
  unsigned int chunk[LIST_MOST];            // first chunk of every tensor
  unsigned char type[LIST_MOST];
  int tensors;
  unsigned int chunks;                      // of all
  int first_sum, sums;                      // of this launch's workgroups; of all of them (where they are read)
};

}  // namespace cnn355
