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

constexpr int OUT_SUMS = 2;   // batched forward pass, in the place of CNN_OUTPUT_*: the output layer's sums, without units

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
constexpr int LIST_MOST = 120;     // tensors of a kernel's argument (below 4 KB)
constexpr int LIST_FEW = 16;       // tensors of a smaller one
constexpr int LIST_CHUNK = 16384;  // bytes: gradients are cut into chunks of so many
constexpr int LIST_SUMS = 1024;    // workgroups that leave a sum, at most

struct TensorEntry {
  const CNN_GLOBAL void* from;     // gradients
  CNN_GLOBAL void* to;             // what is written: clipped gradients, or weights (float)
  unsigned long long n;            // elements, at least one
  unsigned int chunk;              // its first chunk among those of all tensors
  int type;
};
struct TensorHead {
  const CNN_GLOBAL TensorEntry* table;   // where they do not fit in `e`
  int tensors;
  unsigned int chunks;             // of all tensors
  int sums;                        // workgroups that leave a sum
  const CNN_GLOBAL int* label;     // null, or of the image that the gradients are of: outside [0, classes) it is passed over
  int classes;
};
template <int N>
struct TensorsOf : TensorHead {
  static constexpr int MOST = N;
  TensorEntry e[N];
};
typedef TensorsOf<LIST_MOST> TensorJob;
typedef TensorsOf<LIST_FEW> TensorJobFew;   // (a launch of a small argument takes the host less)

}  // namespace cnn355
