// What the host side of the operators of a model's end (ops_api.hip) and their kernels share: argument blocks and
// launch functions.  Every launch goes to the caller's stream and allocates nothing.
#pragma once
#include "../../include/adapm.h"
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace adapm {

// sets the thread's error message and returns the code (adapm_api.hip)
adapm_status_t fail(adapm_status_t code, const char* fmt, ...);

// ---- dropout, norm (k_rowops.hip) ------------------------------------------------------------------------------------
struct DropDev {
  uint32_t k0, k1;               // key of the generator
  uint64_t offset;
  const uint64_t* offset_dev;    // added to offset where it is given
  uint32_t thr;                  // an element is kept if its 16 random bits are >= thr; 0: no dropout
  float scale;                   // 65536 / (65536 - thr)
};

struct Rows {                    // matrix of activations: row r starts at p + r * stride elements
  void* p;
  int64_t stride;
};

struct NormDev {
  int64_t rows;
  int cols;
  float eps;
  Rows x, residual, h, y;        // forward; residual.p, h.p may be null
  Rows dy, dh, dx, dres;         // backward; dh.p, dres.p may be null
  const void* weight;
  void* dweight;
  float* y_scale;                // e4m3 output
  float* rstd;
  float* partial;                // backward: [groups][cols]
  DropDev drop;
  int w_bf16, g_bf16, out8;      // types of weight and dweight; 8-bit output
};

void launch_dropout(bool bf16, Rows y, Rows x, Rows residual, int64_t rows, int64_t cols, const DropDev& d, hipStream_t s);
void launch_norm_forward(bool bf16, const NormDev& n, hipStream_t s);
// workgroups of the backward pass, each with one row of partial sums of dweight
int norm_backward_groups(int64_t rows, int64_t cols);
void launch_norm_backward(bool bf16, const NormDev& n, hipStream_t s);

// ---- loss over the vocabulary (k_head.hip) ---------------------------------------------------------------------------
// Workspace of one call, in bytes from its start; -1: absent
struct HeadLayout {
  int64_t head, counts, list, place, target, weight, lse;     // the rows that count (HeadHeader; int32 / float [rows])
  int64_t x, w;                                               // packed x [rows][pitch], packed W [vocab][pitch]
  int kind;                                                   // which tiles the products take
  int64_t part, hit, sums;                                    // forward: maxima and sums of the tiles, target logits, loss sums
  int tiles;                                                  // ... of which each row has so many
  int64_t p, acc;                                             // backward: a piece of P, sums of dx
  int64_t p_rows;                                             // ... rows of P, of packed x and of a part of dx that there is space for
  int64_t width;                                              // ... vocabulary rows of a piece
  int splits;                                                 // ... parts of dx's contraction over them
  bool dx_first;                                              // ... dx's tiles are given out before dW's
  int64_t bytes;
  int64_t threads;                                            // of the largest launch of the products
};

struct HeadDev {
  int64_t rows, vocab;
  int cols, pitch;               // pitch: elements of a row of packed x, whole steps of the contraction
  int bf16, mean;
  float scale;
  Rows x, w, dx, dw;             // dx.p, dw.p may be null
  const int64_t* targets;
  const float* row_weight;       // may be null
  const float* upstream;         // may be null
  float *loss, *row_loss, *lse;  // lse is read by the backward pass
  char* ws;
  HeadLayout lay;
  int w_packed;
  int direct;                    // forward: x is read where it is
  int whole;                     // x is read where it is if all of its rows count
  int twin_rows;                 // backward: P as two numbers if no more rows count
};

// backward: up to how many rows that count P is kept as two numbers
int head_twin_rows(bool bf16, bool weighted);

// whether a forward pass of so many rows reads x where it is, if x's rows are whole aligned vectors
bool head_direct(int64_t rows);
// whether a pass of so many rows does, if all of them count
bool head_whole(int64_t rows);

// backward: whether space for the gradients' pass is wanted (else the forward pass)
HeadLayout head_layout(int64_t rows, int64_t vocab, int64_t cols, bool bf16, bool w_packed, bool backward, bool want_dx, int twin_rows);
void launch_head_loss(const HeadDev& h, hipStream_t s);
void launch_head_backward(const HeadDev& h, hipStream_t s);

}  // namespace adapm
