// Tensor-core products of the linear layers (nf_gemm.cu).
#pragma once
#include "nf_internal.h"

// What happens to the sum at (p, q): bias and residual are added in fp32, every stored value is rounded once
struct Epilogue {
  const float* bias;     // [Q] or NULL
  const void* residual;  // [P][Q] or NULL
  int act;
  void* pre;             // [P][Q] or NULL: the value before the activation
  void* out;             // [P][Q]
  int out_f32;           // out is float whatever the operands' type
};

// C[p][q] = sum over r of A(p, r) B(q, r), bf16 operands; `planes` parts (1, or 3 whose sum is an fp32 operand), `plane` elements apart
struct GemmOperand {
  const bf16* base;
  size_t ld;      // elements between rows, a multiple of 8
  size_t plane;
  bool along_r;   // rows run along r (row p at base + p ld); else along p / q (row r at base + r ld)
};
struct GemmProblem {
  GemmOperand A, B;
  int P, Q, R, planes;
  int out_f32;    // C in fp32: the sums leave the tensor core in short segments
};
// splits of r that nf_gemm_tc makes (1: the epilogue is applied; more: partial sums go to part[split][P][Q])
int nf_gemm_splits(int P, int Q, int R, int planes);
int nf_gemm_tc(const GemmProblem& g, const Epilogue& e, float* part);
