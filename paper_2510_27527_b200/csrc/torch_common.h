// What the translation units of the Python module `_node` share: outputs, and library errors as the binding's exceptions.
#pragma once
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <ATen/ATen.h>

#include "../../include/nvfp4.h"

namespace nvfp4_torch {

constexpr int64_t up(int64_t n, int64_t to) { return (n + to - 1) / to * to; }

// Row-major matrix whose rows start on 16-byte boundaries. (Not a tracked view of its buffer: a result of its own.)
inline at::Tensor matrix(int64_t rows, int64_t cols, const at::TensorOptions& opt) {
  const int64_t ld = up(cols, 8);
  at::Tensor t = at::empty({rows, ld}, opt);
  if (ld == cols) return t;
  at::AutoDispatchBelowADInplaceOrView below;
  return t.narrow(1, 0, cols);
}

// Status of a library call, as the exception that the binding raises for it.
[[noreturn]] void raise_status(nvfp4_status status, const char* where);

// The calls around the linears (torch_calls.cpp).
extern PyMethodDef block_methods[];

}  // namespace nvfp4_torch
