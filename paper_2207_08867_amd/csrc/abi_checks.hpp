// abi_checks.hpp -- argument checks that the entry points on low-precision tensors and on rows of
// logits share.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/mcf.h"

namespace {

constexpr int MAX_NC = 4;

int64_t elem_size(int dtype) { return dtype == MCF_F32 ? 4 : 2; }

bool overlap(const void *a, int64_t abytes, const void *b, int64_t bbytes) {
  if (!a || !b || abytes <= 0 || bbytes <= 0) return false;
  const uintptr_t a0 = (uintptr_t)a, b0 = (uintptr_t)b;
  return a0 < b0 + (uintptr_t)bbytes && b0 < a0 + (uintptr_t)abytes;
}

bool aligned(const void *p, uintptr_t to) { return (uintptr_t)p % to == 0; }

// a * b stays below 2^50, so byte counts and offsets never overflow int64; a, b >= 0.
bool elems_fit(int64_t a, int64_t b) { return b == 0 || a <= ((int64_t)1 << 50) / b; }

int hip_status(hipError_t e) { return e == hipSuccess ? MCF_OK : MCF_E_HIP; }

bool plain_format(int dtype) { return dtype == MCF_F16 || dtype == MCF_BF16 || dtype == MCF_F32; }

bool nc_ok(int nc) { return nc >= 1 && nc <= MAX_NC; }

struct Span {
  const void *p;
  int64_t bytes;
};

// Whether any of the outputs overlaps an input or another output.
template <int NO, int NI>
bool outputs_overlap(const Span (&outs)[NO], const Span (&ins)[NI]) {
  for (int o = 0; o < NO; ++o) {
    for (int i = 0; i < NI; ++i)
      if (overlap(outs[o].p, outs[o].bytes, ins[i].p, ins[i].bytes)) return true;
    for (int p = o + 1; p < NO; ++p)
      if (overlap(outs[o].p, outs[o].bytes, outs[p].p, outs[p].bytes)) return true;
  }
  return false;
}

int workspace_check(const void *workspace, int64_t given, int64_t needed) {
  if (needed <= 0) return MCF_OK;
  if (!workspace) return MCF_E_NULL;
  if (given < needed || !aligned(workspace, 16)) return MCF_E_ARG;
  return MCF_OK;
}

}  // namespace
