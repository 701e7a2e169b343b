// The inverted lists of an index: what both libraries read of it.
#pragma once
#include <stdint.h>

#include "internal.hpp"

struct IvfStore {
  IvfpqDims g{};
  int device = 0;
  float* centroids = nullptr;   // [nlist, d]
  float* codebooks = nullptr;   // [M, K, dsub]
  int64_t ntotal = 0;
  uint8_t* codes = nullptr;     // [ntotal, code_size], list-contiguous
  int64_t* ids = nullptr;       // [ntotal], behind codes
  int64_t* list_off = nullptr;  // device [nlist + 1]
  int64_t max_list = 0;         // the longest list's length
};
