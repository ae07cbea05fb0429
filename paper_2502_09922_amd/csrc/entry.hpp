// How an entry point of include/ls_stage.h that is not a stage's answers.
#pragma once
#include "../../include/ls_stage.h"
#include "kernels.hpp"

namespace ls {

inline ls_status bad(const char* who, const char* what) {
  set_last_error("%s: %s", who, what);
  return LS_ERR_INVALID_ARG;
}

// Behind the launches of a call.
inline ls_status launched(const char* who) {
  const hipError_t e = hipGetLastError();
  if (e == hipSuccess) return LS_OK;
  set_last_error("%s: %s", who, hipGetErrorString(e));
  return LS_ERR_HIP;
}

// What is wrong with the argument, or null.
const char* heads_error(const ls_heads* h);
const char* tree_error(const ls_tree* t, int batch, int max_batch, bool with_parents, int* rows, int* min_nodes, int* max_nodes);  // min_nodes: of the trees that have any

}  // namespace ls
