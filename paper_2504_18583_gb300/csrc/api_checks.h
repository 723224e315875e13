// What the C entries of the operators on caller-owned memory check and report alike.
#pragma once

#include <cmath>
#include <exception>
#include <string>

#include "pard.h"
#include "tree.h"

namespace pard {
void set_error(const std::string& msg);  // api.cu

namespace {

pard_status refuse(pard_status code, const char* why) {
  set_error(why);
  return code;
}

template <typename F>
pard_status launched(F&& f) {
  try {
    f();
    return PARD_OK;
  } catch (cudaError_t e) {
    set_error(std::string("kernel launch: ") + cudaGetErrorString(e));
  } catch (const std::exception& e) {
    set_error(e.what());
  }
  return PARD_ERR_CUDA;
}

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
bool two_byte(int dtype) { return dtype == DT_BF16 || dtype == DT_F16; }

// the paged cache's shape; pages of `page_stride` entries hold [head][16][head_dim]
const char* bad_cache(int n_kv_heads, int head_dim, int64_t page_stride, int n_pages) {
  if (head_dim != 64 && head_dim != 128) return "head_dim must be 64 or 128";
  if (n_kv_heads < 1 || n_kv_heads > 1024) return "key/value heads outside [1, 1024]";
  if (n_pages < 1) return "the cache has no pages";
  if (page_stride < (int64_t)n_kv_heads * kPageTok * head_dim) return "pages overlap: page stride too small";
  if (page_stride % 8) return "page stride must be a multiple of 8 entries";
  return nullptr;
}

}  // namespace
}  // namespace pard
