// Shared by the operators over a paged cache: argument checks and cache addressing.
#pragma once
#include "common.h"
#include "status.h"

namespace atspeed {

constexpr int kMaxRequests = 1024;
// Workgroups of 256 threads of a launch: it holds fewer than 2^32 threads.
constexpr long long kMaxGroups = (1LL << 24) - 1;

// The device's view of atspeed_pages: element offsets, page size as a shift.
struct PagesDev {
  const char* data;
  int64_t page, token, head;   // bytes
};

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
inline int log2_of(int x) { return __builtin_ctz((unsigned)x); }

inline PagesDev pages_dev(const atspeed_pages& p, int es) {
  return {static_cast<const char*>(p.data), p.page_stride * es, p.token_stride * es, p.head_stride * es};
}

inline atspeed_status check_paging(int page_size, int n_pool) {
  if (page_size < 1 || page_size > 1024 || (page_size & (page_size - 1)))
    return fail(ATSPEED_E_INVALID, "page_size must be a power of two up to 1024");
  if (n_pool < 1) return fail(ATSPEED_E_INVALID, "n_pool must be >= 1");
  if ((long long)page_size * n_pool >= (1LL << 31)) return fail(ATSPEED_E_SHAPE, "page_size x n_pool must be below 2^31");
  return ATSPEED_OK;
}

inline atspeed_status check_head(int dtype, int d_head) {
  if (dtype != ATSPEED_FP32 && dtype != ATSPEED_BF16) return fail(ATSPEED_E_INVALID, "dtype");
  const bool ok = d_head == 64 || d_head == 128 || (d_head == 32 && dtype == ATSPEED_FP32);
  if (!ok) return fail(ATSPEED_E_SHAPE, "d_head must be 64 or 128 (bf16) or 32, 64 or 128 (fp32)");
  return ATSPEED_OK;
}

inline atspeed_status check_rows(const void* p, int64_t row, int64_t head, int es, const char* who) {
  if (!p) return fail(ATSPEED_E_INVALID, std::string(who) + " is null");
  if (!aligned16(p) || (row * es) % 16 || (head * es) % 16)
    return fail(ATSPEED_E_INVALID, std::string(who) + ": the data and its strides must be multiples of 16 bytes");
  return ATSPEED_OK;
}

inline atspeed_status check_pages(const atspeed_pages& p, int es, const char* who) {
  ST_TRY(check_rows(p.data, p.token_stride, p.head_stride, es, who));
  if ((p.page_stride * es) % 16) return fail(ATSPEED_E_INVALID, std::string(who) + ": the page stride must be a multiple of 16 bytes");
  return ATSPEED_OK;
}

}  // namespace atspeed
