// Argument checks that the C ABI files share (each a copy of its own: internal linkage).
#pragma once
#include <cstdarg>
#include <cstdio>

#include "../../include/hla.h"
#include "common.h"
#include "mixer.h"

namespace hla {
int api_fail(int code, const char* msg);
}

namespace {

int fail(int code, const char* fmt, ...) {
  char msg[512];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(msg, sizeof(msg), fmt, ap);
  va_end(ap);
  return hla::api_fail(code, msg);
}

int done(hipError_t e, const char* what) {
  if (e != hipSuccess) return fail(HLA_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
  return hla::api_fail(HLA_OK, "");
}

int esize(int dtype) { return dtype == HLA_BF16 ? 2 : 4; }

int check_type(int dtype, const char* name) {
  if (dtype != HLA_FP32 && dtype != HLA_BF16) return fail(HLA_ERR_INVALID, "%s must be HLA_FP32 or HLA_BF16", name);
  return HLA_OK;
}

int check_flag(int f, const char* name) {
  if (f != 0 && f != 1) return fail(HLA_ERR_INVALID, "%s must be 0 or 1", name);
  return HLA_OK;
}

bool aligned(const void* p, unsigned a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

// A tensor whose elements are read one by one (weights, tables): its own alignment.
int check_own(const void* p, unsigned a, const char* name, bool need = true) {
  if (!p) return need ? fail(HLA_ERR_INVALID, "%s is NULL", name) : HLA_OK;
  if (!aligned(p, a)) return fail(HLA_ERR_INVALID, "%s is not %u-byte aligned", name, a);
  return HLA_OK;
}
int check_16(const void* p, const char* name, bool need = true) { return check_own(p, 16, name, need); }

// The strides of dimensions of size one are not used, whatever they are.
void drop_unused(hla::Rows& r, int B, int n) {
  if (B == 1) r.bs = 0;
  if (n == 1) r.ts = 0;
}

int check_stride(long long bs, long long ts, const char* name) {
  if (bs < 0 || ts < 0) return fail(HLA_ERR_INVALID, "%s: strides must be >= 0 (got %lld, %lld)", name, bs, ts);
  return HLA_OK;
}

// Rows read in 16-byte pieces: the base and both strides in whole pieces.
int check_rows(const hla::Rows& r, int dtype, const char* name) {
  int rc;
  if ((rc = check_16(r.p, name)) || (rc = check_stride(r.bs, r.ts, name))) return rc;
  const int v = 16 / esize(dtype);
  if (r.bs % v || r.ts % v)
    return fail(HLA_ERR_INVALID, "%s: strides must be whole 16-byte pieces (got %lld, %lld elements)", name, r.bs, r.ts);
  return HLA_OK;
}

int check_ws(const void* ws, size_t have, size_t need) {
  if (!ws || have < need) return fail(HLA_ERR_WORKSPACE, "workspace of %zu bytes needed, %zu given", need, have);
  return check_16(ws, "workspace");
}

}  // namespace
