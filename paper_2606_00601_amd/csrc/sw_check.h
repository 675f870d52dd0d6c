// sw_check.h -- argument checks shared by the C-ABI layers (not installed).
#pragma once

#include <string.h>

#include <initializer_list>

#include "sw_internal.h"

namespace sw {

struct Span {
  const void* p;
  size_t bytes;
  const char* name;
};

inline bool overlaps(const Span& a, const Span& b) {
  if (!a.p || !b.p || a.bytes == 0 || b.bytes == 0) return false;
  const uintptr_t a0 = (uintptr_t)a.p, b0 = (uintptr_t)b.p;
  return a0 < b0 + b.bytes && b0 < a0 + a.bytes;
}

// Multiply non-negative sizes; false on overflow of int64.
inline bool mul_ok(int64_t a, int64_t b, int64_t* out) { return !__builtin_mul_overflow(a, b, out); }

inline int check_ptr(const void* p, size_t align, const char* name, bool required, int device) {
  if (!p) {
    if (required) return fail(SW_ERR_INVALID_ARG, "%s is NULL", name);
    return SW_OK;
  }
  if ((uintptr_t)p % align != 0)
    return fail(SW_ERR_INVALID_ARG, "%s is not %zu-byte aligned", name, align);
  hipPointerAttribute_t attr;
  memset(&attr, 0, sizeof(attr));
  hipError_t e = hipPointerGetAttributes(&attr, p);
  if (e != hipSuccess) {
    (void)hipGetLastError();  // the query failure is not a sticky launch error
    return fail(SW_ERR_INVALID_ARG, "%s is not device memory (%s)", name, hipGetErrorString(e));
  }
  if (attr.type != hipMemoryTypeDevice && attr.type != hipMemoryTypeManaged &&
      attr.type != hipMemoryTypeUnified)
    return fail(SW_ERR_INVALID_ARG, "%s is not device memory (memory type %d)", name,
                (int)attr.type);
  if (attr.device != device)
    return fail(SW_ERR_INVALID_ARG, "%s lives on device %d, current device is %d", name,
                attr.device, device);
  return SW_OK;
}

inline int current_device(int* dev) {
  hipError_t e = hipGetDevice(dev);
  if (e != hipSuccess) return fail(SW_ERR_HIP, "hipGetDevice: %s", hipGetErrorString(e));
  return SW_OK;
}

inline int check_spans(const Span* outs, int nout, const Span* ins, int nin) {
  for (int i = 0; i < nout; ++i) {
    for (int j = 0; j < nin; ++j)
      if (overlaps(outs[i], ins[j]))
        return fail(SW_ERR_INVALID_ARG, "output %s overlaps input %s", outs[i].name,
                    ins[j].name);
    for (int j = i + 1; j < nout; ++j)
      if (overlaps(outs[i], outs[j]))
        return fail(SW_ERR_INVALID_ARG, "outputs %s and %s overlap", outs[i].name,
                    outs[j].name);
  }
  return SW_OK;
}

inline bool all_aligned16(std::initializer_list<const void*> ps) {
  for (const void* p : ps)
    if (p && (uintptr_t)p % 16 != 0) return false;
  return true;
}

}  // namespace sw
