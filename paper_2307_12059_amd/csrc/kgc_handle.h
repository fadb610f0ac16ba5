// What the operators on embedding tables (kgc_embed.hip) see of a handle: its settings, its stream, its error message.
#pragma once
#include <hip/hip_runtime.h>

#include "../../include/kgc.h"

namespace kgc {

struct HandleView {
  int dtype, max_d, device;
  hipStream_t stream;
};

#define KGC_HIDDEN __attribute__((visibility("hidden")))
KGC_HIDDEN HandleView handle_view(const kgc_handle* hd);
KGC_HIDDEN int handle_fail(kgc_handle* hd, int code, const char* what, hipError_t e = hipSuccess);
KGC_HIDDEN void handle_clear(kgc_handle* hd);

}  // namespace kgc
