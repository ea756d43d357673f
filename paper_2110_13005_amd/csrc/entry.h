// What the files with C entry points share (defined in stage.cpp): the thread's error message and the launch timing.
#pragma once
#include "common.h"

namespace axonn {

// Categories of axonn_profile_*, in the order of their names (kProfNames).
enum ProfCat { PC_GEMM_FWD, PC_GEMM_DGRAD, PC_GEMM_WGRAD, PC_ATTN_FWD, PC_ATTN_BWD, PC_LN_FWD,
               PC_LN_BWD, PC_GRAD_CONVERT, PC_ADAM, PC_COPY_IN, PC_EMBED, PC_XENT, PC_QK_NORM, PC_DROPOUT, PC_FP8_QUANT,
               PC_GEMM_FP8, PC_COUNT };

// Sets the message of axonn_last_error and returns `code`.
int fail_entry(int code, const char* fmt, ...);

// Times what is launched on `stream` during its life, while timing is on.
class LaunchTiming {
 public:
  LaunchTiming(ProfCat category, hipStream_t stream);
  ~LaunchTiming();
  LaunchTiming(const LaunchTiming&) = delete;

 private:
  void* scope;
};

}  // namespace axonn
