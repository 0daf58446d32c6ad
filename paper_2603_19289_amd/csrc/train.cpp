// The text of the last failure of the training operators, one per thread.
#include "train_common.h"

namespace moe_spec {
namespace { thread_local char g_train_error[256] = ""; }

int train_fail(int code, const char *fmt, ...) {
  va_list args;
  va_start(args, fmt);
  vsnprintf(g_train_error, sizeof(g_train_error), fmt, args);
  va_end(args);
  return code;
}

}  // namespace moe_spec

extern "C" const char *moe_spec_train_last_error(void) { return moe_spec::g_train_error; }
