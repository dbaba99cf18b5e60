// Error text for a library of some of the sources (in the whole one fmha_varlen.hip holds it).
#include <cstdarg>
#include <cstdio>

#include "../../include/fmha_varlen.h"
#include "../../paper_2208_08124_amd/csrc/host_error.h"

namespace fmha_host {
thread_local char g_err[512] = "";
int fail(int code, const char* fmt, ...) {
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(g_err, sizeof(g_err), fmt, ap);
  va_end(ap);
  return code;
}
}  // namespace fmha_host
extern "C" const char* fmha_last_error(void) { return fmha_host::g_err; }
