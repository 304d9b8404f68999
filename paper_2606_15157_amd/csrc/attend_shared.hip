// Attention over pages (attend_rows.h): 16-bit pools whose sequences share prefixes.
#include "attend_rows.h"

namespace rkv {

int launch_attend_shared(const AttendLaunch& A, void* stream) { return launch_rows<true>(A, stream); }

}  // namespace rkv
