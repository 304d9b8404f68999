// Attention over pages (attend_rows.h): 8-bit pools whose sequences share prefixes.
#include "attend_rows.h"

namespace rkv {

int launch_attend8_shared(const AttendLaunch& A, void* stream) { return launch_codes<true>(A, stream); }

}  // namespace rkv
