// Attention over pages (attend_rows.h): 8-bit pools.
#include "attend_rows.h"

namespace rkv {

int launch_attend8(const AttendLaunch& A, void* stream) { return launch_codes<false>(A, stream); }

}  // namespace rkv
