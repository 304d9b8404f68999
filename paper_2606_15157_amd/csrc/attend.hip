// Attention over pages (attend_rows.h): 16-bit pools.
#include "attend_rows.h"

namespace rkv {

int launch_attend(const AttendLaunch& A, void* stream) { return launch_rows<false>(A, stream); }

}  // namespace rkv
