// Attention over pages (attend_rows.h): 16-bit pools.
#include "attend_rows.h"

namespace rkv {

int launch_attend(const AttendLaunch& A, void* stream) {
  hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  by_scores(A, [&](auto f16, auto cap, auto bias) {
    if (pages_of_16(A)) launch_kernels<f16.value, cap.value, bias.value, kPages16>(A, st);
    else launch_kernels<f16.value, cap.value, bias.value, kAnyPages>(A, st);
  });
  return (int)hipGetLastError();
}

}  // namespace rkv
