// Attention over pages (attend_dealt.h): 8-bit pools whose sequences share prefixes.
#include "attend_dealt.h"

namespace rkv {

int launch_attend8_shared(const AttendLaunch& A, void* stream) {
  hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  by_scores(A, [&](auto f16, auto cap, auto bias) {
    if (dense_codes(A)) launch_dealt<f16.value, cap.value, bias.value, kCodes8, true>(A, st);
    else launch_dealt<f16.value, cap.value, bias.value, kCodes, true>(A, st);
  });
  return (int)hipGetLastError();
}

}  // namespace rkv
