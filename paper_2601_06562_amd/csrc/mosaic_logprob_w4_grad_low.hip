// The same with low halves (mosaic_logprob_w4.h).
#include "mosaic_logprob_w4.h"

namespace mosaic {
namespace logprob {

int launch_gradients_low_w4(const LogitParams& p, hipStream_t stream) {
  LogitParams g = p;
  g.sched.slots64 = INT32_MAX;   // no parts' arrays
  return launch<kGradientsLow>(g, stream);
}

}  // namespace logprob
}  // namespace mosaic
