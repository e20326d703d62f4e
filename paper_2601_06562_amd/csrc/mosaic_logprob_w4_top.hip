// The same with a row's most probable ids (mosaic_logprob_w4.h).
#include "mosaic_logprob_w4.h"

namespace mosaic {
namespace logprob {

int64_t w4_list_bytes() { return (int64_t)kCus * 4 * 64 * 8 * kListRoom * (int64_t)sizeof(Entry); }

int launch_alternatives_w4(const LogitParams& p, hipStream_t stream) { return launch<kAlternatives>(p, stream); }

}  // namespace logprob
}  // namespace mosaic
