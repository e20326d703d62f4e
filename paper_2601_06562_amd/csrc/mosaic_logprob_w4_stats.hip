// Log probabilities, entropies and log-sum-exps on the hand-scheduled K-loop (mosaic_logprob_w4.h).
#include "mosaic_logprob_w4.h"

namespace mosaic {
namespace logprob {

constexpr int kRaggedKTiles = 5;   // as the mask-only pass

bool w4_takes(int32_t d, int32_t V) {
  return d % kTileK == 0 && V >= kVocab && (V % kVocab == 0 || d / kTileK >= kRaggedKTiles) && (int64_t)kVocab * d * 2 < (int64_t)1 << 32;
}

int launch_statistics_w4(const LogitParams& p, hipStream_t stream) { return launch<kStatistics>(p, stream); }

}  // namespace logprob
}  // namespace mosaic
