// The attention over reconstructed tiles with queries and rows of bf16.
#include "oqm_attend_shared.h"

namespace oqm {

void start_attend_shared_bf16(const AttendArgs& g, hipStream_t s) { start_shared<In_bf16>(g, s); }

}  // namespace oqm
