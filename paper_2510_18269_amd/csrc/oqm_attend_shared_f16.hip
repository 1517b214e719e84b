// The attention over reconstructed tiles with queries and rows of f16.
#include "oqm_attend_shared.h"

namespace oqm {

void start_attend_shared_f16(const AttendArgs& g, hipStream_t s) { start_shared<In_f16>(g, s); }

}  // namespace oqm
