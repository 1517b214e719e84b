// The folded attention over codes of 2 bits with queries and rows of f16.
#include "oqm_attend_folded.h"

namespace oqm {

void start_attend_f16_2bit(const AttendArgs& g, const AttendForm& form, hipStream_t s) { start_folded_of<In_f16, 2>(g, form, s); }

}  // namespace oqm
