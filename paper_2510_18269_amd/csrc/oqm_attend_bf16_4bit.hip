// The folded attention over codes of 4 bits with queries and rows of bf16.
#include "oqm_attend_folded.h"

namespace oqm {

void start_attend_bf16_4bit(const AttendArgs& g, const AttendForm& form, hipStream_t s) { start_folded_of<In_bf16, 4>(g, form, s); }

}  // namespace oqm
