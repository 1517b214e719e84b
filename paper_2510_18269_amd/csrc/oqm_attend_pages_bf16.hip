// The attention over pages with queries and rows of bf16.
#include "oqm_attend_pages_few.h"

namespace oqm {

void start_attend_pages_bf16(const PagesArgs& g, const PagesForm&, hipStream_t s) { start_pages_few<In_bf16>(g, s); }

}  // namespace oqm
