// The attention over pages with queries and rows of f16.
#include "oqm_attend_pages_few.h"

namespace oqm {

void start_attend_pages_f16(const PagesArgs& g, const PagesForm&, hipStream_t s) { start_pages_few<In_f16>(g, s); }

}  // namespace oqm
