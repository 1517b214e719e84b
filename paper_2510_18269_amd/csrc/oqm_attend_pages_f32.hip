// The attention over pages with queries and rows of f32.
#include "oqm_attend_pages_few.h"

namespace oqm {

void start_attend_pages_f32(const PagesArgs& g, const PagesForm&, hipStream_t s) { start_pages_few<In_f32>(g, s); }

}  // namespace oqm
