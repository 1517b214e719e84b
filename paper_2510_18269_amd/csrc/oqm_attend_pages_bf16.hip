// The attention over pages with queries and rows of bf16.
#include "oqm_attend_pages_few.h"
#include "oqm_attend_pages_many.h"

namespace oqm {

void start_attend_pages_bf16(const PagesArgs& g, const PagesForm& form, hipStream_t s) {
    if (form.block_rows == 16) start_pages_few<In_bf16>(g, s);
    else start_pages_many<In_bf16>(g, form, s);
}

}  // namespace oqm
