// The kernel with 4-bit weights for few rows of fp16 x.
#include "q4_few.h"

namespace ebag {

q4_fn pick_q4_few_f16(const Q4FewKind& k) { return pick_few<1>(k); }

}  // namespace ebag
