// The selective scan's gradient in one format.
#include "selective_grad_launch.h"

namespace pg {

template hipError_t selective_grad<BF16>(const SelCall&, const SelPlan&, const Launch&);

}  // namespace pg
