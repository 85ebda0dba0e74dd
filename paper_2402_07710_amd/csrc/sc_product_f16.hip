// The product kernels on f16 rows.
#include "sc_product.h"

namespace sc {
int launch_product_f16(int mode, const Product& p, int cus, hipStream_t s) { return launch_product<SC_F16>(mode, p, cus, s); }
}  // namespace sc
