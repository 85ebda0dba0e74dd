// The product kernels on bf16 rows.
#include "sc_product.h"

namespace sc {
int launch_product_bf16(int mode, const Product& p, bool whole, int cus, hipStream_t s) { return launch_product<SC_BF16>(mode, p, whole, cus, s); }
}  // namespace sc
