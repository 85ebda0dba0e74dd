// The product kernels on bf16 rows.
#include "sc_product.h"

namespace sc {
int launch_product_bf16(int mode, const Product& p, int cus, hipStream_t s) { return launch_product<SC_BF16>(mode, p, cus, s); }
}  // namespace sc
