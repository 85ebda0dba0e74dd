// The product kernels on f32 rows.
#include "sc_product.h"

namespace sc {
int launch_product_f32(int mode, const Product& p, int cus, hipStream_t s) { return launch_product<SC_F32>(mode, p, cus, s); }
}  // namespace sc
