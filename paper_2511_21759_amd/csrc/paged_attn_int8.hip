// The kernels of odb_paged_attention_quant for INT8 codes.
#include "paged_attn_quant.h"

namespace odb {

void launch_paged_attention_int8(const PagedAttnQuant &a, int nt, hipStream_t s) { launch_quant_codes<ODB_INT8>(a, nt, s); }

}  // namespace odb
