// The kernels of odb_paged_attention_quant for E4M3 codes.
#include "paged_attn_quant.h"

namespace odb {

void launch_paged_attention_e4m3(const PagedAttnQuant &a, int nt, hipStream_t s) { launch_quant_codes<ODB_E4M3>(a, nt, s); }

}  // namespace odb
