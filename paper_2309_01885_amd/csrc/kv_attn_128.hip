// Attention over the 4-bit cache: heads padded to 128 channels.
#include "kv_attn.h"

namespace qe {
template void kv_attn_width<128>(const KvAttn&, const KvPlan&, KvForm, dim3, hipStream_t);
}
