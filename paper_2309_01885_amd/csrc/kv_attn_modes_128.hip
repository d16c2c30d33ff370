// Attention over the 4-bit cache with first tokens that stay visible, and by lists: heads padded to 128 channels.
#include "kv_attn_modes.h"

namespace qe {
template void kv_sinks_width<128>(const KvAttn&, const KvPlan&, KvForm, dim3, hipStream_t);
template void kv_listed_width<128>(const KvAttn&, const KvPlan&, const KvShared&, KvForm, KvForm, hipStream_t);
}
