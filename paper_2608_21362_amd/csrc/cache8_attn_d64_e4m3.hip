// The attention kernels of kvb_cache8_attn for head size 64 and e4m3 codes (a translation unit of
// their own: there are 24 of them).
#include "cache8_attn_kernels.h"

namespace kvb {

void attn8_d64_e4m3(const Attn8Plan& plan, const Attn8& a, int block_len, float* po, float* ml, float* parts,
               hipStream_t s) {
  launch_kernels<64, KVB_E4M3>(plan, a, block_len, po, ml, parts, s);
}

}  // namespace kvb
