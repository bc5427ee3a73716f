// naut_packed_inst.hip -- the kernels of packed sequences for one (input type, output type) pair and some head widths.
//
// Compiled once per pair and widths with the defines of naut_attn_inst.hip; naut_packed.hip declares these launchers extern.
#include "naut_attn_kernels.h"
#include "naut_packed_launch.h"

#if !defined(NAUT_INST_IN) || !defined(NAUT_INST_OUT) || !defined(NAUT_INST_W)  // a bare compile of this file
#undef NAUT_INST_IN
#undef NAUT_INST_OUT
#undef NAUT_INST_W
#define NAUT_INST_IN NAUT_BF16
#define NAUT_INST_OUT NAUT_BF16
#define NAUT_INST_W 128
#endif

namespace naut_k {

#if NAUT_INST_W == 64
template int launch_packed<64, NAUT_INST_IN, NAUT_INST_OUT>(PackedParams, int, hipStream_t);
#elif NAUT_INST_W == 96
template int launch_packed<80, NAUT_INST_IN, NAUT_INST_OUT>(PackedParams, int, hipStream_t);
template int launch_packed<96, NAUT_INST_IN, NAUT_INST_OUT>(PackedParams, int, hipStream_t);
#elif NAUT_INST_W == 128
template int launch_packed<128, NAUT_INST_IN, NAUT_INST_OUT>(PackedParams, int, hipStream_t);
#else
template int launch_packed<192, NAUT_INST_IN, NAUT_INST_OUT>(PackedParams, int, hipStream_t);
template int launch_packed<256, NAUT_INST_IN, NAUT_INST_OUT>(PackedParams, int, hipStream_t);
#endif

}  // namespace naut_k
