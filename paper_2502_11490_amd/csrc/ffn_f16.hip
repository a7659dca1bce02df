// The fp16 products of the gated feed-forward block.
#include "ffn_mfma16.h"

namespace gmpgr {
template int launch_ffn16<ANN_F16>(const FfnProduct &, int, hipStream_t);
}
