// Instantiations of the attention of a few rows over another sequence's states.
#include "tir_cross_token.h"
#include "tir_host.h"
#include "tir_launch.h"

namespace tir {

template <int DT, int DH> static hipError_t launch_rows(const CrossParams& p, hipStream_t stream) {
    const dim3 grid((unsigned)p.batch, (unsigned)p.slices), block(kTokenWaves * 64);
    if (!grid_fits(p.batch, kTokenWaves * 64)) return hipErrorInvalidConfiguration;
    if (p.M == 1) return launch_kernel(&cross_token_kernel<DT, DH, 1>, grid, block, stream, p);
    if (p.M == 2) return launch_kernel(&cross_token_kernel<DT, DH, 2>, grid, block, stream, p);
    if (p.M == 3) return launch_kernel(&cross_token_kernel<DT, DH, 3>, grid, block, stream, p);
    if (p.M == 4) return launch_kernel(&cross_token_kernel<DT, DH, 4>, grid, block, stream, p);
    return hipErrorInvalidValue;
}
hipError_t launch_cross_token(const CrossParams& p, int dt, int dh, hipStream_t stream) {
    if (dt == DT_F16) return dh == 64 ? launch_rows<DT_F16, 64>(p, stream) : launch_rows<DT_F16, 128>(p, stream);
    return dh == 64 ? launch_rows<DT_BF16, 64>(p, stream) : launch_rows<DT_BF16, 128>(p, stream);
}

}  // namespace tir
