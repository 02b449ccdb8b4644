// Few rows, results in bf16.
#include "project_fp8_rows.h"

namespace dsla {
bool launch_fp8_rows(ProfileScope &ps, const Fp8Args &a, int N, int mt, int nt, bool e8m0, hipStream_t stream)
{
    return launch_few_of<false>(ps, a, N, mt, nt, e8m0, stream);
}
}  // namespace dsla
