// The kernels of fp8lin_ffn.h for kEpiGluBwd (files of their own: they build side by side).
#include "fp8lin_ffn.h"

namespace fp8lin {

void launch_ffn_glu_bwd(bool ragged, const Epi& e, hipStream_t s) { launch_mode<kEpiGluBwd>(ragged, e, s); }

}  // namespace fp8lin
