// The kernels of fp8lin_ffn.h for kEpiAct (files of their own: they build side by side).
#include "fp8lin_ffn.h"

namespace fp8lin {

void launch_ffn_act(bool ragged, const Epi& e, hipStream_t s) { launch_mode<kEpiAct>(ragged, e, s); }

}  // namespace fp8lin
