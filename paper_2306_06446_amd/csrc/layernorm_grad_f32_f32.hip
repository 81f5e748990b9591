// The gradient of LayerNorm: kernels of one pair of row types.
#include "layernorm_grad.h"

template int sa::launch_norm_grad_rows<float, float>(const NormGradArgs &, int *, hipStream_t);
