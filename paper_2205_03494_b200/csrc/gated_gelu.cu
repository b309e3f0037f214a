// The gated layer's backward kernels for one activation.
#include "gated.cuh"

int omc::gate::backward_gelu(const Backward &c) { return backward<OMC_GATE_GELU>(c); }
