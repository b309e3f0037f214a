// The gated layer's backward kernels for one activation.
#include "gated.cuh"

int omc::gate::backward_silu(const Backward &c) { return backward<OMC_GATE_SILU>(c); }
