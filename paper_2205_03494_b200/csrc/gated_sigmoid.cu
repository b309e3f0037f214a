// The gated layer's backward kernels for one activation.
#include "gated.cuh"

int omc::gate::backward_sigmoid(const Backward &c) { return backward<OMC_GATE_SIGMOID>(c); }
