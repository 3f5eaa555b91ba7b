// gq_w4_matvec for activations in int8.
#include <hip/hip_runtime.h>
#include <stdint.h>
#include <stddef.h>

#include "gqsgd.h"
#include "matvec.hpp"

template gq_status gq::matvec<int8_t>(const gq::MatvecArgs &, int, int, hipStream_t);
