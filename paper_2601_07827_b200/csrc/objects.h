// The library objects that more than one translation unit looks into.
#pragma once

#include "plan.h"

struct btc_handle_s {
    int device = -1;       // -1: no CUDA device (objects can be validated and planned, not run)
    int sm_count = 148;
};

struct btc_tensor_info_s {
    btc::TensorDesc desc;
};
