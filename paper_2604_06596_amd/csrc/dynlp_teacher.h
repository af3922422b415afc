// A teacher of which each row keeps its first classes.
#pragma once

#include <stdint.h>

namespace dynlp {

struct Teacher {
    const int32_t* classes;  // rows x kept
    const float* logits;
    const float* row_weight; // or NULL
    int32_t* rejected;       // or NULL
    int kept, count;         // of a list; classes of the head
    float inverse;           // 1 / T
    float temperature;       // T
};

}  // namespace dynlp
