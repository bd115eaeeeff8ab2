// What the calls of attention over either cache share (token_api.hip): checks of the descriptor, its kernels' arguments, scratch, the launch.
#pragma once
#include "../../include/int8t.h"
#include "tokens.h"

namespace int8t {

int8t_status attend_desc_ok(const int8t_attend_desc* d, int heads, int page_size);
AttendArgs attend_args(const CacheArgs& c, const int8t_attend_desc* d, int mx);
size_t attend_bytes(const AttendArgs& a);
int8t_status attend_call(AttendArgs a, const int8t_attend_desc* desc, const void* q_dev, const int* starts_dev, const int* lengths_dev, const int* table_dev, void* out_dev,
                         float* lse_dev, void* ws_dev, size_t ws_bytes, void* stream);

}  // namespace int8t
