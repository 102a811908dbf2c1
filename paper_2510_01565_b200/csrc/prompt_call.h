// dit_prompt_attention for a caller that allocates the workspace itself: the batch is laid out once per call, not once for the size of the workspace
// and once for the launch (up to 17 us each where long pairs are cut).  Internal to this repository; not part of the C ABI.
#pragma once
#include "../../include/dit_ops.h"

namespace dit {

// args' workspace is not looked at.  room(context, bytes) is called at most once, when every argument is in order and bytes > 0, and returns 16-byte
// aligned device memory; an exception that it throws leaves this function.
dit_status prompt_attention_in(const dit_prompt_attention_args& args, void* (*room)(void* context, size_t bytes), void* context, void* stream);

}  // namespace dit
