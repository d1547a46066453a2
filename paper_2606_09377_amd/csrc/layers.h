// Shared by the entry points on layers' weights (layers.hip, orthogonalize.hip).  Not part of the C ABI.
#pragma once

#include "ctx.h"

// The context's room for a call on its current stream, at least so many bytes (nothing in it is
// kept from call to call).  Each stream has its own, so that calls on two streams share no memory; under the
// workspace cap, which is theirs together, idle ones of other streams are freed for it.
vcr_status op_space(vcr_ctx *c, size_t bytes, vcr_internal::Workspace **out);
// Before the first and after the last launch of a call
vcr_status op_begin(vcr_ctx *c);
vcr_status op_end(vcr_ctx *c);
vcr_status check_mat(vcr_ctx *c, const vcr_mat *m, const char *name);
vcr_status check_contraction(vcr_ctx *c, int64_t k);
