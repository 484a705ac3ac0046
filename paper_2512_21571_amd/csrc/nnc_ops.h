// Host-side pieces that the C entry points of nnc_api.hip and nnc_ops.hip share.
#pragma once
#include "../../include/nnc.h"
#include "nnc_pages.h"

namespace nnc {

// Record the message of nnc_last_error and hand the status back.
nnc_status fail(nnc_status st, const char* fmt, ...);
nnc_status dev_fail(hipError_t e, const char* what);

nnc_status check_pages(const nnc_pages* p);
// (of a pool that has passed check_pages)
nnc_status check_table(const nnc_pages* p, const nnc_page_table* t);
PagePool pool_layer(const nnc_pages* p, uint32_t layer);
nnc_status check_beams(uint32_t n_groups, uint32_t width);
PageReorder reorder_of(const nnc_pages* p, const nnc_page_table* before, int32_t* after, const int32_t* lens, const int32_t* parents,
                       uint32_t width);

}  // namespace nnc
