// A KV cache in pages: what the kernels need of it.
#pragma once
#include "gsd_internal.cuh"

namespace gsd {

// The first entry outside [0, num_pages) among entries [first, end) of a sequence's row of the page table that the calling
// threads find, thread `at` of `step`; `end` if there is none among the thread's own.
__device__ __forceinline__ int first_bad_page(const int32_t* row, int first, int end, int num_pages, int at, int step) {
    for (int i = first + at; i < end; i += step)
        if ((unsigned)row[i] >= (unsigned)num_pages) return i;
    return end;
}

}  // namespace gsd
