// What the handle's calls (tabed.cu) use of the paged caches (pages.cu).
#pragma once
#include <cuda_runtime.h>

#include "../../include/tabed.h"

namespace tabed {

// A row of a handle's dense caches: k and v at its beginning, [L][Hkv][cap][hd] floats or bf16 values; its committed length (on the device).
struct DenseRow { void *k, *v; int cap; bool f32; int* len; };

// Whether the caches are those of a drafter of these sizes (TABED_OK, or why not).
int pages_match(const tabed_pages* p, int L, int Hkv, int hd, int device);
// Positions start .. start + len - 1 of the row to the same ones of the sequence, if the row has them; the first len tokens of the sequence to the
// row, and len to its length.  Kernels launched are added to *launches.
int pages_store_row(const tabed_pages* p, cudaStream_t stream, const DenseRow& r, int seq, int start, int len, int64_t* launches);
int pages_load_row(const tabed_pages* p, cudaStream_t stream, const DenseRow& r, int seq, int len, int64_t* launches);

}  // namespace tabed
