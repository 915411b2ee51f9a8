// Attention over runs of pages (attention_rows.hip): draft form over a cache with raw exponents.
#include "attention_rows_kernel.inl"

namespace cas {
template int launch_rows_partial<false, false>(cas_ctx*, const RowsArgs&, int, int);
}  // namespace cas
