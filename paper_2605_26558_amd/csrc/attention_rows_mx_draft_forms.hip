// Attention over runs of pages (attention_rows.hip): draft form over a cache with shared exponents.
#include "attention_rows_kernel.inl"

namespace cas {
template int launch_rows_partial<false, true, RowsArgs>(cas_ctx*, const RowsArgs&, int, int);
}  // namespace cas
