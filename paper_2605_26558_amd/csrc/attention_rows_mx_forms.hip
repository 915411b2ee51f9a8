// Attention over runs of pages (attention_rows.hip): exact form over a cache with shared exponents.
#include "attention_rows_kernel.inl"

namespace cas {
template int launch_rows_partial<true, true, RowsArgs>(cas_ctx*, const RowsArgs&, int, int);
}  // namespace cas
