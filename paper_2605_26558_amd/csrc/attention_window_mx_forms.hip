// Attention within a window (attention_rows.hip): exact form over a cache with shared exponents.
#include "attention_rows_kernel.inl"

namespace cas {
template int launch_rows_partial<true, true, RowsWindowArgs>(cas_ctx*, const RowsWindowArgs&, int, int);
}  // namespace cas
