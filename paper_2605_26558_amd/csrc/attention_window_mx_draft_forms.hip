// Attention within a window (attention_rows.hip): draft form over a cache with shared exponents.
#include "attention_rows_kernel.inl"

namespace cas {
template int launch_rows_partial<false, true, RowsWindowArgs>(cas_ctx*, const RowsWindowArgs&, int, int);
}  // namespace cas
