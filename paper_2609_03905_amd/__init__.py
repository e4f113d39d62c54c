"""One GPU's share of a block join-agg (Einsummable's "every kernel is a join")
on AMD MI355X.  The compute path is libea.so (hand-written HIP for gfx950,
C ABI in include/ea.h); this package is its Python binding."""
from .ea import (AGG_LSE, AGG_MAX, AGG_NONE, AGG_SUM, BF16, E4M3, E5M2, F16, F32, JOIN_ADD, JOIN_MUL, OP_ATTENTION,
                 OP_RMSNORM, OP_SOFTMAX, OP_SWIGLU, PAGED_MAX_SEQ, PAGES_NONE_FREE, PAGES_OK, PAGES_TOO_LONG, EAError,
                 Relation, attention_paged, attention_paged_workspace, from_dense, heads, heads_backward, join_tuples,
                 joinagg, joinagg_workspace, layout_nbytes, lib, new_workspace, overlay, pages_compact, pages_extend,
                 pages_read, pages_select, pages_workspace, pages_write, plan_cache_clear, plan_cache_size,
                 repartition, repartition_plan, to_dense,
                 version)
