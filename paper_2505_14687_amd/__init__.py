"""GRAT grouped sparse attention for AMD MI355X: Python binding over the libgrat C ABI."""
from .grat import (GratError, grat_attention_fwd, grat_attention_global_fwd, grat_attention_packed_fwd,
                   grat_block_list_shape, grat_build_block_lists, grat_dense_attention_fwd,
                   grat_validate_block_lists, lib)
from .probe import grat_probe_mfma
from .sequence import (grat_block_means, grat_block_scores, grat_rotary, grat_rotary_append, grat_rotary_table,
                       grat_select_blocks, grat_selected_attention_bwd, grat_selected_attention_fwd)

__all__ = ["GratError", "grat_attention_fwd", "grat_attention_global_fwd", "grat_attention_packed_fwd",
           "grat_block_list_shape", "grat_block_means", "grat_block_scores", "grat_build_block_lists",
           "grat_dense_attention_fwd", "grat_probe_mfma", "grat_rotary", "grat_rotary_append", "grat_rotary_table",
           "grat_select_blocks", "grat_selected_attention_bwd", "grat_selected_attention_fwd", "grat_validate_block_lists", "lib"]
