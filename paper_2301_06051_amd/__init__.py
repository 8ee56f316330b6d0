"""MI355X-native Dynamic Sparse Window Attention (DSVT, arXiv 2301.06051).

The package is a thin binding over libdsvt.so (hand-written HIP for gfx950); see binding.py.
"""
from .binding import (  # noqa: F401
    DsvtError, LayerNorm, LayerWeights, PoolWeights, SetMaps, SetMapsXY, SetMha, Vfe, dsvt_vfe, dsvt_vfe_workspace_size, dsvt_set_attention_workspace_size, dsvt_attn_pool, dsvt_attn_pool_static, dsvt_attn_pool_workspace_size, dsvt_bev_scatter, dsvt_block,
    dsvt_block_workspace_size, dsvt_partition, dsvt_partition_bound, dsvt_partition_xy, dsvt_partition_xy_multi, dsvt_set_attention, lib, part_cfg,
    dsvt_layer_norm, dsvt_layer_norm_backward, dsvt_layer_norm_backward_workspace_size, dsvt_rel_buckets, dsvt_set_mha, dsvt_set_mha_backward,
    dsvt_set_mha_backward_workspace_size,
    prof_collect, prof_enable)
