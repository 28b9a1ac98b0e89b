"""B200 (sm_100a) implementation of VarDrop's per-batch training path behind a C ABI (see include/vardrop.h).

``binding`` holds the ctypes front end (same names as the C entry points), ``inputs`` the seeded synthetic
workloads, ``build`` the nvcc build step.
"""
from . import binding, inputs  # noqa: F401
from .binding import (ActCfg, AttnCfg, ClipCfg, EmbedCfg, HashCfg, LossCfg, NormCfg, PackedCfg, SelectCfg, VardropError, vardrop_attn_bwd, vardrop_attn_fwd,  # noqa: F401
                      vardrop_attn_packed_bwd, vardrop_attn_packed_fwd, vardrop_attn_packed_workspace_bytes, vardrop_packed_plan, vardrop_packed_plan_bytes,
                      vardrop_attn_workspace_bytes, vardrop_grad_clip, vardrop_grad_clip_workspace_bytes, vardrop_hash, vardrop_hash_workspace_bytes, vardrop_norm_bwd, vardrop_norm_fwd,
                      vardrop_norm_workspace_bytes, vardrop_select, vardrop_embed_fwd, vardrop_embed_bwd, vardrop_embed_workspace_bytes, vardrop_act_fwd, vardrop_act_bwd, vardrop_act_ckpt_bytes,
                      vardrop_loss_fwd, vardrop_loss_bwd, vardrop_loss_workspace_bytes,
                      vardrop_select_workspace_bytes)
