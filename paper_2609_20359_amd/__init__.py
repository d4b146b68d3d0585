"""MI355X-native parameter-sync path of FL+FSDP / FL+HSDP training.

One GPU's share of the method of "Accelerating Sharded Data Parallelism at
Scale with Federated Learning" (Section 4.2): the local arithmetic of the
gradient reduce-scatter, the AdamW step on the fp32 master shard, and the
FedAvg of the federation groups' replicas, as a C-ABI library (libflround.so,
include/flround.h) of hand-written gfx950 kernels; and the output head, where a
step's gradients begin: cross entropy, distillation from top logits, and their
gradients; the embedding and the layer norm with theirs; and AdamW over many
tensors, with moments in 32 or in 8 bits.  The Python face below is a thin ctypes binding with the same names.
"""
from .flround import (FL_BF16, FL_F32, FL_MAX_GROUPS, FL_MAX_PEERS, FL_MAX_TARGETS,
                      FL_NOALLOC_SCRATCH_BYTES, HIP_EVENT_DISABLE_SYSTEM_FENCE, FlError,
                      HipEvents, Layout, Tensors, embed_workspace_bytes, fingerprint, fl_adamw_step,
                      fl_adamw_tensors, fl_broadcast_recv, fl_embed, fl_embed_grad, fl_fedavg,
                      fl_fedopt, fl_grad_sumsq, fl_head_distill, fl_head_distill_grad,
                      fl_head_loss, fl_head_loss_grad, fl_layer_norm, fl_layer_norm_grad,
                      fl_local_step, fl_local_step_clipped,
                      fl_round, fl_round_hsdp, fl_round_noalloc, fl_round_outer, fl_shard_reduce,
                      fl_shard_reduce_wire, fl_state_convert, fl_top_logits, head_workspace_bytes,
                      layer_norm_workspace_bytes, lib, lr_cosine,
                      make_hsdp_cfg, make_round_cfg, noalloc_workspace_bytes, set_blocks_per_cu,
                      status_string, top_workspace_bytes)
from .arena import place_arrays, separate_arrays

__all__ = ["FL_BF16", "FL_F32", "FL_MAX_GROUPS", "FL_MAX_PEERS", "FL_MAX_TARGETS",
           "FL_NOALLOC_SCRATCH_BYTES", "HIP_EVENT_DISABLE_SYSTEM_FENCE", "FlError", "HipEvents", "Layout", "Tensors",
           "embed_workspace_bytes", "fingerprint",
           "fl_adamw_step", "fl_adamw_tensors", "fl_broadcast_recv", "fl_embed", "fl_embed_grad", "fl_fedavg", "fl_fedopt", "fl_grad_sumsq",
           "fl_head_distill", "fl_head_distill_grad", "fl_head_loss", "fl_head_loss_grad", "fl_layer_norm", "fl_layer_norm_grad",
           "fl_local_step", "fl_local_step_clipped",
           "fl_round", "fl_round_hsdp", "fl_round_noalloc", "fl_round_outer", "fl_shard_reduce",
           "fl_shard_reduce_wire", "fl_state_convert", "fl_top_logits", "head_workspace_bytes",
           "layer_norm_workspace_bytes", "lib", "lr_cosine", "make_hsdp_cfg", "make_round_cfg",
           "noalloc_workspace_bytes", "place_arrays", "set_blocks_per_cu", "separate_arrays",
           "status_string", "top_workspace_bytes"]
