"""MI355X-native phrase-boosting tree (GPU-PB shallow-fusion context biasing): Python binding of libpb.so."""
from .binding import (  # noqa: F401
    EXPORTS, PB_BF16, PB_DISTILL_RENORM, PB_DISTILL_TAIL, PB_EHIP, PB_EINVAL, PB_ENOMEM, PB_ERANGE, PB_EUNSUPPORTED, PB_F16, PB_F32, PB_OK, PB_SELECT_FUSED, PB_SELECT_TWO_STAGE, PB_SELECT_TWO_STAGE_CTC, PB_W_LOGDEPTH, PB_W_UNIFORM, PB_W_UNIFORM_FINAL,
    Forest, PbError, Tree, library_path, load, pb_build, pb_forest_build, pb_forest_free, pb_free, pb_fuse_frames_forest, pb_fuse_step_beam_forest, pb_fuse_step_forest, pb_score_forest, pb_fuse_frames, pb_fuse_frames_select, pb_fuse_frames_plan, pb_fuse_frames_workspace_bytes, pb_fuse_frames_ws, pb_fuse_frames_static, pb_fuse_step, pb_fuse_step_select, pb_fuse_step_beam,
    pb_host_arrays, pb_info, pb_score, pb_state_prefix, pb_validate, pb_validate_states, strerror,
    Tensors, pb_embed_tokens, pb_embed_tokens_backward, pb_embed_tokens_backward_workspace_bytes, pb_grad_clip, pb_grad_norm, pb_grad_norm_workspace_bytes, pb_tensors_build, pb_tensors_free, pb_verify_draft, pb_verify_draft_workspace_bytes,
    pb_distill_topk, pb_distill_topk_workspace_bytes, pb_token_logprobs, pb_token_logprobs_backward, pb_token_logprobs_workspace_bytes,
)
