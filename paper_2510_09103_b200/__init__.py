"""B200-native AdaPM optimizer step: a C-ABI CUDA library (csrc/, include/adapm.h) and its ctypes binding."""
from .binding import (  # noqa: F401
    MOM_NONE, MOM_FULL, MOM_LOWRANK, V_ELEMENT, V_BLOCKMEAN, GRAD_F32, GRAD_BF16, PATH_AUTO, PATH_SIMT,
    PATH_TENSOR, FLAG_NO_PANEL_TEAMS, FLAG_FORCE_PANEL_TEAMS, FLAG_NO_SUMSQ_FOLD, FLAG_CHECK_FINITE, ST_WAIT_TEAM, ST_NONFINITE_GRAD, STATE_M, STATE_L, STATE_R, STATE_V, EXPORTS, AdapmError, Context, adapm_block, adapm_hparams,
    adapm_tensor, adapm_create, adapm_plan_default, adapm_version, adapm_group_meansq,
    adapm_group_meansq_scratch_bytes, adapm_group_meansq_static, STATIC_SCRATCH_FLOATS, hparams, lib_path, load, strerror, last_cuda_error,
    TYPE_F32, TYPE_BF16, adapm_rmsnorm, adapm_head_loss, rmsnorm_desc, head_loss_desc, adapm_dropout, adapm_rmsnorm_forward,
    adapm_rmsnorm_backward_scratch_bytes, adapm_rmsnorm_backward, adapm_head_loss_scratch_bytes, adapm_head_loss_forward,
    adapm_head_loss_backward, adapm_head_loss_status,
    CODE_INT8, CODE_E4M3, LINEAR8_FORWARD, LINEAR8_INPUT_GRAD, LINEAR8_WEIGHT_GRAD, adapm_codes8, adapm_linear8, quant8_desc, linear8_desc,
    adapm_quant8, adapm_dequant8, adapm_linear8_scratch_bytes, adapm_linear8_forward, adapm_linear8_input_grad,
    adapm_linear8_weight_grad, adapm_linear8_status,
)
