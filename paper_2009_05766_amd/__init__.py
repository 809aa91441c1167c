"""MI355X-native NetMax iteration: thin Python binding of libnetmax.so (HIP kernels, C ABI)."""
from .binding import *  # noqa: F401,F403
from .binding import NetMax, NetmaxError, load, EXPORTS, LIB_PATH  # noqa: F401
from .lm_ops import netmax_linear, netmax_linear_grad, netmax_orthogonalize, netmax_policy_loss, netmax_preference_loss  # noqa: F401
from .lm_step_ops import Gradients, netmax_block_norm, netmax_block_norm_grad, netmax_clip_grads, netmax_embed, netmax_embed_grad, netmax_grad_norm  # noqa: F401
