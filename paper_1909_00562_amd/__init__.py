"""MI355X-native attention-softmax forward/backward (section 3.2 of the hybrid
data-model parallel Seq2Seq RNN MT paper), the stacked-LSTM part that feeds it,
the operators over the vocabulary at the two ends of a model over words, and those
of serving word by word (a paged cache, attention over it, drafted words), as a
C-ABI HIP library plus this thin ctypes binding.  Importing the package does not
load the library; the first call does, and fails loudly if it has not been built."""
from .binding import (  # noqa: F401
    AS_BF16, AS_F32, KC_BF16, KC_E4M3, KC_F32, KC_INT8, STAGE_NAMES, AsAdam, AsShape, AttnSoftmaxError, DeviceBatch,
    DeviceEmbed, DeviceKvAttn, DeviceKvCache, DeviceLstm, DeviceVocabLoss, DeviceVocabVerify, KcAttn, KcCache, LsShape,
    VoEmbed, VoShape, VoTeacher, VoVerify, kv_cache_attn, kv_cache_attn_workspace_bytes, kv_cache_read, kv_cache_write,
    vocab_distill_bwd, vocab_distill_fwd, vocab_embed_bwd, vocab_embed_fwd, vocab_embed_workspace_bytes, vocab_verify,
    vocab_verify_workspace_bytes, vocab_xent_bwd, vocab_xent_fwd, vocab_xent_workspace_bytes,
    attn_softmax_adam_step, lstm_stack_bwd, lstm_stack_fwd, lstm_stack_workspace_bytes,
    attn_softmax_bwd, attn_softmax_fwd_static, attn_softmax_stream_probe,
    attn_softmax_fwd, attn_softmax_last_error, attn_softmax_profile_enable,
    attn_softmax_profile_read, attn_softmax_profile_select, attn_softmax_step_fwd, attn_softmax_step_prepare,
    attn_softmax_step_workspace_bytes, attn_softmax_view, attn_softmax_workspace_bytes, library_path, load_library)
