"""B200-native Gumbel-max list sampling (arXiv 2506.05632): Python binding of libgls.

The functions here only marshal arguments (torch tensors -> raw device pointers, strides in
elements) into the C ABI declared in include/gls.h; every step of the method runs in the CUDA
kernels of csrc/.  There is no CPU fallback: if libgls.so cannot be loaded the calls raise.

    draft_sample(logits, ...)                 Algorithm 1 third step / Algorithm 2 draft loop
    target_sample_verify(logits, tokens, ...) Algorithm 2 verification
    draft_verify(draft, target, ...)          both of the above in one call (one sweep launch)
    compress_select(enc, dec, bins, ...)      Sec. 5.1 encoder / decoder index selection
    compress_gaussian(u, a, t, bins, ...)     the same from the source: Appendix C weights computed in the kernels
    token_logprobs(logits, tokens, ...)       log probabilities, entropy, most likely alternatives
    emitted_logprobs(logits, tokens, accept)  the same for the tokens a verification emitted
    embed_tokens(table, tokens, ...)          rows of a table by token, scaled

The last group's token_logprobs and embed_tokens are differentiable in reverse mode (autograd.py); their
gradients are token_logprobs_backward and embed_tokens_backward.  emitted_logprobs has none.
"""
from .autograd import embed_tokens, token_logprobs  # noqa: F401
from .binding import (  # noqa: F401
    COMBINE_ACTIVE, COMBINE_ALL, NO_BONUS, VERIFY_ALL_ROWS, VERIFY_ACTIVE_ROWS, VERIFY_FIRST_PHASE,
    VERIFY_REST, VERIFY_THREE_PHASES, NOISE_SHARED_ACROSS_K,
    DEV_BAD_TOKEN, DEV_EMPTY_SUPPORT, MAX_GIVEN, GlsError,
    build, copy_rows_to_device, debug_bounds, compress_gaussian, compress_gaussian_workspace_bytes, compress_select, draft_sample, draft_sample_sparse, draft_sample_static,
    draft_sample_topm, draft_verify, draft_verify_workspace_bytes, lib_path, load,
    embed_tokens_backward, embed_tokens_backward_workspace_bytes, emitted_logprobs,
    static_scratch_bytes, status_string, target_sample_verify, target_sample_verify_sparse,
    target_sample_verify_topm, token_logprobs_backward, topm_workspace_bytes, verify_phases, verify_walk, version, workspace_bytes)
