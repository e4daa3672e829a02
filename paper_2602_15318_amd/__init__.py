"""MI355X-native hot path of one Sparrow speculative-decoding step.

Thin Python binding over the C-ABI library built from csrc/ (see include/sparrow.h):
draft_window_attn, verify_attn and accept, plus hsr_fc and draft_qkv_append (the draft's input side) and kv_commit (after acceptance); and, over the
C-ABI library of the paged-cache operators (include/sparrow_paged.h), page_update, mrope_table, mrope_append and chunk_attn; and, over that of the operators for
many requests about one long video (include/sparrow_serve.h), mrope_append8, page_gather, chunk_attn8 and prefix_attn.  All computation runs in the HIP kernels;
PyTorch only provides device memory and streams.
"""
__all__ = ["SparrowError", "accept", "accept_workspace_bytes", "draft_window_attn", "last_error",
           "library_path", "verify_attn", "verify_attn_workspace_bytes", "version", "AttnDesc",
           "lib", "hsr_fc", "draft_qkv_append", "kv_commit", "accept_sample",
           "accept_sample_workspace_bytes", "draft_topk", "TreePool", "stream_read",
           "verify_attn_static", "STATIC_WS_BYTES", "debug_validate_parent",
           "debug_validate_text_idx", "accept_sample_q"]
_PAGED = ("page_update", "mrope_table", "mrope_append", "chunk_attn", "chunk_attn_workspace_bytes")
_SERVE = ("mrope_append8", "page_gather", "chunk_attn8", "prefix_attn", "prefix_attn_workspace_bytes")
__all__ += _PAGED + _SERVE


def __getattr__(name):
    # The binding (and with it the library of the name) is loaded on first use of any public name, so that
    # `paper_2602_15318_amd.build` stays importable on a tree that has not been built yet.  A
    # missing library raises ImportError there: there is no fallback path.
    if name in __all__:
        if name in _PAGED:
            from . import paged as module
        elif name in _SERVE:
            from . import serve as module
        else:
            from . import binding as module
        value = globals()[name] = getattr(module, name)       # (found without this function from now on)
        return value
    raise AttributeError(f"module {__name__!r} has no attribute {name!r}")
