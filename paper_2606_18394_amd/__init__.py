"""MI355X-native tree verification for parallel tree drafting speculative
decoding: tree-masked GQA attention and greedy tree acceptance as HIP kernels
for gfx950 behind a C ABI (include/treeverify.h).

Importing the package loads nothing; the first call loads libtreeverify.so
and raises if it is missing.  The public calls are those of ``binding``.
"""

__all__ = ["tree_verify_attention", "tree_verify_attention_paged", "tree_accept",
           "tree_accept_noalloc", "commit_path", "commit_path_paged", "draft_topw",
           "build_tree", "block_causal_attention", "tree_accept_sampled",
           "tree_verify_attention_paged_fp8", "append_paged_fp8", "commit_path_paged_fp8",
           "reserve_pages", "fork_pages", "free_pages", "copy_pages", "compact_pages",
           "load_library"]


def __getattr__(name):
    # lazy: torch and the library load on first use of a call
    if name in __all__:
        from . import binding
        # (kept in the module: the look-up through here costs a call 0.8 us)
        call = globals()[name] = getattr(binding, name)
        return call
    raise AttributeError(f"module {__name__!r} has no attribute {name!r}")
