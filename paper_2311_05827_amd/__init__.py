"""MI355X (gfx950) bit-level compressor / decompressor for pipeline-boundary tensors.

The product is libaccept.so (HIP kernels behind a C ABI, see include/accept.h); this
package holds its sources (csrc/), the build step (build.py) and a ctypes binding
(binding.py; stage_binding.py for the stage operators of include/accept_stage.h, attention_binding.py
for those of include/accept_attention.h).  The binding is imported lazily so that ``python -m
paper_2311_05827_amd.build`` works before the library exists.
"""
import importlib

_BINDING_NAMES = (
    "Desc", "make_desc", "AcceptError", "accept_packed_size", "accept_workspace_size", "accept_compress",
    "accept_decompress", "accept_compress_noalloc", "accept_mbq_init", "accept_mbq_compress_first", "accept_compress_timed", "accept_decompress_timed",
    "accept_compress_polls", "accept_bits_schedule", "accept_stage_name", "alloc_outputs", "dtype_code", "status_string", "version",
    "UNIFORM", "MBQ", "F32", "BF16", "ROUND_NEAREST_EVEN", "ROUND_STOCHASTIC",
    "LAYOUT_PACKED", "LAYOUT_BATCH", "LAYOUT_UNENCODED",
)
_STAGE_NAMES = (
    "NormDesc", "BlockDesc", "MatmulDesc", "make_norm_desc", "make_block_desc", "make_matmul_desc", "accept_norm_workspace_size",
    "accept_matmul_workspace_size", "accept_block_stride", "accept_layer_norm", "accept_layer_norm_quantize",
    "accept_layer_norm_backward", "accept_block_quantize", "accept_block_matmul", "E4M3", "E5M2",
)
_ATTENTION_NAMES = (
    "RotateDesc", "AttentionDesc", "CacheDesc", "make_rotate_desc", "make_attention_desc", "make_cache_desc", "accept_rotate",
    "accept_attention_workspace_size", "accept_attention", "accept_attention_backward_workspace_size", "accept_attention_backward",
    "accept_cache_append", "accept_cache_workspace_size", "accept_cache_attention", "REST_KEPT", "REST_ZEROS", "ROTATE_HALVES",
    "ROTATE_NEIGHBOURS",
)


def __getattr__(name):
    if name in ("boundary", "stage"):
        return importlib.import_module(__name__ + "." + name)
    if name == "binding" or name in _BINDING_NAMES:
        mod = importlib.import_module(__name__ + ".binding")
        value = mod if name == "binding" else getattr(mod, name)
        globals()[name] = value  # found without this function from now on: it took 3.7 us, more than the call it finds
        return value
    if name == "stage_binding" or name in _STAGE_NAMES:
        mod = importlib.import_module(__name__ + ".stage_binding")
        value = mod if name == "stage_binding" else getattr(mod, name)
        globals()[name] = value
        return value
    if name == "attention_binding" or name in _ATTENTION_NAMES:
        mod = importlib.import_module(__name__ + ".attention_binding")
        value = mod if name == "attention_binding" else getattr(mod, name)
        globals()[name] = value
        return value
    raise AttributeError(name)
