"""Faster Flash Decoding (FFD) decode attention for AMD MI355X (gfx950).

The compute path is ``libffd.so`` (HIP kernels behind a C ABI, declared in ``include/ffd.h``);
``ffd`` is its ctypes binding.
"""
from .ffd import (BLOCK, HEAD_DIM, FfdError, FfdLibraryError, decode_attention,  # noqa: F401
                  dense_decode_attention, empty_kv8, empty_paged, empty_quantized, evict_paged, kv8_decode_attention, kv8_shapes,
                  kv8_workspace_bytes, lib, new_kv8_workspace, new_paged_workspace, new_shared_prefix_workspace, new_workspace,
                  paged_attention, paged_attention_weights, paged_workspace_bytes, quantize_keys, quantized_shapes, read_kv8,
                  resolve_splits, shared_prefix_decode_attention, shared_prefix_workspace_bytes, workspace_bytes,
                  write_kv8, write_paged)
