"""WindowKV prefill-time KV-cache window selection for B200 (sm_100a).

`binding`   ctypes face of the C-ABI library (wkv_score_windows, wkv_select_topk_windows,
            wkv_gather_kv, wkv_compress_group; around them wkv_rotate_prompt, wkv_attend_prompt,
            wkv_append_kv_paged, wkv_attend_paged, wkv_evict_kv_paged); the only implementation of the path.
`workloads` seeded synthetic inputs of the benchmark configurations.
`build`     compiles the library in-tree with nvcc.
"""
__all__ = ["binding", "workloads", "build", "replicas"]
