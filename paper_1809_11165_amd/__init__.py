"""MI355X-native BBMM inference hot path (arXiv 1809.11165).

`paper_1809_11165_amd.inputs`  -- seeded synthetic workloads (no method arithmetic)
`paper_1809_11165_amd.binding` -- ctypes binding over libbbmm.so (HIP, gfx950); besides the inference path it holds the
                                 attention calls (`Attention`, `Context.bbmm_attend`, `bbmm_attend_grad`,
                                 `bbmm_bucket_bias`, `bbmm_bucket_bias_grad`) and those of the rotation and the
                                 paged cache (`Rotation`, `Cache`, `CachedAttention`, `Context.bbmm_rotate`,
                                 `bbmm_rotate_grad`, `bbmm_cache_write`, `bbmm_cache_read`, `bbmm_attend_cache`)

Nothing is imported eagerly: the binding loads the shared library on first use
and raises if it has not been built.
"""
__all__ = ["inputs", "binding"]
