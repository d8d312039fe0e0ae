"""MI355X-native temporal neighbourhood sampling (GNNFlow, arXiv 2311.17410, Algorithm 1).

``binding``    ctypes binding of the C ABI (include/tns.h); loads libtns.so lazily
``cache_binding``, ``train_binding``   the same of include/tns_cache.h and include/tns_train.h
``workloads``  seeded synthetic streams and query batches (no sampling arithmetic)
``build``      compiles the HIP library in-tree
"""
