"""INT8 convolution backward with distribution-adaptive gradient quantization, native to MI355X.

``binding`` wraps the C ABI of ``libdaq.so`` (include/daq.h); ``workloads`` holds the seeded synthetic
layer shapes and inputs; ``feed_forward`` is a block on the library's 4-bit products and 8-bit checkpoints, ``experts``
a sparse one on its 8-bit floating point products and router; ``build`` compiles the library.
"""
