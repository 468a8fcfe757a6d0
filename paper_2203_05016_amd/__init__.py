"""MI355X-native Shfl-BW sparse-weight x dense-activation product (linear
layers and implicit-GEMM convolution) and, on the same features x tokens
activations, attention: over a paged cache of keys and values in 4 bits, and of
prompts with a sliding window and sinks; behind a C-ABI library.

``paper_2203_05016_amd.binding`` is the thin ctypes layer over the library;
``paper_2203_05016_amd.synth`` draws seeded synthetic inputs and holds no
arithmetic of the method.  The library is loaded on first use and its
absence is an error: there is no CPU fallback.
"""
__all__ = ["binding", "synth"]
