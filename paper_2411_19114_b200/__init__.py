"""Fused vision preprocessing for B200: ragged uint8 HWC batch -> dense NCHW fp32/fp16.

The work is done by a C-ABI CUDA library (``libpreba.so``, built from ``csrc/``);
``binding`` marshals arguments to it and nothing else.  ``workloads`` holds the
seeded synthetic inputs.  Beside the preprocessing the library has the serving step behind it, for
models that answer in tokens (``include/preba_tokens.h``): pages, positions, rotation with the
cache write, attention over the paged cache; and a beam search over an encoder's states
(``include/preba_beams.h``): attention to the states, selection, block tables of the beams, copies of
their open pages.  Importing the package does not load the library; the
first call does, and fails loudly if it has not been built.
"""
__all__ = ["binding", "workloads"]
