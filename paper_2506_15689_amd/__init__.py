"""MI355X (gfx950) implementation of BASE-Q's W4A4 rotated linear layer.

`binding` holds the ctypes wrappers of the C ABI declared in include/basq.h; `synth_inputs`
draws the seeded synthetic layers; `build` compiles libbasq.so with hipcc.  Nothing is loaded
at import time; the first binding call loads the library and raises if it is missing.  The operators around the linear layer
(norm, rotary positions and cache, attention) and at the ends of a step (cache books, embeddings, logits, tokens) go through `_block`, a compiled module on the same library.
"""
from . import synth_inputs  # noqa: F401

__all__ = ["binding", "build", "synth_inputs"]
