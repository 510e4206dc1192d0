"""4-bit quantised linear layers (W4A16 group-wise weight-only, W4A4 integer
conv-as-GEMM) for AMD MI355X (gfx950), behind a C-ABI library.

Beside them what a decoder layer does between its linears when several requests
are served: norms with the residual (and their gradient), a paged cache of keys
and values with the attention over it, adapters that differ from row to row;
and the policy's ends, which stay in 16 bits: embeddings, linears with an
activation (and the gradients of both), the next token.

`synth` draws the seeded synthetic inputs; `binding` marshals arguments into
`libqail.so`.  Importing the package does not load the native library; the
first call that needs it does, and fails loudly if it is missing.
"""
__all__ = ["synth", "binding"]
