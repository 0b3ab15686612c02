"""Batched CTC loss and gradient for MI355X (gfx950), behind a C-ABI library.

`paper_1512_02595_amd.ctc` is the ctypes binding to the HIP library;
`paper_1512_02595_amd.layer` that of the output layer's calls in the same library,
`paper_1512_02595_amd.block` that of the calls of a recurrent block under it;
`paper_1512_02595_amd.workloads` draws the synthetic batches.  Importing the
package does not load the library; the binding does so on first use and raises
if it has not been built.
"""
__all__ = ["block", "ctc", "layer", "workloads"]
