"""libtng on MI355X: the data-parallel hot path of Trajectory Normalized Gradients.

`paper_1901_08227_amd.binding` is the ctypes binding of the C-ABI library (HIP, gfx950);
`paper_1901_08227_amd.lowbit` runs the layers of a network on 8-bit codes;
`paper_1901_08227_amd.network` trains one with them and the gradient coder;
`paper_1901_08227_amd.synth` draws the seeded synthetic inputs.  Importing the package
loads none: the binding raises at first use when the built library is missing.
"""
__all__ = ["binding", "lowbit", "network", "synth", "build"]
