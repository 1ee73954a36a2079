"""MI355X-native routine-selection CNN inference (SoftNeuro's method).

Layers have several interchangeable routines (direct, implicit-GEMM and
Winograd convolution in NCHW, NHWC or NC8HW8 layouts, plus layout converters);
every routine is profiled on the GPU and a dynamic program over the layer
graph (DPRS) selects the fastest routine path including conversion costs.
Next to the graphs stand sequence operators for nets of gated sequence blocks
(``sequence``): products with 4-bit weights, a selective state space scan with
its causal convolution, and the norms around a block
(``seqnet.SequenceNet`` runs them together).
The work is done by libsoftneuro.so (C ABI in include/softneuro.h, HIP
kernels for gfx950); this package is its Python binding.
"""

from .graph import Graph, build_from_spec, to_device
from .seqnet import SequenceNet
from .sequence import BlockNorm, Linear4, Scan, quantize4
from . import native

__all__ = ["Graph", "build_from_spec", "to_device", "BlockNorm", "Linear4", "Scan", "SequenceNet", "quantize4", "native"]
