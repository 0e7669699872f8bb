"""GB300-native Conduit scoring pass and budgeted selective refresh.

Submodules: ``conduit`` (binding of the libconduit C ABI, loads the CUDA
library), ``pipeline`` (the whole refresh step over one batch), ``context`` (contexts
kept in 4 bits, appended to and attended over), ``synth``
(seeded synthetic workloads) and ``_build`` (nvcc build of the library).
Importing the package itself loads nothing.
"""

__all__ = ["conduit", "context", "pipeline", "synth"]
