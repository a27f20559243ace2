"""MI355X (gfx950) ACDC / AFDF cascade library: HIP kernels behind a C ABI
(include/acdc.h, include/acdc_train.h, include/acdc_train_lm.h) with a thin torch binding.

The cascades are in ``acdc``; the rows that go into them and their
normalisation in ``layers``; the losses on their outputs in ``losses`` and the
step of their parameters in ``optim``."""

from . import layers, losses, optim
from .acdc import (FLAG_COMPLEX, FLAG_PERM, FLAG_RELU, ACDCCascade, ACDCError, acdc_cascade,
                   backward, forward, prepare, supported)

__all__ = ["FLAG_PERM", "FLAG_RELU", "FLAG_COMPLEX", "forward", "backward", "prepare", "supported",
           "acdc_cascade", "ACDCCascade", "ACDCError", "layers", "losses", "optim"]
