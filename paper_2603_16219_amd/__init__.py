"""MI355X-native verify-and-recover block of SpecSteer's Draft-Verify-Recover protocol.

``binding`` wraps the C-ABI HIP library (``libspecsteer.so``, built from
``csrc/``), ``losses`` that of the losses which train the specialist
(``libspecsteer_loss.so``, from ``csrc/loss/``); ``workloads`` holds the seeded synthetic input recipes.  Importing
the package loads neither torch nor a library.
"""

__all__ = ["binding", "losses", "workloads"]
