"""eDKM hot path on MI355X: uniquified DKM weight clustering, forward and backward.

Submodules:
  edkm     — ctypes binding of the C-ABI library ``libedkm.so`` (HIP, gfx950).
  function — ``dkm(w, c0, ...)``, ``linear``, ``palette_linear``, ``embedding``,
             ``palette_embedding``, ``rms_norm``, ``residual_norm`` and
             ``linear_cross_entropy``: the clustering and what a model does with its
             weights as differentiable torch ops.
  optim    — ``AdamW``: a torch optimizer over the library's step.
  runner   — one init_unique + forward (+ backward) call with outputs allocated.
  inputs   — seeded synthetic inputs (weights, initial centroids, gradients).

Importing the package does not load the HIP library; ``edkm`` does, and fails
loudly if it is missing.
"""
