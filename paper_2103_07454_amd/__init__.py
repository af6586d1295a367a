"""EventGraD per-iteration parameter path on MI355X (gfx950).

Sub-modules:
  inputs  -- seeded synthetic workloads (tensor shape lists, initial parameters,
             the five benchmark configurations).  Holds none of the method's
             arithmetic; it feeds both the HIP path and the test oracle.
  nn      -- operators for training feed-forward blocks: norms, the gated block, clipping.
  ffn_ring -- ring workers that train feed-forward blocks with them; also a command.
  evg     -- thin ctypes binding over the C-ABI library ``libevg.so``
             (evg_init / evg_step / evg_stats ...).  Imported lazily so that
             ``inputs`` can be used without the HIP library being built.
"""

__all__ = ["inputs", "evg", "nn", "ffn_ring"]


def __getattr__(name):
    if name in ("inputs", "evg", "nn", "ffn_ring"):
        import importlib
        return importlib.import_module(f"{__name__}.{name}")
    raise AttributeError(name)
