"""B200-native RPS synchronisation step (unreliable parameter-server averaging), and operators for the workers' own
training steps.

The compute path lives in ``csrc/`` (CUDA, sm_100a) behind the C ABIs declared in
``include/rps.h`` and ``include/rps_ops.h``; ``binding`` and ``ops`` are the thin ctypes layers over
them and are imported lazily so that the input generators can be used without the built library.
"""

__all__ = ["workloads", "binding", "ops"]


def __getattr__(name):
    if name in ("binding", "RPS", "load_library"):
        import importlib

        mod = importlib.import_module(".binding", __name__)
        return mod if name == "binding" else getattr(mod, name)
    if name == "ops":
        import importlib

        return importlib.import_module(".ops", __name__)
    raise AttributeError(name)
