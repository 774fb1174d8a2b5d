"""B200 (sm_100a) selective scan (S6): C-ABI CUDA library plus a thin ctypes binding.

`ssm_scan_fwd` / `ssm_scan_bwd` are resolved lazily so that importing the package (for example to reach the
seeded input generator in `synth`) does not need torch or the compiled library.
"""

__all__ = ["ssm_scan_fwd", "ssm_scan_bwd", "ssm_scan_fwd_static", "ssm_step", "ssm_gated_fwd", "ssm_gated_bwd",
           "ssm_gated_step", "ssm_norm_fwd", "ssm_norm_bwd", "binding", "synth", "build"]


def __getattr__(name):
    if name.startswith("ssm_") and name in __all__:
        from . import binding
        return getattr(binding, name)
    if name in ("binding", "synth", "build"):
        import importlib
        return importlib.import_module(f".{name}", __name__)
    raise AttributeError(name)
