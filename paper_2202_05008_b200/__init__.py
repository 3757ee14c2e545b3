"""B200-native evolution-strategy generation (ask -> rollout -> tell) behind a C-ABI.

``operators`` holds the calls that need no solver; ``binding`` is the thin ctypes layer over ``libevo.so``; ``workloads`` holds the synthetic
configurations and seeded input generators; ``build`` compiles the CUDA sources.
"""
from .binding import EvoConfig, EvoError, Solver, load_library  # noqa: F401
from .operators import grouped_linear, mlp_actions, muon_step, orthogonalize  # noqa: F401
from . import workloads  # noqa: F401
