"""CPU oracle of TreeFlash drafting: test infrastructure, never used by the library.

Only the tests, the entry module's smoke check and the benchmark's CPU-baseline
leg import this package.
"""
from .treeflash_oracle import *  # noqa: F401,F403
from .treeflash_oracle import __all__ as _tree_all
from .verify_step_oracle import *  # noqa: F401,F403
from .verify_step_oracle import __all__ as _step_all

__all__ = [*_tree_all, *_step_all]
