"""B200-native EESD decode round: thin Python binding over the C-ABI CUDA library."""
from .binding import (Config, Engine, EesdError, LogitRules, Stats, W4Matrix, accept_resample, lib, lib_path, process_logits,  # noqa: F401
                      project_rows, sample_rows)
