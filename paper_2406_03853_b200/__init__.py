"""B200-native EESD decode round: thin Python binding over the C-ABI CUDA library."""
from .binding import (Config, Engine, EesdError, KV4Cache, LogitRules, Stats, W4Matrix, accept_resample, attend_rows, lib, lib_path,  # noqa: F401
                      process_logits, project_rows, sample_rows)
