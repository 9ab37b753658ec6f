"""Block Transformer KV-cache attention for B200 (sm_100a): ctypes binding over libbt.so.

Importing the package loads (building first if needed) the CUDA library; there is no
CPU or framework fallback.
"""
from .binding import *  # noqa: F401,F403
from .binding import (BlockCache, BlockCacheKV4, BtError, LocalCache, alloc_workspace, alloc_workspace_kv4,  # noqa: F401
                      alloc_workspace_shared, alloc_workspace_weights, bt_config, lib, make_config, status_string)
