"""B200-native load-time checkpoint resharding (arXiv 2407.20143): binding of libbcp.so."""
from .api import (BcpError, Plan, Stager, bcp_decompose, bcp_dedup_assign, bcp_pack, bcp_pack_cache_clear, bcp_pack_layout, bcp_pack_static, bcp_plan,
                  bcp_plan_device_status, bcp_reshard, bcp_reshard_host, bcp_safetensors_export, bcp_safetensors_layout, bcp_unpack, bcp_version)

# The decoding operators take torch tensors; torch is imported when the first of them is asked for by name, so
# that the host-only calls (planning, layouts) load without it.  For the same reason a star import leaves them out.
_DECODE = ("KvCache", "KvWorkspace", "RopeTable", "bcp_kv_attend", "bcp_kv_attend_shared", "bcp_kv_read", "bcp_kv_write", "bcp_rope", "bcp_rope_backward", "bcp_verify_drafts", "rope", "rope_axes",
           "rope_frequencies")

__all__ = ["BcpError", "Plan", "Stager", "bcp_decompose", "bcp_dedup_assign", "bcp_pack", "bcp_pack_cache_clear", "bcp_pack_layout", "bcp_pack_static", "bcp_plan",
           "bcp_plan_device_status", "bcp_reshard", "bcp_reshard_host", "bcp_safetensors_export", "bcp_safetensors_layout", "bcp_unpack", "bcp_version"]


def __getattr__(name):
    if name not in _DECODE:
        raise AttributeError(f"module {__name__!r} has no attribute {name!r}")
    from . import decode

    value = globals()[name] = getattr(decode, name)
    return value


def __dir__():
    return sorted({*globals(), *_DECODE})
