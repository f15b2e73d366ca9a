"""The 8-bit paged KV cache: binding of include/flexco_kv8.h (the same names, argument marshalling only) and owners of its
device memory.

    batch = kv8.DeviceBatch8(cfg, requests, seq_pages, num_pages)    # index maps and runs of a mixed batch
    pool = kv8.DevicePool8(cfg, num_pages)                           # one layer's cache
    kv8.flexco_kv8_append(c, batch.maps, batch.runs, batch.n_runs, qkv, pool.c, q, cfg.q_dim)
    kv8.flexco_kv8_attention(c, batch.maps, q, pool.c, out, lse, ws.ptr, ws.bytes)

Before a finetune window's backward pass flexco_kv8_expand writes the sequence's pages into a pool of the activations' type
(host.DevicePool), which flexco_lora_bwd and flexco_attention_window_bwd take.
"""
import ctypes as C

import numpy as np
import torch

from . import binding as B
from . import host as HH

KV8_ABI_VERSION = 1
EXPORTS = ("flexco_kv8_abi_version", "flexco_kv8_runs", "flexco_kv8_append", "flexco_kv8_attention", "flexco_kv8_expand",
           "flexco_kv8_layer_forward")


class Pool(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("k_codes", "v_codes", "k_scale", "v_scale")] + \
               [("num_pages", C.c_int32), ("page_size", C.c_int32)]


def _load():
    lib = B._lib
    P = C.POINTER
    i32, vp, sz = C.c_int32, C.c_void_p, C.c_size_t
    sigs = {
        "flexco_kv8_abi_version": [],
        "flexco_kv8_runs": [P(B.Maps), vp, i32, P(i32)],
        "flexco_kv8_append": [P(B.LayerCfg), P(B.Maps), vp, i32, vp, P(Pool), vp, sz, vp],
        "flexco_kv8_attention": [P(B.LayerCfg), P(B.Maps), vp, P(Pool), vp, vp, vp, sz, vp],
        "flexco_kv8_expand": [P(B.LayerCfg), P(Pool), vp, i32, P(B.KVPool), vp, vp],
        "flexco_kv8_layer_forward": [P(B.LayerCfg), P(B.BaseWeights), P(B.Lora), P(B.Maps), vp, i32, vp, vp, P(Pool), P(B.FtState),
                                     vp, sz, vp],
    }
    for name, args in sigs.items():
        fn = getattr(lib, name, None)
        if fn is None:
            if B.HOST_ONLY:
                continue
            raise ImportError("libflexco.so lacks the symbol %s" % name)
        fn.argtypes = args
        fn.restype = i32
    if lib.flexco_kv8_abi_version() != KV8_ABI_VERSION:
        raise ImportError("libflexco.so has 8-bit cache ABI version %d, binding expects %d" % (lib.flexco_kv8_abi_version(), KV8_ABI_VERSION))
    return lib


_lib = _load()


def flexco_kv8_abi_version():
    return _lib.flexco_kv8_abi_version()


def flexco_kv8_runs(host_maps, capacity=None):
    """host_maps: Maps with host pointers (of flexco_build_maps).  -> int32 [n_runs, 2]: first token, tokens"""
    cap = host_maps.T if capacity is None else capacity
    runs = np.zeros((max(cap, 1), 2), dtype=np.int32)
    n = C.c_int32(0)
    B._check(_lib.flexco_kv8_runs(C.byref(host_maps), runs.ctypes.data, cap, C.byref(n)))
    return runs[:n.value].copy()


def flexco_kv8_append(cfg, maps, runs, n_runs, qkv, pool, q_out, ld_q, stream=None):
    B._check(_lib.flexco_kv8_append(C.byref(cfg), C.byref(maps), B._ptr(runs), n_runs, B._ptr(qkv), C.byref(pool), B._ptr(q_out), ld_q,
                                    B._stream(stream)))


def flexco_kv8_attention(cfg, maps, q, pool, out, lse, ws, ws_bytes, stream=None):
    B._check(_lib.flexco_kv8_attention(C.byref(cfg), C.byref(maps), B._ptr(q), C.byref(pool), B._ptr(out), B._ptr(lse), B._ptr(ws),
                                       ws_bytes, B._stream(stream)))


def flexco_kv8_expand(cfg, pool, src_pages, n_tokens, wide, dst_pages, stream=None):
    B._check(_lib.flexco_kv8_expand(C.byref(cfg), C.byref(pool), B._ptr(src_pages), n_tokens, C.byref(wide), B._ptr(dst_pages),
                                    B._stream(stream)))


def flexco_kv8_layer_forward(cfg, w, lora, maps, runs, n_runs, x_in, x_out, pool, ft, ws, ws_bytes, stream=None):
    B._check(_lib.flexco_kv8_layer_forward(C.byref(cfg), C.byref(w), B._opt(lora), C.byref(maps), B._ptr(runs), n_runs, B._ptr(x_in),
                                           B._ptr(x_out), C.byref(pool), B._opt(ft), B._ptr(ws), ws_bytes, B._stream(stream)))


class DevicePool8:
    """8-bit paged cache of one layer: codes [P, nkv, d / 16, ps, 16] and [P, nkv, d, ps], scales [P, nkv]."""

    def __init__(self, cfg, num_pages, device="cuda"):
        self.cfg, self.num_pages = cfg, num_pages
        nkv, d, ps = cfg.n_kv_heads, cfg.head_dim, cfg.page_size
        self.k = torch.zeros((num_pages, nkv, d // 16, ps, 16), dtype=torch.uint8, device=device)
        self.v = torch.zeros((num_pages, nkv, d, ps), dtype=torch.uint8, device=device)
        self.k_scale = torch.zeros((num_pages, nkv), dtype=torch.float32, device=device)
        self.v_scale = torch.zeros_like(self.k_scale)
        self.c = Pool(self.k.data_ptr(), self.v.data_ptr(), self.k_scale.data_ptr(), self.v_scale.data_ptr(), num_pages, ps)

    def expand(self, pages, n_tokens, wide, dst_pages, stream=None):
        """The first n_tokens positions of the sequence that holds `pages`, into pages of `wide` (host.DevicePool of the same
        configuration); both lists int32 tensors on the device."""
        flexco_kv8_expand(HH.c_cfg(self.cfg), self.c, pages, n_tokens, wide.c, dst_pages, stream)


class DeviceBatch8(HH.DeviceBatch):
    """Index maps of a mixed batch and its runs, the tokens by the page they are written to."""

    def __init__(self, cfg, requests, seq_pages, num_pages, kv_split_pages=0, device="cuda"):
        super().__init__(cfg, requests, seq_pages, num_pages, kv_split_pages, device)
        self.host_runs = flexco_kv8_runs(self.host_maps)
        self.n_runs = len(self.host_runs)
        self.runs = torch.from_numpy(self.host_runs).to(device) if device is not None else None
