"""MI355X-native batched Autoverse environment step (arXiv 2407.04221, Sec. 2.1).

Python binding of libautoverse.so (C ABI: include/autoverse.h).  The functions below carry
the C names and only marshal arguments: host numpy arrays for rules and checkpoints, torch
device tensors (device memory and streams) for maps, actions, rewards and done flags.
Every step runs in the library's HIP kernels; there is no CPU path.

`Batch` bundles one batch handle with its own output tensors for convenience.
"""
from __future__ import annotations

import ctypes
import os
import struct

import numpy as np

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libautoverse.so")

AV_OK, AV_EINVAL, AV_ENOMEM, AV_EDEVICE, AV_ESTATE = 0, 1, 2, 3, 4
AV_ENGINE_AUTO, AV_ENGINE_GENERIC, AV_ENGINE_LANE16, AV_ENGINE_WAVE, AV_ENGINE_ROWS = 0, 1, 2, 3, 4
AV_ENGINE_GROUP = 5
ENGINES = {"auto": AV_ENGINE_AUTO, "generic": AV_ENGINE_GENERIC, "lane16": AV_ENGINE_LANE16,
           "wave": AV_ENGINE_WAVE, "rows": AV_ENGINE_ROWS, "group": AV_ENGINE_GROUP}
ENGINE_NAMES = {v: k for k, v in ENGINES.items()}
AV_RULES_PARALLEL, AV_RULES_SEQUENTIAL = 0, 1
RULE_MODES = {"parallel": AV_RULES_PARALLEL, "sequential": AV_RULES_SEQUENTIAL}
AV_SITES_ROW_MAJOR, AV_SITES_RANDOM = 0, 1
AV_F32, AV_F16, AV_BF16 = 0, 1, 2
AV_IDS_U8, AV_IDS_I32, AV_IDS_I64 = 0, 1, 2
AV_SCAN_LINEAR, AV_SCAN_GATED = 0, 1
SCAN_FORMS = {"linear": AV_SCAN_LINEAR, "gated": AV_SCAN_GATED}
AV_TOP_MAX = 32
SITE_ORDERS = {"rowmajor": AV_SITES_ROW_MAJOR, "random": AV_SITES_RANDOM}

# Every symbol include/autoverse.h declares.
ABI_SYMBOLS = ("av_create_batch", "av_load_rules", "av_set_rule_control", "av_reset",
               "av_step", "av_step_n", "av_step_observe",
               "av_get_maps", "av_observe", "av_rule_features", "av_state_ptr", "av_get_info",
               "av_get_state", "av_set_state", "av_set_stream", "av_destroy_batch",
               "av_mutate_maps", "av_mutate_rules", "av_search_create", "av_search_load_rules",
               "av_search_begin", "av_search_expand", "av_search_frontier", "av_search_destroy",
               "av_step_n_static", "av_scan_workspace", "av_scan", "av_scan_backward",
               "av_log_probs_workspace", "av_log_probs", "av_log_probs_backward", "av_draw_actions", "av_last_error")


class av_config(ctypes.Structure):
    _fields_ = [("num_envs", ctypes.c_int32), ("height", ctypes.c_int32),
                ("width", ctypes.c_int32), ("channels", ctypes.c_int32),
                ("max_rules", ctypes.c_int32), ("max_pat_h", ctypes.c_int32),
                ("max_pat_w", ctypes.c_int32), ("per_env_rules", ctypes.c_int32),
                ("max_episode_steps", ctypes.c_int32), ("device", ctypes.c_int32),
                ("engine", ctypes.c_int32), ("rule_mode", ctypes.c_int32),
                ("stream", ctypes.c_void_p)]


class av_mutation(ctypes.Structure):
    _fields_ = [("seed", ctypes.c_uint64), ("generation", ctypes.c_uint64),
                ("map_flip_p32", ctypes.c_uint32), ("map_channels", ctypes.c_uint32),
                ("entry_p32", ctypes.c_uint32), ("entry_channels", ctypes.c_uint32),
                ("reward_p32", ctypes.c_uint32), ("reward_lo", ctypes.c_int32),
                ("reward_hi", ctypes.c_int32)]


def p32(p: float) -> int:
    """Probability -> 32-bit threshold (an event happens iff its random word is below it)."""
    return max(0, min(0xFFFFFFFF, int(round(p * 2**32))))


def mutation(seed=0, generation=0, map_flip=0.0, map_channels=0xFFFFFFFF, entry=0.0,
             entry_channels=0xFFFFFFFF, reward=0.0, reward_lo=-1, reward_hi=1) -> av_mutation:
    m = av_mutation()
    m.seed, m.generation = seed, generation
    m.map_flip_p32, m.map_channels = p32(map_flip), map_channels
    m.entry_p32, m.entry_channels = p32(entry), entry_channels
    m.reward_p32, m.reward_lo, m.reward_hi = p32(reward), reward_lo, reward_hi
    return m


class av_search_config(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in (
        "height", "width", "channels", "max_rules", "max_pat_h", "max_pat_w",
        "max_episode_steps", "num_actions", "max_frontier", "table_log2", "device", "engine",
        "rule_mode", "best_first_k", "max_nodes", "hash_bits")] + [("stream", ctypes.c_void_p)]


class av_search_info(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int64) for n in (
        "level", "parents", "children", "terminal", "survivors", "frontier", "visited",
        "best_visit")] + [("best_reward", ctypes.c_int32), ("reserved", ctypes.c_int32)]


class av_info(ctypes.Structure):
    _fields_ = [("num_envs", ctypes.c_int32), ("height", ctypes.c_int32),
                ("width", ctypes.c_int32), ("channels", ctypes.c_int32),
                ("row_bytes", ctypes.c_int32), ("engine", ctypes.c_int32),
                ("state_bytes", ctypes.c_size_t), ("blob_bytes", ctypes.c_size_t)]


class av_scan_config(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_int64) for n in ("steps", "rows", "width")]
                + [(n, ctypes.c_int32) for n in ("dtype", "form", "reverse", "gate_per_value")]
                + [(n, ctypes.c_int64) for n in (
                    "x_step", "x_row", "gate_step", "gate_row", "y_step", "y_row", "cut_step",
                    "cut_row", "dy_step", "dy_row", "dx_step", "dx_row", "dgate_step",
                    "dgate_row")]
                + [("device", ctypes.c_int32), ("reserved", ctypes.c_int32),
                   ("stream", ctypes.c_void_p)])


class av_tokens_config(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int64), ("choices", ctypes.c_int64),
                ("dtype", ctypes.c_int32), ("ids_type", ctypes.c_int32),
                ("row_stride", ctypes.c_int64), ("drow_stride", ctypes.c_int64),
                ("top", ctypes.c_int32), ("device", ctypes.c_int32),
                ("stream", ctypes.c_void_p)]


class AvError(RuntimeError):
    def __init__(self, fn: str, status: int, message: str):
        super().__init__(f"{fn}: status {status}: {message}")
        self.status = status
        self.message = message


_lib = None


def load_library(path: str = LIB_PATH) -> ctypes.CDLL:
    """Load libautoverse.so; raise if it has not been built (there is no fallback)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(path):
        raise RuntimeError(f"{path} is missing: build it with __graft_entry__.build() or "
                           f"python paper_2407_04221_amd/build.py")
    lib = ctypes.CDLL(path)
    P, I32, SZ = ctypes.c_void_p, ctypes.c_int32, ctypes.c_size_t
    sig = {
        "av_create_batch": ([ctypes.POINTER(av_config), ctypes.POINTER(P)], ctypes.c_int),
        "av_load_rules": ([P, I32, P, P, P, P], ctypes.c_int),
        "av_set_rule_control": ([P, P, P, I32, ctypes.c_uint64], ctypes.c_int),
        "av_reset": ([P, P], ctypes.c_int),
        "av_step": ([P, P, P, P], ctypes.c_int),
        "av_step_n": ([P, I32, P, P, P], ctypes.c_int),
        "av_step_observe": ([P, I32, P, P, P, I32, P], ctypes.c_int),
        "av_get_maps": ([P, P], ctypes.c_int),
        "av_observe": ([P, I32, P], ctypes.c_int),
        "av_rule_features": ([P, P], ctypes.c_int),
        "av_state_ptr": ([P], P),
        "av_get_info": ([P, ctypes.POINTER(av_info)], ctypes.c_int),
        "av_get_state": ([P, P, ctypes.POINTER(SZ)], ctypes.c_int),
        "av_set_state": ([P, P, SZ], ctypes.c_int),
        "av_set_stream": ([P, P], ctypes.c_int),
        "av_destroy_batch": ([P], ctypes.c_int),
        "av_mutate_maps": ([P, P, I32, I32, I32, I32, ctypes.POINTER(av_mutation), I32, P],
                           ctypes.c_int),
        "av_mutate_rules": ([I32, I32, I32, I32, I32, P, P, P, P, P, P, P,
                             ctypes.POINTER(av_mutation), I32, P], ctypes.c_int),
        "av_search_create": ([ctypes.POINTER(av_search_config), ctypes.POINTER(P)], ctypes.c_int),
        "av_search_load_rules": ([P, I32, P, P, P, P], ctypes.c_int),
        "av_search_begin": ([P, P], ctypes.c_int),
        "av_search_expand": ([P, ctypes.c_int64, ctypes.POINTER(av_search_info)], ctypes.c_int),
        "av_search_frontier": ([P, P, P, P], ctypes.c_int),
        "av_search_destroy": ([P], ctypes.c_int),
        "av_step_n_static": ([ctypes.POINTER(av_config), I32, P, P, P, P, P, P, P, I32, P, P, P],
                             ctypes.c_int),
        "av_scan_workspace": ([P, I32, ctypes.POINTER(SZ)], ctypes.c_int),
        "av_scan": ([P] * 8 + [SZ], ctypes.c_int),
        "av_scan_backward": ([P] * 12 + [SZ], ctypes.c_int),
        "av_log_probs_workspace": ([P, ctypes.POINTER(SZ)], ctypes.c_int),
        "av_log_probs": ([P] * 9 + [SZ], ctypes.c_int),
        "av_log_probs_backward": ([P] * 8, ctypes.c_int),
        "av_draw_actions": ([P] * 5, ctypes.c_int),
        "av_last_error": ([], ctypes.c_char_p),
    }
    for name, (args, res) in sig.items():
        f = getattr(lib, name)
        f.argtypes = args
        f.restype = res
    _lib = lib
    return lib


def av_last_error() -> str:
    return load_library().av_last_error().decode()


def _check(fn: str, rc: int):
    if rc != AV_OK:
        raise AvError(fn, rc, av_last_error())


def _torch():
    import torch
    return torch


def _dev_ptr(t, dtype, shape, name):
    torch = _torch()
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a device tensor")
    if t.dtype != dtype or tuple(t.shape) != tuple(shape) or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous {dtype} tensor of shape {tuple(shape)}, "
                         f"got {t.dtype} {tuple(t.shape)}")
    return ctypes.c_void_p(t.data_ptr())


def _host(a, dtype, name):
    a = np.ascontiguousarray(a, dtype=dtype)
    return a, a.ctypes.data_as(ctypes.c_void_p)


def current_stream_handle():
    torch = _torch()
    return ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)


def av_create_batch(num_envs, height, width, channels, max_rules, max_pat_h, max_pat_w,
                    per_env_rules=False, max_episode_steps=0, device=None, engine="auto",
                    stream=None, rule_mode="parallel"):
    """Returns an opaque handle (ctypes.c_void_p).  stream: a torch.cuda.Stream, a raw
    handle, or None for torch's current stream on `device`."""
    torch = _torch()
    if device is None:
        device = torch.cuda.current_device()
    if stream is None:
        with torch.cuda.device(device):
            stream = current_stream_handle()
    elif hasattr(stream, "cuda_stream"):
        stream = ctypes.c_void_p(stream.cuda_stream)
    cfg = av_config(num_envs, height, width, channels, max_rules, max_pat_h, max_pat_w,
                    int(bool(per_env_rules)), max_episode_steps, int(device),
                    ENGINES[engine] if isinstance(engine, str) else int(engine),
                    RULE_MODES[rule_mode] if isinstance(rule_mode, str) else int(rule_mode),
                    stream)
    h = ctypes.c_void_p()
    _check("av_create_batch", load_library().av_create_batch(ctypes.byref(cfg), ctypes.byref(h)))
    return h


def av_load_rules(batch, shape, in_pat, out_pat, reward):
    """Host arrays: shape int32 [S][R][2], in_pat / out_pat int8 [S][R][C+1][mh][mw],
    reward int32 [S][R]."""
    shape, ps = _host(shape, np.int32, "shape")
    in_pat, pi = _host(in_pat, np.int8, "in_pat")
    out_pat, po = _host(out_pat, np.int8, "out_pat")
    reward, pr = _host(reward, np.int32, "reward")
    R = shape.shape[1] if shape.ndim == 3 else 0
    _check("av_load_rules", load_library().av_load_rules(batch, R, ps, pi, po, pr))


def av_set_rule_control(batch, limit=None, inhibit=None, order=AV_SITES_ROW_MAJOR, seed=0):
    """Host arrays or None: limit int32 [S][R] (0 = every match), inhibit uint8 [S][R][R]
    ([q][r]: q inhibits r, q < r); order AV_SITES_ROW_MAJOR / AV_SITES_RANDOM or its name."""
    pl = pi = None
    if limit is not None:
        limit, pl = _host(limit, np.int32, "limit")
    if inhibit is not None:
        inhibit, pi = _host(inhibit, np.uint8, "inhibit")
    order = SITE_ORDERS.get(order, order) if isinstance(order, str) else order
    _check("av_set_rule_control",
           load_library().av_set_rule_control(batch, pl, pi, int(order), int(seed)))


def av_mutate_maps(src, dst, m: av_mutation):
    """src, dst: device uint8 tensors [n][C][H][W] (may be the same tensor); runs on the
    current stream of their device."""
    torch = _torch()
    shp = tuple(src.shape)
    if len(shp) != 4:
        raise ValueError("maps must be [n][C][H][W]")
    n, C, H, W = shp
    ps = _dev_ptr(src, torch.uint8, shp, "src")
    pd = _dev_ptr(dst, torch.uint8, shp, "dst")
    _check("av_mutate_maps",
           load_library().av_mutate_maps(ps, pd, n, C, H, W, ctypes.byref(m), src.device.index,
                                         current_stream_handle()))


def av_mutate_rules(shape, in_src, out_src, reward_src, in_dst, out_dst, reward_dst,
                    m: av_mutation):
    """Device tensors in the av_load_rules layout: shape int32 [S][R][2], patterns int8
    [S][R][C+1][mh][mw], rewards int32 [S][R]; destinations may be the sources."""
    torch = _torch()
    S, R, C1, mh, mw = tuple(in_src.shape)
    args = [_dev_ptr(shape, torch.int32, (S, R, 2), "shape"),
            _dev_ptr(in_src, torch.int8, (S, R, C1, mh, mw), "in_src"),
            _dev_ptr(out_src, torch.int8, (S, R, C1, mh, mw), "out_src"),
            _dev_ptr(reward_src, torch.int32, (S, R), "reward_src"),
            _dev_ptr(in_dst, torch.int8, (S, R, C1, mh, mw), "in_dst"),
            _dev_ptr(out_dst, torch.int8, (S, R, C1, mh, mw), "out_dst"),
            _dev_ptr(reward_dst, torch.int32, (S, R), "reward_dst")]
    _check("av_mutate_rules",
           load_library().av_mutate_rules(S, R, C1 - 1, mh, mw, *args, ctypes.byref(m),
                                          in_src.device.index, current_stream_handle()))


def av_reset(batch, init_maps):
    info = av_get_info(batch)
    shp = (info["num_envs"], info["channels"], info["height"], info["width"])
    torch = _torch()
    _check("av_reset", load_library().av_reset(batch, _dev_ptr(init_maps, torch.uint8, shp,
                                                                 "init_maps")))


def av_step(batch, actions, rewards, done):
    torch = _torch()
    B = actions.shape[0] if hasattr(actions, "shape") else 0
    _check("av_step", load_library().av_step(
        batch, _dev_ptr(actions, torch.uint8, (B,), "actions"),
        _dev_ptr(rewards, torch.float32, (B,), "rewards"),
        _dev_ptr(done, torch.uint8, (B,), "done")))


def av_step_n(batch, k, actions, rewards, done):
    torch = _torch()
    B = actions.shape[1] if hasattr(actions, "shape") and actions.dim() == 2 else 0
    _check("av_step_n", load_library().av_step_n(
        batch, int(k), _dev_ptr(actions, torch.uint8, (k, B), "actions"),
        _dev_ptr(rewards, torch.float32, (k, B), "rewards"),
        _dev_ptr(done, torch.uint8, (k, B), "done")))


def av_step_n_static(num_envs, height, width, channels, max_rules, max_pat_h, max_pat_w,
                     rules, state, init, counters, actions, rewards, done, per_env_rules=False,
                     max_episode_steps=0, engine="auto", rule_mode="parallel", device=None,
                     stream=None):
    """k steps of caller-owned environments without device allocation.  rules: host
    (shape, in_pat, out_pat, reward) as av_load_rules; state / init: device uint8 tensors of
    the packed layout (C * B * H * row_bytes bytes); counters: device int32 [B]; actions
    uint8 [k][B], rewards float32 [k][B], done uint8 [k][B] device tensors."""
    torch = _torch()
    if device is None:
        device = torch.cuda.current_device()
    if stream is None:
        with torch.cuda.device(device):
            stream = current_stream_handle()
    elif hasattr(stream, "cuda_stream"):
        stream = ctypes.c_void_p(stream.cuda_stream)
    cfg = av_config(num_envs, height, width, channels, max_rules, max_pat_h, max_pat_w,
                    int(bool(per_env_rules)), max_episode_steps, int(device),
                    ENGINES[engine] if isinstance(engine, str) else int(engine),
                    RULE_MODES[rule_mode] if isinstance(rule_mode, str) else int(rule_mode),
                    stream)
    shape, ps = _host(rules[0], np.int32, "shape")
    in_pat, pi = _host(rules[1], np.int8, "in_pat")
    out_pat, po = _host(rules[2], np.int8, "out_pat")
    reward, pr = _host(rules[3], np.int32, "reward")
    R = shape.shape[1] if shape.ndim == 3 else 0
    k = actions.shape[0]
    row_bytes = 2 if width <= 16 else (4 if width <= 32 else 8)
    nbytes = channels * num_envs * height * row_bytes
    _check("av_step_n_static", load_library().av_step_n_static(
        ctypes.byref(cfg), R, ps, pi, po, pr,
        _dev_ptr(state, torch.uint8, (nbytes,), "state"),
        _dev_ptr(init, torch.uint8, (nbytes,), "init"),
        _dev_ptr(counters, torch.int32, (num_envs,), "counters"), int(k),
        _dev_ptr(actions, torch.uint8, (k, num_envs), "actions"),
        _dev_ptr(rewards, torch.float32, (k, num_envs), "rewards"),
        _dev_ptr(done, torch.uint8, (k, num_envs), "done")))


def av_step_observe(batch, k, actions, rewards, done, w, obs):
    """actions [k][B] uint8, rewards [k][B] float32, done [k][B] uint8, obs [B][C][w][w]
    uint8, all device tensors."""
    torch = _torch()
    info = av_get_info(batch)
    B, C = info["num_envs"], info["channels"]
    pa = _dev_ptr(actions, torch.uint8, (k, B), "actions")
    pr = _dev_ptr(rewards, torch.float32, (k, B), "rewards")
    pd = _dev_ptr(done, torch.uint8, (k, B), "done")
    po = _dev_ptr(obs, torch.uint8, (B, C, w, w), "obs")
    _check("av_step_observe", load_library().av_step_observe(batch, k, pa, pr, pd, w, po))


def av_get_maps(batch, dst):
    info = av_get_info(batch)
    shp = (info["num_envs"], info["channels"], info["height"], info["width"])
    torch = _torch()
    _check("av_get_maps", load_library().av_get_maps(batch, _dev_ptr(dst, torch.uint8, shp, "dst")))


def av_observe(batch, w, dst):
    """dst: device uint8 tensor [B][C][w][w]."""
    info = av_get_info(batch)
    shp = (info["num_envs"], info["channels"], w, w)
    torch = _torch()
    _check("av_observe", load_library().av_observe(batch, int(w),
                                                   _dev_ptr(dst, torch.uint8, shp, "dst")))


def av_rule_features(batch, dst):
    """dst: device uint8 tensor [S][R][2][2][C+1][max_pat_h][max_pat_w] (contiguous)."""
    torch = _torch()
    if not isinstance(dst, torch.Tensor) or not dst.is_cuda or dst.dtype != torch.uint8 \
            or not dst.is_contiguous():
        raise TypeError("dst must be a contiguous uint8 device tensor")
    _check("av_rule_features", load_library().av_rule_features(batch, ctypes.c_void_p(dst.data_ptr())))


def av_state_ptr(batch) -> int:
    p = load_library().av_state_ptr(batch)
    if not p:
        raise AvError("av_state_ptr", AV_EINVAL, av_last_error())
    return int(p)


def av_get_info(batch) -> dict:
    info = av_info()
    _check("av_get_info", load_library().av_get_info(batch, ctypes.byref(info)))
    return {f: getattr(info, f) for f, _ in av_info._fields_}


def av_get_state(batch) -> bytes:
    lib = load_library()
    n = ctypes.c_size_t(0)
    _check("av_get_state", lib.av_get_state(batch, None, ctypes.byref(n)))
    buf = ctypes.create_string_buffer(n.value)
    _check("av_get_state", lib.av_get_state(batch, buf, ctypes.byref(n)))
    return buf.raw[:n.value]


def av_set_state(batch, blob: bytes):
    buf = ctypes.create_string_buffer(blob, len(blob))
    _check("av_set_state", load_library().av_set_state(batch, buf, len(blob)))


def av_set_stream(batch, stream):
    if hasattr(stream, "cuda_stream"):
        stream = ctypes.c_void_p(stream.cuda_stream)
    _check("av_set_stream", load_library().av_set_stream(batch, stream))


def av_destroy_batch(batch):
    _check("av_destroy_batch", load_library().av_destroy_batch(batch))


# --- the learner's operators ----------------------------------------------------------------
#
# They read and write the given buffers, and torch's differentiation sees none of it: outputs carry no
# history and no version is counted.  A gradient is asked for (av_scan_backward,
# av_log_probs_backward) and handed on, as in logits.backward(dlogits).

# A call's host time is most of a small operator's cost, so arguments are checked with as few steps as
# will do and its config struct is packed in one (the fields of av_scan_config, av_tokens_config).
_SCAN = struct.Struct("3q4i14q2iP")
_TOKENS = struct.Struct("2q2i2q2iP")
_known = None


def _types():
    """torch's element types and token types as the library numbers them, and what else of torch
    a call needs."""
    global _known
    if _known is None:
        torch = _torch()
        _known = ({torch.float32: AV_F32, torch.float16: AV_F16, torch.bfloat16: AV_BF16},
                  {torch.uint8: AV_IDS_U8, torch.int32: AV_IDS_I32, torch.int64: AV_IDS_I64},
                  torch, torch.Tensor, torch.float32, torch._C._cuda_getCurrentRawStream)
    return _known


def _refuse(t, name, dtype, shape, device):
    if not isinstance(t, _known[3]):
        raise TypeError(f"{name} must be a device tensor")
    raise ValueError(f"{name} must be a {dtype} tensor of shape {tuple(shape)} on {device}, got "
                     f"{t.dtype} {tuple(t.shape)} on {t.device}")


def _operand(t, name, dtype, shape, device):
    """The address of a device tensor of this type, shape and device whose last dimension is
    contiguous, and its strides."""
    if not isinstance(t, _known[3]) or t.dtype is not dtype or t.shape != shape or \
            t.device != device:
        _refuse(t, name, dtype, shape, device)
    strides = t.stride()
    if strides[-1] != 1 and shape[-1] > 1:
        raise ValueError(f"the last dimension of {name} must be contiguous")
    return t.data_ptr(), strides


def _packed(t, name, dtype, shape, device):
    """The address of a contiguous device tensor of this type, shape and device, or None."""
    if t is None:
        return None
    if not isinstance(t, _known[3]) or t.dtype is not dtype or t.shape != shape or \
            t.device != device:
        _refuse(t, name, dtype, shape, device)
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t.data_ptr()


def _run(name, call, size_of, config, which, args, workspace, device):
    """Makes a call that takes a workspace: the caller's, or, where it needs one (most do not, and one
    that does is refused without before any device work), a new one from torch's allocator on the
    current stream."""
    if workspace is None:
        rc = call(config, *args, None, 0)
        if rc == AV_OK:
            return
        n = ctypes.c_size_t(0)
        if rc != AV_EINVAL or size_of(config, *which, ctypes.byref(n)) or n.value == 0:
            _check(name, call(config, *args, None, 0) if rc == AV_EINVAL else rc)
            return
        workspace = _known[2].empty(n.value, dtype=_known[2].uint8, device=device)
    elif not isinstance(workspace, _known[3]) or workspace.dtype != _known[2].uint8 or \
            not workspace.is_contiguous() or workspace.device != device:
        raise ValueError(f"workspace must be a contiguous uint8 tensor on {device}")
    _check(name, call(config, *args, workspace.data_ptr(), workspace.numel()))


def _scan_common(x, gate, cut, form):
    """Checks what both passes share: (floating type number, form, strides and address of x and
    gate, whether the gate is per value, strides and address of cut)."""
    floats, _, torch, tensor, _, _ = _types()
    if not isinstance(x, tensor) or not x.is_cuda or x.dim() != 3 or x.dtype not in floats:
        raise TypeError("x must be a float32, float16 or bfloat16 device tensor [T][B][D]")
    if not isinstance(gate, tensor):
        raise TypeError("gate must be a device tensor")
    shape, device, dtype = x.shape, x.device, x.dtype
    if shape[1] == 0 or shape[2] == 0:
        raise ValueError(f"an empty recurrence: x has shape {tuple(shape)}")
    sx = x.stride()
    if sx[2] != 1 and shape[2] > 1:
        raise ValueError("the last dimension of x must be contiguous")
    per_value = gate.dim() == 1
    pg, sg = _operand(gate, "gate", dtype, shape[2:] if per_value else shape, device)
    pc, sc = None, (0, 0)
    if cut is not None:
        if not isinstance(cut, tensor) or cut.dtype is not torch.uint8 or \
                cut.shape != shape[:2] or cut.device != device:
            _refuse(cut, "cut", torch.uint8, shape[:2], device)
        pc, sc = cut.data_ptr(), cut.stride()
    return (floats[dtype], SCAN_FORMS[form] if isinstance(form, str) else int(form), x.data_ptr(),
            sx, pg, (0, 0) if per_value else sg, 1 if per_value else 0, pc, sc)


def av_scan_workspace(steps, rows, width, gate_per_value=False, backward=False, dtype=AV_F32) -> int:
    """Bytes of workspace av_scan (or av_scan_backward) uses for these sizes (dtype: AV_F32, AV_F16
    or AV_BF16)."""
    c = av_scan_config()
    c.steps, c.rows, c.width, c.gate_per_value = steps, rows, width, int(bool(gate_per_value))
    c.dtype = dtype
    n = ctypes.c_size_t(0)
    _check("av_scan_workspace", load_library().av_scan_workspace(
        ctypes.byref(c), int(bool(backward)), ctypes.byref(n)))
    return n.value


def av_scan(x, gate, y, h0=None, last=None, cut=None, form="linear", reverse=False,
            workspace=None):
    """Gated linear recurrence over time.  x, y: device tensors [T][B][D] of one floating type, B and D
    at least 1;
    gate the same, or [D]; h0, last: float32 [B][D] or None; cut: uint8 [T][B] or None (a step
    whose flag is set starts anew).  y may be x, and last may be h0, if no gradient follows that reads
    them.  Runs on the current stream of x's device."""
    lib = load_library()
    kind, form, px, sx, pg, sg, per_value, pc, sc = _scan_common(x, gate, cut, form)
    shape, device = x.shape, x.device
    py, sy = _operand(y, "y", x.dtype, shape, device)
    f32, stream = _known[4], _known[5]
    ph = _packed(h0, "h0", f32, shape[1:], device)
    pl = _packed(last, "last", f32, shape[1:], device)
    c = _SCAN.pack(*shape, kind, form, 1 if reverse else 0, per_value, sx[0], sx[1], sg[0], sg[1],
                   sy[0], sy[1], sc[0], sc[1], 0, 0, 0, 0, 0, 0, device.index, 0,
                   stream(device.index))
    _run("av_scan", lib.av_scan, lib.av_scan_workspace, c, (0,), (px, pg, pc, ph, py, pl), workspace,
         device)


def av_scan_backward(x, gate, y, dy, dx, dgate=None, h0=None, dlast=None, dh0=None, cut=None,
                     form="linear", reverse=False, workspace=None):
    """Gradients of av_scan, called as it was (x, gate, cut and h0 with the values they had then; x is y
    where a linear one was written over x): y its output, dy and dlast the gradients of y and last; dx, dgate (like gate, or None) and dh0 (float32 [B][D], or None) are written."""
    lib = load_library()
    kind, form, px, sx, pg, sg, per_value, pc, sc = _scan_common(x, gate, cut, form)
    shape, device, dtype = x.shape, x.device, x.dtype
    py, sy = _operand(y, "y", dtype, shape, device)
    pdy, sdy = _operand(dy, "dy", dtype, shape, device)
    pdx, sdx = _operand(dx, "dx", dtype, shape, device)
    pdg, sdg = None, (0, 0)
    if per_value:
        pdg = _packed(dgate, "dgate", dtype, shape[2:], device)
    elif dgate is not None:
        pdg, sdg = _operand(dgate, "dgate", dtype, shape, device)
    f32, stream = _known[4], _known[5]
    ph = _packed(h0, "h0", f32, shape[1:], device)
    pdl = _packed(dlast, "dlast", f32, shape[1:], device)
    pdh = _packed(dh0, "dh0", f32, shape[1:], device)
    c = _SCAN.pack(*shape, kind, form, 1 if reverse else 0, per_value, sx[0], sx[1], sg[0], sg[1],
                   sy[0], sy[1], sc[0], sc[1], sdy[0], sdy[1], sdx[0], sdx[1], sdg[0], sdg[1],
                   device.index, 0, stream(device.index))
    _run("av_scan_backward", lib.av_scan_backward, lib.av_scan_workspace, c, (1,),
         (px, pg, pc, ph, py, pdy, pdl, pdx, pdg, pdh), workspace, device)


def _logits(logits):
    """The logits' address, row stride and floating type number."""
    floats, _, _, tensor, _, _ = _types()
    if not isinstance(logits, tensor) or not logits.is_cuda or logits.dim() != 2 or \
            logits.dtype not in floats:
        raise TypeError("logits must be a float32, float16 or bfloat16 device tensor [N][A]")
    strides = logits.stride()
    if strides[1] != 1 and logits.shape[1] > 1:
        raise ValueError("the last dimension of logits must be contiguous")
    return logits.data_ptr(), strides[0], floats[logits.dtype]


def _token_ids(ids, rows, device):
    """The given tokens' address and type number."""
    if ids is None:
        return None, 0
    whole = _known[1]
    if not isinstance(ids, _known[3]) or ids.dtype not in whole:
        raise TypeError("ids must be a uint8, int32 or int64 device tensor [N]")
    return _packed(ids, "ids", ids.dtype, rows, device), whole[ids.dtype]


def av_log_probs_workspace(rows, choices, top=0, dtype=AV_F32) -> int:
    """Bytes of workspace av_log_probs uses for these sizes (dtype: AV_F32, AV_F16 or AV_BF16)."""
    c = av_tokens_config()
    c.rows, c.choices, c.top, c.dtype = rows, choices, top, dtype
    n = ctypes.c_size_t(0)
    _check("av_log_probs_workspace",
           load_library().av_log_probs_workspace(ctypes.byref(c), ctypes.byref(n)))
    return n.value


def av_log_probs(logits, ids=None, logp=None, entropy=None, stats=None, top_logp=None,
                 top_ids=None, workspace=None):
    """Log-probabilities of the given tokens.  logits: device tensor [N][A]; ids: uint8, int32 or
    int64 [N] (outside [0, A): padding); logp, entropy: float32 [N]; stats: float32 [N][2], for
    av_log_probs_backward; top_logp, top_ids: float32 / int32 [N][k], the k <= 32 most likely.
    What is None is not written.  Runs on the current stream of the logits' device."""
    lib = load_library()
    pl, stride, kind = _logits(logits)
    _, _, torch, _, f32, stream = _known
    shape, device = logits.shape, logits.device
    N, row = shape[0], shape[:1]
    pi, ids_type = _token_ids(ids, row, device)
    plp = _packed(logp, "logp", f32, row, device)
    pe = _packed(entropy, "entropy", f32, row, device)
    ps = _packed(stats, "stats", f32, (N, 2), device)
    top, ptl, pti = 0, None, None
    if top_logp is not None or top_ids is not None:
        if top_logp is None or top_ids is None or top_logp.dim() != 2:
            raise ValueError("top_logp and top_ids [N][k] go together")
        top = top_logp.shape[1]
        ptl = _packed(top_logp, "top_logp", f32, (N, top), device)
        pti = _packed(top_ids, "top_ids", torch.int32, (N, top), device)
    c = _TOKENS.pack(N, shape[1], kind, ids_type, stride, 0, top, device.index,
                     stream(device.index))
    _run("av_log_probs", lib.av_log_probs, lib.av_log_probs_workspace, c, (),
         (pl, pi, plp, pe, ps, ptl, pti), workspace, device)


def av_log_probs_backward(logits, ids, stats, entropy, dlogp, dentropy, dlogits):
    """Gradient of av_log_probs: stats and entropy as it stored them, dlogp and dentropy float32
    [N] or None (then ids, or entropy, may be None too), dlogits like logits; it may be logits."""
    lib = load_library()
    pl, stride, kind = _logits(logits)
    f32, stream = _known[4], _known[5]
    shape, device = logits.shape, logits.device
    row = shape[:1]
    pi, ids_type = _token_ids(ids, row, device)
    pd, sd = _operand(dlogits, "dlogits", logits.dtype, shape, device)
    c = _TOKENS.pack(shape[0], shape[1], kind, ids_type, stride, sd[0], 0, device.index,
                     stream(device.index))
    rc = lib.av_log_probs_backward(
        c, pl, pi, _packed(stats, "stats", f32, (row[0], 2), device),
        _packed(entropy, "entropy", f32, row, device), _packed(dlogp, "dlogp", f32, row, device),
        _packed(dentropy, "dentropy", f32, row, device), pd)
    if rc:
        _check("av_log_probs_backward", rc)


def av_draw_actions(logits, uniform, actions, logp=None):
    """Draw an action per row of logits [N][A], A <= 256: uniform float32 [N] in [0, 1), actions
    uint8 [N], logp float32 [N] or None."""
    lib = load_library()
    pl, stride, kind = _logits(logits)
    _, _, torch, _, f32, raw_stream = _known
    shape, device = logits.shape, logits.device
    row = shape[:1]
    pu = _packed(uniform, "uniform", f32, row, device)
    pa = _packed(actions, "actions", torch.uint8, row, device)
    plp = _packed(logp, "logp", f32, row, device)
    c = _TOKENS.pack(shape[0], shape[1], kind, 0, stride, 0, 0, device.index,
                     raw_stream(device.index))
    rc = lib.av_draw_actions(c, pl, pu, pa, plp)
    if rc:
        _check("av_draw_actions", rc)


class Batch:
    """A batch of B environments on one GPU, with reusable device buffers for actions,
    rewards and done flags."""

    def __init__(self, num_envs, height, width, channels, max_rules, max_pat_h, max_pat_w,
                 per_env_rules=False, max_episode_steps=0, device=None, engine="auto",
                 rule_mode="parallel"):
        torch = _torch()
        self.device = torch.device("cuda", torch.cuda.current_device() if device is None
                                   else device)
        self.B, self.H, self.W, self.C = num_envs, height, width, channels
        self.h = av_create_batch(num_envs, height, width, channels, max_rules, max_pat_h,
                                 max_pat_w, per_env_rules, max_episode_steps,
                                 self.device.index, engine, rule_mode=rule_mode)
        self.rewards = torch.zeros(num_envs, dtype=torch.float32, device=self.device)
        self.done = torch.zeros(num_envs, dtype=torch.uint8, device=self.device)

    @classmethod
    def for_workload(cls, wl, B=None, device=None, engine="auto", rule_mode="parallel"):
        return cls(wl.B if B is None else B, wl.H, wl.W, wl.C, wl.R, wl.max_h, wl.max_w,
                   wl.per_env, wl.L, device=device, engine=engine, rule_mode=rule_mode)

    @property
    def info(self):
        return av_get_info(self.h)

    def load_rules(self, shape, in_pat, out_pat, reward):
        av_load_rules(self.h, shape, in_pat, out_pat, reward)
        self.S, self.R = (np.shape(shape)[0], np.shape(shape)[1]) if np.ndim(shape) == 3 \
            else (1, 0)

    def set_rule_control(self, limit=None, inhibit=None, order="rowmajor", seed=0):
        S, R = getattr(self, "S", 1), getattr(self, "R", 0)
        if limit is not None and np.shape(limit) != (S, R):
            raise ValueError(f"limit must have shape {(S, R)}, got {np.shape(limit)}")
        if inhibit is not None and np.shape(inhibit) != (S, R, R):
            raise ValueError(f"inhibit must have shape {(S, R, R)}, got {np.shape(inhibit)}")
        av_set_rule_control(self.h, limit, inhibit, order, seed)

    def reset(self, init_maps):
        torch = _torch()
        if not isinstance(init_maps, torch.Tensor):
            init_maps = torch.from_numpy(np.ascontiguousarray(init_maps, dtype=np.uint8))
        av_reset(self.h, init_maps.to(self.device).contiguous())

    def step(self, actions):
        """actions: uint8 device tensor [B]; returns this batch's (rewards, done) tensors."""
        av_step(self.h, actions, self.rewards, self.done)
        return self.rewards, self.done

    def step_n(self, actions, rewards=None, done=None):
        """actions [k][B] uint8 on the device; returns rewards [k][B], done [k][B]."""
        torch = _torch()
        k = actions.shape[0]
        if rewards is None:
            rewards = torch.empty((k, self.B), dtype=torch.float32, device=self.device)
        if done is None:
            done = torch.empty((k, self.B), dtype=torch.uint8, device=self.device)
        av_step_n(self.h, k, actions, rewards, done)
        return rewards, done

    def step_observe(self, actions, w, obs=None, rewards=None, done=None):
        """actions [k][B] on the device; returns (rewards [k][B], done [k][B], obs [B][C][w][w])
        with obs taken after the k-th step."""
        torch = _torch()
        k = actions.shape[0]
        if rewards is None:
            rewards = torch.empty((k, self.B), dtype=torch.float32, device=self.device)
        if done is None:
            done = torch.empty((k, self.B), dtype=torch.uint8, device=self.device)
        if obs is None:
            obs = torch.empty((self.B, self.C, w, w), dtype=torch.uint8, device=self.device)
        av_step_observe(self.h, k, actions, rewards, done, w, obs)
        return rewards, done, obs

    def act(self, logits, uniform, actions=None, logp=None):
        """Draw every environment's action for the next step: logits [B][A] and uniform numbers
        float32 [B] on the device; returns (actions uint8 [B], their log-probabilities [B], which
        carry no history of torch's).  Runs on torch's current stream."""
        torch = _torch()
        if tuple(logits.shape[:1]) != (self.B,):
            raise ValueError(f"logits must have {self.B} rows, got {tuple(logits.shape)}")
        if actions is None:
            actions = torch.empty(self.B, dtype=torch.uint8, device=self.device)
        if logp is None:
            logp = torch.empty(self.B, dtype=torch.float32, device=self.device)
        av_draw_actions(logits, uniform, actions, logp)
        return actions, logp

    def returns(self, rewards, done, gamma, after=None, out=None):
        """Discounted returns of a rollout: rewards float32 [k][B] (or temporal-difference errors,
        for advantages) and done [k][B] as step_n gives them, gamma a float32 device tensor [1] or a
        number (which every call copies into one), after float32 [B] the value of what follows the
        last step (or None); returns out [k][B], out[t] = rewards[t] + gamma (1 - done[t]) out[t + 1].
        Runs on torch's current stream."""
        torch = _torch()
        if rewards.dim() != 2 or rewards.shape[1] != self.B:
            raise ValueError(f"rewards must be [k][{self.B}], got {tuple(rewards.shape)}")
        if not isinstance(gamma, torch.Tensor):
            gamma = torch.full((1,), gamma, dtype=torch.float32, device=self.device)
        if out is None:
            out = torch.empty_like(rewards)
        av_scan(rewards[:, :, None], gamma, out[:, :, None],
                h0=None if after is None else after[:, None], cut=done, reverse=True)
        return out

    def maps(self, out=None):
        torch = _torch()
        if out is None:
            out = torch.empty((self.B, self.C, self.H, self.W), dtype=torch.uint8,
                              device=self.device)
        av_get_maps(self.h, out)
        return out

    def observe(self, w, out=None):
        torch = _torch()
        if out is None:
            out = torch.empty((self.B, self.C, w, w), dtype=torch.uint8, device=self.device)
        av_observe(self.h, w, out)
        return out

    def state_ptr(self) -> int:
        return av_state_ptr(self.h)

    def get_state(self) -> bytes:
        return av_get_state(self.h)

    def set_state(self, blob: bytes):
        av_set_state(self.h, blob)

    def close(self):
        if getattr(self, "h", None) is not None:
            av_destroy_batch(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class Search:
    """Level-synchronous search over action sequences on one GPU (av_search_*): every level
    steps all (frontier node, action) pairs as one batch and deduplicates states in a device
    hash table.  The methods marshal arguments only."""

    def __init__(self, height, width, channels, max_rules, max_pat_h, max_pat_w,
                 max_episode_steps=0, num_actions=5, max_frontier=1 << 16, table_log2=20,
                 device=None, engine="auto", rule_mode="parallel", best_first_k=0,
                 max_nodes=1 << 20, hash_bits=0):
        torch = _torch()
        self.device = torch.device("cuda", torch.cuda.current_device() if device is None
                                   else device)
        self.H, self.W, self.C = height, width, channels
        cfg = av_search_config(height, width, channels, max_rules, max_pat_h, max_pat_w,
                               max_episode_steps, num_actions, max_frontier, table_log2,
                               self.device.index, ENGINES[engine] if isinstance(engine, str)
                               else engine, RULE_MODES[rule_mode] if isinstance(rule_mode, str)
                               else rule_mode, best_first_k, max_nodes, hash_bits,
                               current_stream_handle())
        h = ctypes.c_void_p()
        _check("av_search_create", load_library().av_search_create(ctypes.byref(cfg),
                                                                   ctypes.byref(h)))
        self.h = h
        self.n_front = 0

    def load_rules(self, shape, in_pat, out_pat, reward):
        shape, ps = _host(shape, np.int32, "shape")
        in_pat, pi = _host(in_pat, np.int8, "in_pat")
        out_pat, po = _host(out_pat, np.int8, "out_pat")
        reward, pr = _host(reward, np.int32, "reward")
        if shape.ndim == 3 and shape.shape[0] != 1:
            raise ValueError("a search takes one rule set (S = 1)")
        R = shape.shape[1] if shape.ndim == 3 else 0
        _check("av_search_load_rules",
               load_library().av_search_load_rules(self.h, R, ps, pi, po, pr))

    def begin(self, root):
        torch = _torch()
        if not isinstance(root, torch.Tensor):
            root = torch.from_numpy(np.ascontiguousarray(root, dtype=np.uint8))
        root = root.to(self.device).contiguous()
        p = _dev_ptr(root, torch.uint8, (self.C, self.H, self.W), "root")
        _check("av_search_begin", load_library().av_search_begin(self.h, p))
        self.n_front = 1

    def expand(self, max_children) -> dict:
        info = av_search_info()
        _check("av_search_expand",
               load_library().av_search_expand(self.h, int(max_children), ctypes.byref(info)))
        self.n_front = info.frontier
        return {k: getattr(info, k) for k, _ in av_search_info._fields_ if k != "reserved"}

    def frontier(self):
        """(maps uint8 [N][C][H][W], reward int32 [N], depth int32 [N]) device tensors."""
        torch = _torch()
        n = self.n_front
        maps = torch.empty((n, self.C, self.H, self.W), dtype=torch.uint8, device=self.device)
        reward = torch.empty(n, dtype=torch.int32, device=self.device)
        depth = torch.empty(n, dtype=torch.int32, device=self.device)
        if n:
            _check("av_search_frontier", load_library().av_search_frontier(
                self.h, ctypes.c_void_p(maps.data_ptr()), ctypes.c_void_p(reward.data_ptr()),
                ctypes.c_void_p(depth.data_ptr())))
        return maps, reward, depth

    def run(self, root, budget, max_levels=1 << 30):
        self.begin(root)
        out = []
        visited = 0
        while self.n_front and visited < budget and len(out) < max_levels:
            info = self.expand(budget - visited)
            visited = info["visited"]
            out.append(info)
        return out

    def close(self):
        if getattr(self, "h", None) is not None:
            load_library().av_search_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
