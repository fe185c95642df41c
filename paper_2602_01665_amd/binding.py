"""Thin Python binding of libtabx.so (the C ABI declared in include/tabx.h).

Argument marshalling only: every stage of the environment tick runs inside the
HIP kernels.  PyTorch owns the device memory and the stream; this module turns
tensors into the pointer structs the library takes.  There is no CPU fallback:
if the library has not been built, importing fails loudly.
"""
from __future__ import annotations

import ctypes as C
import os

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libtabx.so")

_F = C.POINTER(C.c_float)
_U8 = C.POINTER(C.c_uint8)

SCENARIO_FLOAT = ("init_x", "init_y", "init_theta", "hmax", "radius", "mass", "speed", "dmg",
                  "range", "cooldown", "sight_angle", "sight_cos_half", "sight_range",
                  "hurt_halfwidth")
STATE_FLOAT = ("x", "y", "vx", "vy", "theta", "hp", "cd", "reveal", "cur_speed")

EXPORTS = ("tabx_obs_dim", "tabx_num_actions", "tabx_reset", "tabx_step", "tabx_observe",
           "tabx_step_observe", "tabx_global_state", "tabx_heuristic_actions",
           "tabx_policy_step_observe", "tabx_scripted_step_observe", "tabx_part", "tabx_launch_info",
           "tabx_row_form", "tabx_layer_norm", "tabx_layer_norm_backward",
           "tabx_layer_norm_workspace", "tabx_sample_actions", "tabx_sample_levels",
           "tabx_action_log_prob", "tabx_action_log_prob_backward", "tabx_strerror")

_I8 = C.POINTER(C.c_int8)
_I32 = C.POINTER(C.c_int32)
METRICS = (("ret_run", _F, torch.float32), ("kill_run", _I8, torch.int8),
           ("ep_count", _I32, torch.int32), ("ep_len", _I32, torch.int32),
           ("ep_return", _F, torch.float32), ("ep_win", _I8, torch.int8),
           ("ep_first_kill", _I8, torch.int8))


LEVELS = ("level", "next_level", "level_draws")


class TabxParams(C.Structure):
    _fields_ = [(n, C.c_int32) for n in
                ("num_envs", "num_units", "grid_w", "grid_h", "max_zones", "max_steps")] + \
               [(n, C.c_float) for n in
                ("map_w", "map_h", "cell_size", "dt", "turn_rate", "lava_dps", "swamp_mult",
                 "reveal_time", "boundary_frac", "collision_alpha", "collision_slop")] + \
               [("zone_shapes", C.c_int32), ("num_levels", C.c_int32), ("level_seed", C.c_uint32),
                ("hurtbox_cone", C.c_int32), ("hit_all", C.c_int32),
                ("env_id_offset", C.c_int32), ("dynamics", C.c_int32),
                ("move_gain", C.c_float), ("restitution", C.c_float),
                ("shared_machine", C.c_int32)]


class TabxScenario(C.Structure):
    _fields_ = [(n, _F) for n in SCENARIO_FLOAT] + \
               [("team", _U8), ("enabled", _U8), ("terrain", C.POINTER(C.c_int8)),
                ("zone_desc", _F)]


class TabxState(C.Structure):
    _fields_ = [(n, _F) for n in STATE_FLOAT] + \
               [("alive", _U8), ("t", C.POINTER(C.c_int32)), ("phi_prev", _F)] + \
               [(n, t) for n, t, _ in METRICS] + \
               [(n, _I32) for n in LEVELS] + [("global_state", _F), ("ax", _F), ("ay", _F)]


class TabxError(RuntimeError):
    pass


class TabxPolicy(C.Structure):
    _fields_ = [("epsilon", C.c_float), ("xi", C.c_float), ("assassin_speed", C.c_float),
                ("ranger_range", C.c_float), ("seed", C.c_uint32)]


class TabxPolicyMemory(C.Structure):
    _fields_ = [("mem_x", _F), ("mem_y", _F), ("mem_valid", _U8), ("next_action", _U8)]


class TabxRows(C.Structure):
    _fields_ = [("data", C.c_void_p), ("stride", C.c_int64), ("type", C.c_int32)]


class TabxSampling(C.Structure):
    """How a choice is drawn: temperature (0: the largest score), top_k (0: all), top_p (1: all),
    min_p (0: all)."""
    _fields_ = [("temperature", C.c_double), ("top_k", C.c_int32), ("top_p", C.c_float),
                ("min_p", C.c_float)]

    def __init__(self, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
        # more choices than there can be are all; what 32 bits do not hold would be cut off
        super().__init__(temperature, max(-1, min(top_k, 2 ** 31 - 1)), top_p, min_p)


def load_library(path: str = LIB_PATH) -> C.CDLL:
    if not os.path.exists(path):
        raise ImportError(
            f"{path} is missing: build it with `python -m paper_2602_01665_amd.build` "
            "(hipcc, gfx950).  There is no fallback path.")
    lib = C.CDLL(path)
    P, S, T, V = C.POINTER(TabxParams), C.POINTER(TabxScenario), C.POINTER(TabxState), C.c_void_p
    lib.tabx_obs_dim.argtypes = [P]
    lib.tabx_num_actions.argtypes = []
    lib.tabx_reset.argtypes = [P, S, T, V, V]
    lib.tabx_step.argtypes = [P, S, T, V, V, V, V]
    lib.tabx_observe.argtypes = [P, S, T, V, V, V, V]
    lib.tabx_step_observe.argtypes = [P, S, T, V, V, V, V, V, V, V]
    lib.tabx_global_state.argtypes = [P, S, T, V, V]
    lib.tabx_heuristic_actions.argtypes = [P, S, T, C.POINTER(TabxPolicy),
                                           C.POINTER(TabxPolicyMemory), V, V, V]
    lib.tabx_policy_step_observe.argtypes = [P, S, T, C.POINTER(TabxPolicy),
                                             C.POINTER(TabxPolicyMemory)] + [V] * 8
    lib.tabx_scripted_step_observe.argtypes = lib.tabx_policy_step_observe.argtypes
    lib.tabx_strerror.argtypes = [C.c_int]
    lib.tabx_strerror.restype = C.c_char_p
    R, W, I64, I32 = C.POINTER(TabxRows), C.POINTER(TabxSampling), C.c_int64, C.c_int32
    F32, F64 = C.c_float, C.c_double
    lib.tabx_layer_norm.argtypes = [I64, I32, R, V, V, V, F32, R, V, V, V]
    lib.tabx_layer_norm_backward.argtypes = [I64, I32, R, V, V, V, V, R, R, V, V, V, I64, V]
    lib.tabx_layer_norm_workspace.argtypes = [I64, I32]
    lib.tabx_sample_actions.argtypes = [I64, R, V, V, W, V, V, V, V]
    lib.tabx_sample_levels.argtypes = [I64, I32, R, V, V, W, V, V, V]
    lib.tabx_action_log_prob.argtypes = [I64, R, V, V, V, F64, V, V, V]
    lib.tabx_action_log_prob_backward.argtypes = [I64, R, V, V, V, F64, V, V, R, V]
    for name in EXPORTS[:-1]:
        getattr(lib, name).restype = C.c_int
    lib.tabx_layer_norm_workspace.restype = I64
    return lib


_lib = load_library()


def _check(rc: int, what: str):
    if rc != 0:
        raise TabxError(f"{what}: {_lib.tabx_strerror(rc).decode()} ({rc})")


def _ptr(t):
    return None if t is None else C.c_void_p(t.data_ptr())


def _cast(t, typ):
    return C.cast(C.c_void_p(t.data_ptr()), typ) if t is not None else C.cast(None, typ)


def make_params(p: dict) -> TabxParams:
    return TabxParams(**{k: p.get(k, 0) for k, _ in TabxParams._fields_})


def tabx_obs_dim(params: TabxParams) -> int:
    d = _lib.tabx_obs_dim(C.byref(params))
    if d < 0:
        _check(d, "tabx_obs_dim")
    return d


def tabx_part(params: TabxParams, scenario: TabxScenario, state: TabxState, first_env: int,
              count: int):
    """The structs of the envs [first_env, first_env + count) of a batch."""
    pp, psc, pst = TabxParams(), TabxScenario(), TabxState()
    _check(_lib.tabx_part(C.byref(params), C.byref(scenario), C.byref(state), int(first_env),
                          int(count), C.byref(pp), C.byref(psc), C.byref(pst)), "tabx_part")
    return pp, psc, pst


class TabxLaunchInfo(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("workgroups", "threads_per_workgroup", "envs_per_workgroup",
                                          "wavefronts_per_env_group", "rows_per_flush",
                                          "dynamic_lds_bytes", "assumed_compute_units",
                                          "assumed_lds_per_cu_bytes",
                                          "assumed_lds_per_workgroup_bytes",
                                          "assumed_wavefront_lanes")]


CALLS = {"reset": 0, "step": 1, "observe": 2, "step_observe": 3, "heuristic_actions": 4,
         "policy_step_observe": 5, "scripted_step_observe": 6}


def tabx_launch_info(params: TabxParams, call: str) -> dict:
    """How the library would lay the call out (host only, nothing is enqueued)."""
    info = TabxLaunchInfo()
    _check(_lib.tabx_launch_info(C.byref(params), CALLS[call], C.byref(info)), "tabx_launch_info")
    return {n: getattr(info, n) for n, _ in TabxLaunchInfo._fields_}


class TabxRowForm(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("lines", "pace", "wavefronts_per_simd", "streams_global_state")]


def tabx_row_form(params: TabxParams, call: str) -> dict:
    """Which form of the row writers the call takes (host only, nothing is enqueued)."""
    form = TabxRowForm()
    _check(_lib.tabx_row_form(C.byref(params), CALLS[call], C.byref(form)), "tabx_row_form")
    return {n: getattr(form, n) for n, _ in TabxRowForm._fields_}


def tabx_num_actions() -> int:
    return _lib.tabx_num_actions()


def _stream_ptr(stream):
    if stream is None:
        stream = torch.cuda.current_stream()
    return C.c_void_p(stream.cuda_stream)


def tabx_reset(params, scenario, state, env_mask=None, stream=None):
    _check(_lib.tabx_reset(C.byref(params), C.byref(scenario), C.byref(state), _ptr(env_mask),
                           _stream_ptr(stream)), "tabx_reset")


def tabx_step(params, scenario, state, actions, rewards, dones, stream=None):
    _check(_lib.tabx_step(C.byref(params), C.byref(scenario), C.byref(state), _ptr(actions),
                          _ptr(rewards), _ptr(dones), _stream_ptr(stream)), "tabx_step")


def tabx_observe(params, scenario, state, obs, vis_mask=None, action_mask=None, stream=None):
    _check(_lib.tabx_observe(C.byref(params), C.byref(scenario), C.byref(state), _ptr(obs),
                             _ptr(vis_mask), _ptr(action_mask), _stream_ptr(stream)),
           "tabx_observe")


def tabx_step_observe(params, scenario, state, actions, rewards, dones, obs, vis_mask=None,
                      action_mask=None, stream=None):
    _check(_lib.tabx_step_observe(C.byref(params), C.byref(scenario), C.byref(state),
                                  _ptr(actions), _ptr(rewards), _ptr(dones), _ptr(obs),
                                  _ptr(vis_mask), _ptr(action_mask), _stream_ptr(stream)),
           "tabx_step_observe")


def tabx_global_state(params, scenario, state, out, stream=None):
    _check(_lib.tabx_global_state(C.byref(params), C.byref(scenario), C.byref(state), _ptr(out),
                                  _stream_ptr(stream)), "tabx_global_state")


def tabx_heuristic_actions(params, scenario, state, policy, memory, controlled, actions,
                           stream=None):
    _check(_lib.tabx_heuristic_actions(C.byref(params), C.byref(scenario), C.byref(state),
                                       C.byref(policy), C.byref(memory), _ptr(controlled),
                                       _ptr(actions), _stream_ptr(stream)),
           "tabx_heuristic_actions")


def tabx_policy_step_observe(params, scenario, state, policy, memory, controlled, actions,
                             rewards, dones, obs, vis_mask=None, action_mask=None, stream=None):
    _check(_lib.tabx_policy_step_observe(C.byref(params), C.byref(scenario), C.byref(state),
                                         C.byref(policy), C.byref(memory), _ptr(controlled),
                                         _ptr(actions), _ptr(rewards), _ptr(dones), _ptr(obs),
                                         _ptr(vis_mask), _ptr(action_mask), _stream_ptr(stream)),
           "tabx_policy_step_observe")


def tabx_scripted_step_observe(params, scenario, state, policy, memory, controlled, actions,
                               rewards, dones, obs, vis_mask=None, action_mask=None, stream=None):
    _check(_lib.tabx_scripted_step_observe(C.byref(params), C.byref(scenario), C.byref(state),
                                           C.byref(policy), C.byref(memory), _ptr(controlled),
                                           _ptr(actions), _ptr(rewards), _ptr(dones), _ptr(obs),
                                           _ptr(vis_mask), _ptr(action_mask),
                                           _stream_ptr(stream)),
           "tabx_scripted_step_observe")


# --- the learner's side of the tick: tensors of its own, checked before their addresses are taken ---

TYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
_MOST = 2 ** 31 - 1                     # (ctypes would cut off what a 32-bit argument does not hold)


# The calls are not part of PyTorch's graph: inputs count as detached, and each way back is a call of its own.
# What a call on a few thousand rows costs is the time until it is enqueued: the checks are plain
# functions of few steps (a small tabx_sample_actions takes the host 6.4 us, 0.1 of them to tell PyTorch what
# was written; 10.1 as methods of an object with torch.cuda.current_stream()).  `device` is that of a call's first tensor, -1 the host.


def _refuse(what, why):
    raise TabxError(f"{what}: {why}")


def _elsewhere(what, t, name, device):
    place = "cpu" if device < 0 else f"cuda:{device}"
    _refuse(what, f"{name} is on {t.device}, not on {place}")


def _rows(what, t, name, width, device=None):
    """(TabxRows, rows) of a tensor [..., width] whose rows lie at equal distances."""
    code = TYPES.get(t.dtype)
    if code is None:
        _refuse(what, f"{name} is {t.dtype}, not one of float32, bfloat16, float16")
    shape = t.shape
    if not shape:
        _refuse(what, f"{name} has no dimensions")
    wide = shape[-1]
    if wide != width and width:
        _refuse(what, f"{name} has rows of {wide} elements, not {width}")
    if wide > _MOST:
        _refuse(what, f"{name} has rows of {wide} elements")
    if device is not None and t.get_device() != device:
        _elsewhere(what, t, name, device)
    if t.is_contiguous():
        return TabxRows(t.data_ptr(), wide, code), t.numel() // wide if wide else 0
    stride = t.stride()
    if wide > 1 and stride[-1] != 1:
        _refuse(what, f"the elements of a row of {name} are not next to each other")
    count, apart = 1, 0
    for k in range(len(shape) - 2, -1, -1):    # the leading dimensions have to be one run of rows
        if shape[k] == 1:
            continue
        if count == 1:
            apart = stride[k]
        elif stride[k] != apart * count:
            _refuse(what, f"the rows of {name} do not lie at equal distances")
        count *= shape[k]
    if count > 1 and apart < wide:
        _refuse(what, f"the rows of {name} overlap")
    return TabxRows(t.data_ptr(), max(apart, wide), code), count


def _same_rows(what, t, name, width, device, rows):
    """The same for a tensor that has to have as many rows."""
    r, n = _rows(what, t, name, width, device)
    if n != rows:
        _refuse(what, f"{name} has {n} rows, not {rows}")
    return r


def _array(what, t, name, count, dtype, device):
    """Address of a contiguous tensor of `count` elements, None for None."""
    if t is None:
        return None
    if t.dtype is not dtype:
        _refuse(what, f"{name} is {t.dtype}, not {dtype}")
    if t.numel() != count:
        _refuse(what, f"{name} has {t.numel()} elements, not {count}")
    if not t.is_contiguous():
        _refuse(what, f"{name} is not contiguous")
    if t.get_device() != device:
        _elsewhere(what, t, name, device)
    return t.data_ptr()


def _needed(what, t, name, count, dtype, device):
    if t is None:
        _refuse(what, f"{name} is needed")
    return _array(what, t, name, count, dtype, device)


def _enqueue(what, function, device, stream, written, *args):
    """Makes the call; `written`: the tensors it writes (or None), of which PyTorch's graph is told, so that a
    backward pass that needs what they held before is refused, as after PyTorch's own calls in place."""
    if device < 0:
        _refuse(what, "the tensors are not on a GPU")
    if stream is None:
        raw = torch._C._cuda_getCurrentRawStream(device)
    elif stream.device_index == device:
        raw = stream.cuda_stream
    else:
        _refuse(what, f"the stream is on {stream.device}, the tensors are on cuda:{device}")
    if torch._C._cuda_getDevice() == device:
        rc = function(*args, raw)
    else:
        with torch.cuda.device(device):
            rc = function(*args, raw)
    if rc != 0:
        _check(rc, what)
    torch._C._increment_version([t for t in written if t is not None])


def tabx_layer_norm(x, weight, bias, eps, y, mean=None, rstd=None, row_mask=None, stream=None):
    """y = layer norm of the rows of x (over the last dimension) whose row_mask byte is not 0.  Other rows
    of y keep what they hold: finite values, where a product will read them too."""
    what, f32, dev = "tabx_layer_norm", torch.float32, x.get_device()
    xr, rows = _rows(what, x, "x", 0)
    width = x.shape[-1]
    yr = _same_rows(what, y, "y", width, dev, rows)
    _enqueue(what, _lib.tabx_layer_norm, dev, stream, (y, mean, rstd), rows, width, C.byref(xr),
             _array(what, row_mask, "row_mask", rows, torch.uint8, dev),
             _array(what, weight, "weight", width, f32, dev),
             _array(what, bias, "bias", width, f32, dev), eps, C.byref(yr),
             _array(what, mean, "mean", rows, f32, dev),
             _array(what, rstd, "rstd", rows, f32, dev))


def tabx_layer_norm_workspace(rows: int, width: int) -> int:
    """Bytes of workspace that tabx_layer_norm_backward needs for the weight's and bias's gradients."""
    if not (-1 <= width <= _MOST and -1 <= rows < 2 ** 63):
        _refuse("tabx_layer_norm_workspace", f"{rows} rows of {width} elements")
    n = _lib.tabx_layer_norm_workspace(rows, width)
    if n < 0:
        _check(n, "tabx_layer_norm_workspace")
    return n


def tabx_layer_norm_backward(x, weight, mean, rstd, grad_y, grad_x=None, grad_weight=None,
                             grad_bias=None, workspace=None, row_mask=None, stream=None):
    """The gradients of tabx_layer_norm; those that are None are not computed."""
    what, f32, dev = "tabx_layer_norm_backward", torch.float32, x.get_device()
    xr, rows = _rows(what, x, "x", 0)
    width = x.shape[-1]
    gr = _same_rows(what, grad_y, "grad_y", width, dev, rows)
    ir = None
    if grad_x is not None:
        ir = C.byref(_same_rows(what, grad_x, "grad_x", width, dev, rows))
    size = 0 if workspace is None else workspace.numel()
    _enqueue(what, _lib.tabx_layer_norm_backward, dev, stream, (grad_x, grad_weight, grad_bias), rows,
             width, C.byref(xr),
             _array(what, row_mask, "row_mask", rows, torch.uint8, dev),
             _array(what, weight, "weight", width, f32, dev),
             _needed(what, mean, "mean", rows, f32, dev),
             _needed(what, rstd, "rstd", rows, f32, dev), C.byref(gr), ir,
             _array(what, grad_weight, "grad_weight", width, f32, dev),
             _array(what, grad_bias, "grad_bias", width, f32, dev),
             _array(what, workspace, "workspace", size, torch.uint8, dev), size)


def tabx_sample_actions(logits, sampling, uniform, actions, log_prob=None, action_mask=None,
                        controlled=None, stream=None):
    """Draws an action from each unit's eight logits, into `actions` (uint8, in place)."""
    what, f32, u8, dev = "tabx_sample_actions", torch.float32, torch.uint8, logits.get_device()
    lr, rows = _rows(what, logits, "logits", 8)
    _enqueue(what, _lib.tabx_sample_actions, dev, stream, (actions, log_prob), rows, C.byref(lr),
             _array(what, action_mask, "action_mask", rows, u8, dev),
             _array(what, controlled, "controlled", rows, u8, dev), C.byref(sampling),
             _needed(what, uniform, "uniform", rows, f32, dev),
             _needed(what, actions, "actions", rows, u8, dev),
             _array(what, log_prob, "log_prob", rows, f32, dev))


def tabx_sample_levels(scores, sampling, uniform, next_level, level_mask=None, env_mask=None,
                       stream=None):
    """Draws each env's next level from scores [levels] of all envs or [envs, levels] of each."""
    what, u8, dev = "tabx_sample_levels", torch.uint8, scores.get_device()
    if next_level is None:
        _refuse(what, "next_level is needed")
    envs, n = next_level.numel(), scores.dim()
    if n > 2:
        _refuse(what, f"scores has {n} dimensions")
    if n == 2:
        if scores.shape[0] != envs:
            _refuse(what, f"scores has {scores.shape[0]} rows, next_level {envs} elements")
        if envs and scores.stride(0) == 0:     # one row, expanded
            scores, n = scores[0], 1
    sr, _ = _rows(what, scores, "scores", 0)
    levels = scores.shape[-1]
    if n == 1:
        sr.stride = 0
    _enqueue(what, _lib.tabx_sample_levels, dev, stream, (next_level,), envs, levels, C.byref(sr),
             _array(what, level_mask, "level_mask", levels, u8, dev),
             _array(what, env_mask, "env_mask", envs, u8, dev), C.byref(sampling),
             _needed(what, uniform, "uniform", envs, torch.float32, dev),
             _needed(what, next_level, "next_level", envs, torch.int32, dev))


def tabx_action_log_prob(logits, actions, temperature, log_prob, entropy=None, action_mask=None,
                         controlled=None, stream=None):
    """log_prob (and entropy) of the actions under the distribution of their logits."""
    what, f32, u8, dev = "tabx_action_log_prob", torch.float32, torch.uint8, logits.get_device()
    lr, rows = _rows(what, logits, "logits", 8)
    _enqueue(what, _lib.tabx_action_log_prob, dev, stream, (log_prob, entropy), rows, C.byref(lr),
             _array(what, action_mask, "action_mask", rows, u8, dev),
             _array(what, controlled, "controlled", rows, u8, dev),
             _needed(what, actions, "actions", rows, u8, dev), temperature,
             _needed(what, log_prob, "log_prob", rows, f32, dev),
             _array(what, entropy, "entropy", rows, f32, dev))


def tabx_action_log_prob_backward(logits, actions, temperature, grad_log_prob, grad_entropy,
                                  grad_logits, action_mask=None, controlled=None, stream=None):
    """The logits' gradient, from those of log_prob and entropy (either may be None: zero)."""
    what, f32, u8 = "tabx_action_log_prob_backward", torch.float32, torch.uint8
    dev = logits.get_device()
    lr, rows = _rows(what, logits, "logits", 8)
    gr = _same_rows(what, grad_logits, "grad_logits", 8, dev, rows)
    _enqueue(what, _lib.tabx_action_log_prob_backward, dev, stream, (grad_logits,), rows, C.byref(lr),
             _array(what, action_mask, "action_mask", rows, u8, dev),
             _array(what, controlled, "controlled", rows, u8, dev),
             _needed(what, actions, "actions", rows, u8, dev), temperature,
             _array(what, grad_log_prob, "grad_log_prob", rows, f32, dev),
             _array(what, grad_entropy, "grad_entropy", rows, f32, dev), C.byref(gr))


class TabxEnv:
    """Device buffers of one batch of environments plus the calls on them."""

    def __init__(self, params: dict, scenario: dict, device="cuda:0", want_vis=True,
                 want_action_mask=True, want_metrics=False, want_global_state=False):
        self.device = torch.device(device)
        self.p = dict(params)
        self.params = make_params(self.p)
        E, N = self.p["num_envs"], self.p["num_units"]
        self.E, self.N = E, N
        L = self.p.get("num_levels", 0)
        rows = L if L > 0 else E           # scenario rows: a bank of levels, or one per env
        self.D = tabx_obs_dim(self.params)
        self.words = (N + 63) // 64
        dev = self.device

        def up(a, dtype):
            return torch.as_tensor(a, dtype=dtype).contiguous().to(dev)

        self.sc = {k: up(scenario[k], torch.float32).reshape(rows * N) for k in SCENARIO_FLOAT}
        self.sc["team"] = up(scenario["team"], torch.uint8).reshape(rows * N)
        self.sc["enabled"] = up(scenario["enabled"], torch.uint8).reshape(rows * N)
        ter = scenario.get("terrain")
        self.sc["terrain"] = None if ter is None else up(ter, torch.int8)
        zd = scenario.get("zone_desc") if self.p["max_zones"] > 0 else None
        self.sc["zone_desc"] = None if zd is None else up(zd, torch.float32)
        self.scenario = TabxScenario(
            **{k: _cast(self.sc[k], _F) for k in SCENARIO_FLOAT},
            team=_cast(self.sc["team"], _U8), enabled=_cast(self.sc["enabled"], _U8),
            terrain=_cast(self.sc["terrain"], C.POINTER(C.c_int8)),
            zone_desc=_cast(self.sc["zone_desc"], _F))

        self.st = {k: torch.zeros(E * N, dtype=torch.float32, device=dev) for k in STATE_FLOAT}
        self.st["alive"] = torch.zeros(E * N, dtype=torch.uint8, device=dev)
        self.st["t"] = torch.zeros(E, dtype=torch.int32, device=dev)
        self.st["phi_prev"] = torch.zeros(E, dtype=torch.float32, device=dev)
        self.metrics = {}
        if want_metrics:
            self.metrics = {n: torch.zeros(E, dtype=dt, device=dev) for n, _, dt in METRICS}
        if L > 0:
            self.st["level"] = torch.zeros(E, dtype=torch.int32, device=dev)
            self.st["next_level"] = (torch.arange(E, device=dev) % L).to(torch.int32)
            self.st["level_draws"] = torch.zeros(E, dtype=torch.int32, device=dev)
        if self.p.get("dynamics", 0) == 1:     # persistent velocities: the acceleration is state
            self.st["ax"] = torch.zeros(E * N, dtype=torch.float32, device=dev)
            self.st["ay"] = torch.zeros(E * N, dtype=torch.float32, device=dev)
        # global state written by every observing call (else only by global_state())
        self.gs_live = (torch.zeros(E, self.D, dtype=torch.float32, device=dev)
                        if want_global_state else None)
        self.state = self._state_struct(self.st, self.metrics, self.gs_live)
        self.gstate = None
        self.memory = None

        self.rewards = torch.zeros(E, N, dtype=torch.float32, device=dev)
        self.dones = torch.zeros(E, dtype=torch.uint8, device=dev)
        self.obs = torch.zeros(E, N, self.D, dtype=torch.float32, device=dev)
        self.vis = (torch.zeros(E, N, self.words, dtype=torch.int64, device=dev)
                    if want_vis else None)
        self.amask = (torch.zeros(E, N, dtype=torch.uint8, device=dev)
                      if want_action_mask else None)

    @staticmethod
    def _state_struct(st: dict, metrics: dict, global_state=None) -> TabxState:
        return TabxState(**{k: _cast(st[k], _F) for k in STATE_FLOAT},
                         alive=_cast(st["alive"], _U8),
                         t=_cast(st["t"], C.POINTER(C.c_int32)),
                         phi_prev=_cast(st["phi_prev"], _F),
                         **{n: _cast(metrics[n], t) for n, t, _ in METRICS if n in metrics},
                         **{n: _cast(st[n], _I32) for n in LEVELS if n in st},
                         **{n: _cast(st[n], _F) for n in ("ax", "ay") if n in st},
                         global_state=_cast(global_state, _F))

    def parts(self, k: int):
        """This batch as k consecutive parts that share its device tensors (views, nothing is
        copied): each part is a TabxEnv of its own with `env_id_offset` set, so calls on the
        parts compute exactly what the same calls on the whole batch would.  Launching the
        parts on different streams lets one part's launch fill the start and the end of
        another's.  Part boundaries are multiples of four envs (pointer alignment)."""
        E, N = self.E, self.N
        L = self.p.get("num_levels", 0)
        self._policy_memory()
        cuts = [min(E, (j * E // k + 3) // 4 * 4) for j in range(k)] + [E]
        out = []
        for start, stop in zip(cuts[:-1], cuts[1:]):
            count = stop - start
            if count <= 0:
                continue

            def unit(t):
                return t[start * N:stop * N]

            def env(t):
                return None if t is None else t[start:stop]

            v = object.__new__(TabxEnv)
            v.device, v.N, v.D, v.words, v.E = self.device, N, self.D, self.words, count
            v.p = dict(self.p, num_envs=count,
                       env_id_offset=self.p.get("env_id_offset", 0) + start)
            v.params, v.scenario, v.state = tabx_part(self.params, self.scenario, self.state,
                                                      start, count)
            v.p["shared_machine"] = v.params.shared_machine
            names = list(SCENARIO_FLOAT) + ["team", "enabled"]
            v.sc = {n: (self.sc[n] if L > 0 else unit(self.sc[n])) for n in names}
            v.sc["terrain"] = self.sc["terrain"] if L > 0 else env(self.sc["terrain"])
            v.sc["zone_desc"] = self.sc["zone_desc"] if L > 0 else env(self.sc["zone_desc"])
            v.st = {n: (unit(t) if t.numel() == E * N else env(t)) for n, t in self.st.items()}
            v.metrics = {n: env(t) for n, t in self.metrics.items()}
            v.gs_live = env(self.gs_live)
            v.gstate = env(self.gstate)
            v.mem = {n: unit(t) for n, t in self.mem.items()}
            v.memory = TabxPolicyMemory(mem_x=_cast(v.mem["mem_x"], _F),
                                        mem_y=_cast(v.mem["mem_y"], _F),
                                        mem_valid=_cast(v.mem["mem_valid"], _U8),
                                        next_action=_cast(v.mem["next_action"], _U8))
            v.rewards, v.dones, v.obs = env(self.rewards), env(self.dones), env(self.obs)
            v.vis, v.amask = env(self.vis), env(self.amask)
            v.first_env = start
            out.append(v)
        return out

    def global_state(self, stream=None):
        if self.gstate is None:
            self.gstate = torch.zeros(self.E, 16 * self.N + 6 * self.p["max_zones"],
                                      dtype=torch.float32, device=self.device)
        tabx_global_state(self.params, self.scenario, self.state, self.gstate, stream)
        return self.gstate

    def _policy_memory(self):
        if self.memory is None:
            n = self.E * self.N
            self.mem = {"mem_x": torch.zeros(n, dtype=torch.float32, device=self.device),
                        "mem_y": torch.zeros(n, dtype=torch.float32, device=self.device),
                        "mem_valid": torch.zeros(n, dtype=torch.uint8, device=self.device),
                        "next_action": torch.zeros(n, dtype=torch.uint8, device=self.device)}
            self.memory = TabxPolicyMemory(mem_x=_cast(self.mem["mem_x"], _F),
                                           mem_y=_cast(self.mem["mem_y"], _F),
                                           mem_valid=_cast(self.mem["mem_valid"], _U8),
                                           next_action=_cast(self.mem["next_action"], _U8))
        return self.memory

    def heuristic_actions(self, policy: dict, controlled, actions, stream=None):
        """Fills `actions` (uint8 [E, N] on the device, in place) for the controlled units."""
        self._policy_memory()
        tabx_heuristic_actions(self.params, self.scenario, self.state, TabxPolicy(**policy),
                               self.memory, controlled, actions, stream)
        return actions

    def policy_step_observe(self, policy: dict, controlled, actions, stream=None):
        tabx_policy_step_observe(self.params, self.scenario, self.state, TabxPolicy(**policy),
                                 self._policy_memory(), controlled, actions, self.rewards,
                                 self.dones, self.obs, self.vis, self.amask, stream)

    def prime_scripted(self, policy: dict, controlled, stream=None):
        """Decides the scripted units' first actions (after a reset or any outside change)."""
        self._policy_memory()
        tabx_heuristic_actions(self.params, self.scenario, self.state, TabxPolicy(**policy),
                               self.memory, controlled, self.mem["next_action"], stream)

    def scripted_step_observe(self, policy: dict, controlled, actions, stream=None):
        tabx_scripted_step_observe(self.params, self.scenario, self.state, TabxPolicy(**policy),
                                   self._policy_memory(), controlled, actions, self.rewards,
                                   self.dones, self.obs, self.vis, self.amask, stream)

    def reset(self, env_mask=None, stream=None):
        tabx_reset(self.params, self.scenario, self.state, env_mask, stream)

    def step(self, actions, stream=None):
        tabx_step(self.params, self.scenario, self.state, actions, self.rewards, self.dones,
                  stream)

    def observe(self, stream=None):
        tabx_observe(self.params, self.scenario, self.state, self.obs, self.vis, self.amask,
                     stream)

    def step_observe(self, actions, stream=None):
        tabx_step_observe(self.params, self.scenario, self.state, actions, self.rewards,
                          self.dones, self.obs, self.vis, self.amask, stream)

    def norm_obs(self, weight, bias, eps, y, mean=None, rstd=None, controlled=None, stream=None):
        """y [E, N, D] = layer norm of the observation rows, of the controlled units (None: all): those that
        learn, not those that the policy's calls take as controlled.  Other rows of y keep what they hold."""
        tabx_layer_norm(self.obs, weight, bias, eps, y, mean, rstd, controlled, stream)

    def sample_actions(self, logits, sampling, uniform, actions, log_prob=None, controlled=None,
                       stream=None):
        """Fills `actions` (uint8 [E, N], in place) for the controlled units (None: all; those that learn, not
        those that the policy's calls take) from their logits [E, N, 8], with the combat action for those
        that the last observation lets strike."""
        if self.amask is None:
            _refuse("sample_actions", "this batch keeps no action mask (want_action_mask=False)")
        tabx_sample_actions(logits, sampling, uniform, actions, log_prob, self.amask, controlled,
                            stream)
        return actions

    def sample_levels(self, scores, sampling, uniform, level_mask=None, env_mask=None, stream=None):
        """Draws the levels that the envs' next episodes take (instead of the uniform draw), out of the
        batch's num_levels."""
        levels = self.p.get("num_levels", 0)
        if levels < 1:
            _refuse("sample_levels", "this batch has no bank of levels (num_levels)")
        if scores.dim() and scores.shape[-1] != levels:    # (a reset takes next_level modulo num_levels)
            _refuse("sample_levels", f"scores has rows of {scores.shape[-1]} elements, not {levels}")
        tabx_sample_levels(scores, sampling, uniform, self.st["next_level"], level_mask, env_mask,
                           stream)

    def snapshot(self) -> dict:
        return {k: v.clone() for k, v in self.st.items()}

    def restore(self, snap: dict):
        for k, v in snap.items():
            self.st[k].copy_(v)

    def state_numpy(self) -> dict:
        out = {}
        for k, v in self.st.items():
            a = v.cpu().numpy()
            per_env = k in ("t", "phi_prev") or k in LEVELS
            out[k] = a if per_env else a.reshape(self.E, self.N)
        return out
