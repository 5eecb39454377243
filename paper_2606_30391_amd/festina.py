"""Thin ctypes binding of the C ABI in include/festina.h.

Argument marshalling only: every step of the search runs in the HIP library
(``libfestina.so`` built from ``csrc/festina.hip``, ``csrc/fronts.hip``, ``csrc/sweep.hip``,
``csrc/preferred.hip``, ``csrc/dispatch.hip`` and ``csrc/transfer.hip``; the serving step's kernels
from ``csrc/blocks.hip``, ``csrc/cache.hip``, ``csrc/attend.hip``, ``csrc/drafts.hip`` and
``csrc/rotate.hip``).  PyTorch provides device
memory and streams.  There is no CPU fallback: if the library is missing this
module raises.
"""
from __future__ import annotations

import ctypes as C
import math
import os

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libfestina.so")

FESTINA_OK = 0
FESTINA_ERR_INVALID = 1
FESTINA_ERR_DEVICE = 2
FESTINA_ERR_UNSUPPORTED = 3
FESTINA_ERR_TOO_LARGE = 4
FESTINA_NOALLOC_WORKSPACE_BYTES = 32 << 20
FESTINA_STATIC_PER_TASK = 0      # sweep energy readings (festina_batches.static_power)
FESTINA_STATIC_PER_BATCH = 1
FESTINA_BF16 = 0                 # element types of keys, values, queries and outputs
FESTINA_F16 = 1
FESTINA_F32 = 2


class FestinaError(RuntimeError):
    def __init__(self, status: int, what: str):
        super().__init__(f"{what}: {festina_status_string(status)} (status {status})")
        self.status = status


class festina_lut(C.Structure):
    _fields_ = [("n_models", C.c_int32), ("n_rows", C.c_int32), ("n_sm", C.c_int32),
                ("n_freq", C.c_int32), ("sm_level", C.c_void_p), ("freq_level", C.c_void_p),
                ("pf", C.c_void_p), ("dc", C.c_void_p), ("p0_w", C.c_float)]


class festina_gpus(C.Structure):
    _fields_ = [("n_gpus", C.c_int32), ("n_waves", C.c_int32), ("batch", C.c_void_p),
                ("k_dyn_w", C.c_void_p), ("resident", C.c_void_p), ("cap_pf", C.c_void_p),
                ("cap_dc", C.c_void_p)]


class festina_requests(C.Structure):
    _fields_ = [("n_requests", C.c_int32), ("model", C.c_void_p), ("wave", C.c_void_p),
                ("prompt_tokens", C.c_void_p), ("pred_out_tokens", C.c_void_p),
                ("slo_ttft_ms", C.c_void_p), ("slo_tbt_ms", C.c_void_p)]


class festina_placements(C.Structure):
    _fields_ = [("choice", C.c_void_p), ("feasible", C.c_void_p), ("energy_mj", C.c_void_p)]


class festina_fleet(C.Structure):
    _fields_ = [("n_gpus", C.c_int32), ("max_inst", C.c_int32), ("n_inst", C.c_void_p),
                ("inst_model", C.c_void_p), ("inst_prompt_tokens", C.c_void_p),
                ("inst_batch", C.c_void_p), ("inst_sm", C.c_void_p),
                ("inst_slo_ttft_ms", C.c_void_p), ("inst_slo_tbt_ms", C.c_void_p),
                ("hbm_mib", C.c_void_p), ("sm_permille", C.c_void_p), ("util", C.c_void_p),
                ("k_dyn_w", C.c_void_p), ("hbm_cap_mib", C.c_int32), ("sm_cap_permille", C.c_int32)]


class festina_migrations(C.Structure):
    _fields_ = [("best_dst", C.c_void_p), ("saving_w", C.c_void_p), ("freq_level", C.c_void_p)]


class festina_batches(C.Structure):
    _fields_ = [("n_batches", C.c_int32), ("max_tasks", C.c_int32), ("n_tasks", C.c_void_p),
                ("task_model", C.c_void_p), ("task_phase", C.c_void_p), ("task_tokens", C.c_void_p),
                ("task_slack_ms", C.c_void_p), ("k_dyn_w", C.c_void_p), ("util", C.c_void_p),
                ("sm_units", C.c_void_p), ("sm_budget", C.c_int32), ("static_power", C.c_int32)]


class festina_sweep_result(C.Structure):
    _fields_ = [("freq_level", C.c_void_p), ("feasible", C.c_void_p), ("energy_mj", C.c_void_p),
                ("task_sm", C.c_void_p)]


class festina_llms(C.Structure):
    _fields_ = [("n_gpus", C.c_int32), ("max_inst", C.c_int32), ("n_inst", C.c_void_p),
                ("model", C.c_void_p), ("avg_in_tokens", C.c_void_p), ("avg_out_tokens", C.c_void_p),
                ("batch", C.c_void_p), ("slo_ttft_ms", C.c_void_p), ("slo_tbt_ms", C.c_void_p),
                ("k_dyn_w", C.c_void_p)]


class festina_preferred(C.Structure):
    _fields_ = [("sm_p", C.c_void_p), ("f_p", C.c_void_p), ("sm_d", C.c_void_p), ("f_d", C.c_void_p),
                ("t_p_ms", C.c_void_p), ("t_d_ms", C.c_void_p), ("p_p_w", C.c_void_p), ("p_d_w", C.c_void_p),
                ("t_ms", C.c_void_p), ("sm_pref", C.c_void_p), ("f_pref", C.c_void_p), ("feasible", C.c_void_p)]


class festina_ewr(C.Structure):
    _fields_ = [("f_gpu", C.c_void_p), ("waste_gpu", C.c_void_p), ("totals", C.c_void_p)]


class festina_gpu_avail(C.Structure):
    _fields_ = [("n_gpus", C.c_int32), ("n_steps", C.c_int32), ("freq_cur", C.c_void_p), ("batch", C.c_void_p),
                ("k_dyn_w", C.c_void_p), ("resident", C.c_void_p), ("t_avail_ms", C.c_void_p),
                ("mem_free_mib", C.c_void_p), ("sm_free", C.c_void_p), ("kv_kib_per_token", C.c_void_p),
                ("k_new_w", C.c_float)]


class festina_dispatches(C.Structure):
    _fields_ = [("gpu", C.c_void_p), ("freq_level", C.c_void_p), ("sm_level", C.c_void_p),
                ("phase", C.c_void_p), ("energy_mj", C.c_void_p)]


class festina_gpu_state(C.Structure):
    _fields_ = [("freq_cur", C.c_void_p), ("batch", C.c_void_p), ("mem_free_mib", C.c_void_p)]


class festina_transfer(C.Structure):
    _fields_ = [("n_gpus", C.c_int32), ("n_models", C.c_int32), ("resident", C.c_void_p),
                ("weights_mib", C.c_void_p), ("state_mib", C.c_void_p), ("node", C.c_void_p),
                ("bw_intra_gbs", C.c_float), ("bw_inter_gbs", C.c_float)]


class festina_plan(C.Structure):
    _fields_ = [("dest", C.c_void_p), ("freq_cur", C.c_void_p), ("sm_cur", C.c_void_p), ("batch", C.c_void_p)]


class festina_inflight(C.Structure):
    _fields_ = [("n_requests", C.c_int32), ("src", C.c_void_p), ("model", C.c_void_p),
                ("context_tokens", C.c_void_p), ("remaining_tokens", C.c_void_p), ("kv_kib", C.c_void_p),
                ("token_kib", C.c_void_p)]


class festina_moves(C.Structure):
    _fields_ = [("decision", C.c_void_p), ("remaining_ms", C.c_void_p), ("migrate_ms", C.c_void_p)]


class festina_kv_requests(C.Structure):
    _fields_ = [("n_requests", C.c_int32), ("max_blocks", C.c_int32), ("block_tokens", C.c_int32),
                ("n_blocks", C.c_int32), ("held", C.c_void_p), ("add", C.c_void_p), ("block_table", C.c_void_p),
                ("free_ids", C.c_void_p), ("n_free", C.c_void_p)]


class festina_kv_step(C.Structure):
    _fields_ = [("max_tokens", C.c_int32), ("first", C.c_void_p), ("slot", C.c_void_p), ("length", C.c_void_p),
                ("served", C.c_void_p), ("n_free_out", C.c_void_p)]


class festina_kv_cache(C.Structure):
    _fields_ = [("n_blocks", C.c_int32), ("block_tokens", C.c_int32), ("n_kv_heads", C.c_int32),
                ("head_dim", C.c_int32), ("k", C.c_void_p), ("v", C.c_void_p), ("k_scale", C.c_void_p),
                ("v_scale", C.c_void_p)]


class festina_kv_tokens(C.Structure):
    _fields_ = [("n_tokens", C.c_int32), ("dtype", C.c_int32), ("k", C.c_void_p), ("v", C.c_void_p),
                ("k_token_stride", C.c_int64), ("k_head_stride", C.c_int64), ("v_token_stride", C.c_int64),
                ("v_head_stride", C.c_int64), ("slot", C.c_void_p)]


class festina_attention(C.Structure):
    _fields_ = [("n_requests", C.c_int32), ("max_blocks", C.c_int32), ("n_tokens", C.c_int32),
                ("n_heads", C.c_int32), ("max_new", C.c_int32), ("dtype", C.c_int32), ("window", C.c_int32),
                ("scale", C.c_float), ("block_table", C.c_void_p), ("length", C.c_void_p), ("first", C.c_void_p),
                ("q", C.c_void_p), ("q_token_stride", C.c_int64), ("q_head_stride", C.c_int64),
                ("out", C.c_void_p), ("out_token_stride", C.c_int64), ("out_head_stride", C.c_int64),
                ("lse", C.c_void_p)]


class festina_drafts(C.Structure):
    _fields_ = [("n_requests", C.c_int32), ("n_tokens", C.c_int32), ("first", C.c_void_p), ("length", C.c_void_p),
                ("parent", C.c_void_p)]


class festina_accepted(C.Structure):
    _fields_ = [("path", C.c_void_p), ("kept", C.c_void_p), ("next", C.c_void_p), ("length", C.c_void_p)]


class festina_kept(C.Structure):
    _fields_ = [("n_requests", C.c_int32), ("max_blocks", C.c_int32), ("n_tokens", C.c_int32),
                ("block_table", C.c_void_p), ("length", C.c_void_p), ("first", C.c_void_p), ("path", C.c_void_p),
                ("kept", C.c_void_p)]


class festina_rotary(C.Structure):
    _fields_ = [("head_dim", C.c_int32), ("rotated", C.c_int32), ("interleaved", C.c_int32), ("eps", C.c_float),
                ("turn", C.c_void_p), ("q_weight", C.c_void_p), ("k_weight", C.c_void_p)]


class festina_heads(C.Structure):
    _fields_ = [("n_tokens", C.c_int32), ("n_heads", C.c_int32), ("n_kv_heads", C.c_int32), ("dtype", C.c_int32),
                ("position", C.c_void_p), ("q", C.c_void_p), ("k", C.c_void_p), ("q_token_stride", C.c_int64),
                ("q_head_stride", C.c_int64), ("k_token_stride", C.c_int64), ("k_head_stride", C.c_int64),
                ("q_out", C.c_void_p), ("k_out", C.c_void_p), ("q_out_token_stride", C.c_int64),
                ("q_out_head_stride", C.c_int64), ("k_out_token_stride", C.c_int64), ("k_out_head_stride", C.c_int64)]


EXPORTED = ("festina_abi_version", "festina_status_string", "festina_placements_workspace_bytes",
            "festina_score_placements", "festina_score_placements_noalloc", "festina_migrations_workspace_bytes",
            "festina_score_migrations",
            "festina_sweep_batches", "festina_preferred_configs", "festina_ewr_workspace_bytes",
            "festina_fleet_ewr", "festina_dispatch_workspace_bytes", "festina_dispatch_requests",
            "festina_transfer_costs", "festina_request_moves", "festina_score_placements_timed",
            "festina_score_migrations_timed", "festina_dispatch_waves_workspace_bytes", "festina_dispatch_waves",
            "festina_blocks_workspace_bytes", "festina_extend_blocks", "festina_release_blocks", "festina_store_kv",
            "festina_attend_workspace_bytes", "festina_attend", "festina_trim_blocks", "festina_plan_drafts",
            "festina_accept_drafts", "festina_attend_drafts_workspace_bytes", "festina_attend_drafts",
            "festina_keep_tokens", "festina_rotate_heads")

_lib = None


def _check_fresh():
    """Raise unless the library was built from the sources now in the tree."""
    from .build import HASH_FILE, source_hash
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"HIP library {LIB_PATH} is not built; run __graft_entry__.build()")
    try:
        with open(HASH_FILE) as f:
            built = f.read().strip()
    except OSError:
        built = ""
    if built != source_hash():
        raise RuntimeError(f"HIP library {LIB_PATH} was not built from the sources in this tree "
                           "(csrc/, include/festina.h or the flags changed); run __graft_entry__.build()")


def lib():
    """Load the built HIP library (raises if it has not been built, or was built from other
    sources than the ones in the tree)."""
    global _lib
    if _lib is None:
        _check_fresh()
        L = C.CDLL(LIB_PATH)
        P = C.POINTER
        L.festina_abi_version.restype = C.c_int32
        L.festina_status_string.argtypes = [C.c_int]
        L.festina_status_string.restype = C.c_char_p
        L.festina_placements_workspace_bytes.argtypes = [P(festina_lut), P(festina_gpus), P(festina_requests)]
        L.festina_placements_workspace_bytes.restype = C.c_size_t
        L.festina_score_placements.argtypes = [P(festina_lut), P(festina_gpus), P(festina_requests),
                                               P(festina_placements), C.c_void_p, C.c_size_t, C.c_void_p]
        L.festina_score_placements.restype = C.c_int
        L.festina_score_placements_noalloc.argtypes = [P(festina_lut), P(festina_gpus), P(festina_requests),
                                                       P(festina_placements), C.c_void_p]
        L.festina_score_placements_noalloc.restype = C.c_int
        L.festina_migrations_workspace_bytes.argtypes = [P(festina_lut), P(festina_fleet)]
        L.festina_migrations_workspace_bytes.restype = C.c_size_t
        L.festina_score_migrations.argtypes = [P(festina_lut), P(festina_fleet), P(festina_migrations),
                                               C.c_void_p, C.c_size_t, C.c_void_p]
        L.festina_score_migrations.restype = C.c_int
        L.festina_sweep_batches.argtypes = [P(festina_lut), P(festina_batches), P(festina_sweep_result),
                                            C.c_void_p]
        L.festina_sweep_batches.restype = C.c_int
        L.festina_preferred_configs.argtypes = [P(festina_lut), P(festina_llms), P(festina_preferred),
                                                C.c_void_p]
        L.festina_preferred_configs.restype = C.c_int
        L.festina_ewr_workspace_bytes.argtypes = [C.c_int32]
        L.festina_ewr_workspace_bytes.restype = C.c_size_t
        L.festina_fleet_ewr.argtypes = [C.c_int32, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p,
                                        P(festina_ewr), C.c_void_p, C.c_size_t, C.c_void_p]
        L.festina_fleet_ewr.restype = C.c_int
        L.festina_dispatch_workspace_bytes.argtypes = [P(festina_lut), P(festina_gpu_avail)]
        L.festina_dispatch_workspace_bytes.restype = C.c_size_t
        L.festina_dispatch_requests.argtypes = [P(festina_lut), P(festina_gpu_avail), P(festina_requests),
                                                P(festina_dispatches), C.c_void_p, C.c_size_t, C.c_void_p]
        L.festina_dispatch_requests.restype = C.c_int
        L.festina_dispatch_waves_workspace_bytes.argtypes = [P(festina_lut), P(festina_gpu_avail)]
        L.festina_dispatch_waves_workspace_bytes.restype = C.c_size_t
        L.festina_dispatch_waves.argtypes = [P(festina_lut), P(festina_gpu_avail), P(festina_requests), C.c_int32,
                                             C.c_void_p, P(festina_gpu_state), P(festina_dispatches), C.c_void_p,
                                             C.c_size_t, C.c_void_p]
        L.festina_dispatch_waves.restype = C.c_int
        L.festina_transfer_costs.argtypes = [P(festina_transfer), C.c_void_p, C.c_void_p]
        L.festina_transfer_costs.restype = C.c_int
        L.festina_request_moves.argtypes = [P(festina_lut), P(festina_transfer), P(festina_plan),
                                            P(festina_inflight), P(festina_moves), C.c_void_p]
        L.festina_request_moves.restype = C.c_int
        L.festina_score_placements_timed.argtypes = L.festina_score_placements.argtypes + [C.c_void_p, C.c_void_p]
        L.festina_score_placements_timed.restype = C.c_int
        L.festina_score_migrations_timed.argtypes = L.festina_score_migrations.argtypes + [C.c_void_p, C.c_void_p]
        L.festina_score_migrations_timed.restype = C.c_int
        L.festina_blocks_workspace_bytes.argtypes = [C.c_int32, C.c_int32]
        L.festina_blocks_workspace_bytes.restype = C.c_size_t
        L.festina_extend_blocks.argtypes = [P(festina_kv_requests), P(festina_kv_step), C.c_void_p, C.c_size_t,
                                            C.c_void_p]
        L.festina_extend_blocks.restype = C.c_int
        L.festina_release_blocks.argtypes = [P(festina_kv_requests), C.c_void_p, P(festina_kv_step), C.c_void_p,
                                             C.c_size_t, C.c_void_p]
        L.festina_release_blocks.restype = C.c_int
        L.festina_store_kv.argtypes = [P(festina_kv_cache), P(festina_kv_tokens), C.c_void_p]
        L.festina_store_kv.restype = C.c_int
        L.festina_attend_workspace_bytes.argtypes = [P(festina_kv_cache), P(festina_attention)]
        L.festina_attend_workspace_bytes.restype = C.c_size_t
        L.festina_attend.argtypes = [P(festina_kv_cache), P(festina_attention), C.c_void_p, C.c_size_t, C.c_void_p]
        L.festina_attend.restype = C.c_int
        L.festina_trim_blocks.argtypes = L.festina_release_blocks.argtypes
        L.festina_trim_blocks.restype = C.c_int
        L.festina_plan_drafts.argtypes = [P(festina_drafts), C.c_void_p, C.c_void_p, C.c_void_p]
        L.festina_plan_drafts.restype = C.c_int
        L.festina_accept_drafts.argtypes = [P(festina_drafts), C.c_void_p, C.c_void_p, P(festina_accepted), C.c_void_p]
        L.festina_accept_drafts.restype = C.c_int
        L.festina_attend_drafts_workspace_bytes.argtypes = L.festina_attend_workspace_bytes.argtypes
        L.festina_attend_drafts_workspace_bytes.restype = C.c_size_t
        L.festina_attend_drafts.argtypes = [P(festina_kv_cache), P(festina_attention), C.c_void_p, C.c_void_p, C.c_size_t,
                                            C.c_void_p]
        L.festina_attend_drafts.restype = C.c_int
        L.festina_keep_tokens.argtypes = [C.c_void_p, C.c_int32, P(festina_kept), C.c_void_p]
        L.festina_keep_tokens.restype = C.c_int
        L.festina_rotate_heads.argtypes = [P(festina_rotary), P(festina_heads), C.c_void_p]
        L.festina_rotate_heads.restype = C.c_int
        _lib = L
    return _lib



def festina_abi_version() -> int:
    return int(lib().festina_abi_version())


def festina_status_string(status: int) -> str:
    return lib().festina_status_string(int(status)).decode()


# ------------------------------------------------------------------ device marshalling
def _ptr(t):
    return None if t is None else C.c_void_p(t.data_ptr())


def _stream_handle(stream):
    if stream is None:
        # the handle of torch.cuda.current_stream() without its Stream object: that object took
        # 3.0 us of the 7 us a one-launch call keeps the host, this 0.3 us (the name is torch's own,
        # so a torch without it takes the public way)
        import torch
        raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
        if raw is None:
            return C.c_void_p(torch.cuda.current_stream().cuda_stream)
        return C.c_void_p(raw(torch.cuda.current_device()))
    if isinstance(stream, int):
        return C.c_void_p(stream)
    return C.c_void_p(stream.cuda_stream)


def _dev(a, dtype, device):
    import torch
    if a is None:
        return None
    return torch.from_numpy(np.ascontiguousarray(a, dtype=dtype)).to(device)


class DevicePlacement:
    """Placement inputs copied to device memory once, with the ABI structs pointing at them."""

    def __init__(self, inp: dict, device="cuda"):
        import torch
        lut, gp, rq = inp["lut"], inp["gpus"], inp["requests"]
        d = lambda a, t: _dev(a, t, device)
        self.t = {
            "sm_level": d(lut["sm_level"], np.float32), "freq_level": d(lut["freq_level"], np.float32),
            "pf": d(lut["pf"], np.float32), "dc": d(lut["dc"], np.float32),
            "batch": d(gp["batch"], np.int32), "k_dyn_w": d(gp["k_dyn_w"], np.float32),
            "resident": d(np.asarray(gp["resident"], np.uint32).view(np.int32), np.int32),
            "cap_pf": d(gp.get("cap_pf"), np.int8), "cap_dc": d(gp.get("cap_dc"), np.int8),
            "model": d(rq["model"], np.int32), "wave": d(rq.get("wave"), np.int32),
            "prompt_tokens": d(rq["prompt_tokens"], np.int32),
            "pred_out_tokens": d(rq["pred_out_tokens"], np.int32),
            "slo_ttft_ms": d(rq["slo_ttft_ms"], np.float32), "slo_tbt_ms": d(rq["slo_tbt_ms"], np.float32),
        }
        t = self.t
        self.lut = festina_lut(int(lut["n_models"]), int(lut["n_rows"]), int(lut["n_sm"]), int(lut["n_freq"]),
                               _ptr(t["sm_level"]), _ptr(t["freq_level"]), _ptr(t["pf"]), _ptr(t["dc"]),
                               float(lut["p0_w"]))
        self.gpus = festina_gpus(int(gp["n_gpus"]), int(gp["n_waves"]), _ptr(t["batch"]), _ptr(t["k_dyn_w"]),
                                 _ptr(t["resident"]), _ptr(t["cap_pf"]), _ptr(t["cap_dc"]))
        self.R = int(rq["n_requests"])
        self.req = festina_requests(self.R, _ptr(t["model"]), _ptr(t["wave"]), _ptr(t["prompt_tokens"]),
                                    _ptr(t["pred_out_tokens"]), _ptr(t["slo_ttft_ms"]), _ptr(t["slo_tbt_ms"]))
        n = max(self.R, 1)
        self.choice = torch.empty(n, dtype=torch.int32, device=device)
        self.feasible = torch.empty(n, dtype=torch.uint8, device=device)
        self.energy = torch.empty(n, dtype=torch.float32, device=device)
        self.out = festina_placements(_ptr(self.choice), _ptr(self.feasible), _ptr(self.energy))
        self.ws_bytes = festina_placements_workspace_bytes(self.lut, self.gpus, self.req)
        self.workspace = torch.empty(max(self.ws_bytes, 256), dtype=torch.uint8, device=device)

    def run(self, stream=None, events=None):
        """One search; `events` = (begin, end) raw hipEvent_t handles recorded around the
        scoring kernel or kernels (the timed entry point), else None."""
        festina_score_placements(self.lut, self.gpus, self.req, self.out, self.workspace, self.ws_bytes, stream,
                                 events)

    def run_noalloc(self, stream=None):
        """The same search through the allocation-free entry point (the library's scratch)."""
        festina_score_placements_noalloc(self.lut, self.gpus, self.req, self.out, stream)

    def results(self):
        R = self.R
        return (self.choice[:R].cpu().numpy(), self.feasible[:R].cpu().numpy(), self.energy[:R].cpu().numpy())


class DeviceMigration:
    """Consolidation fleet copied to device memory once, with the ABI structs pointing at it."""

    def __init__(self, inp: dict, device="cuda"):
        import torch
        lut, fl = inp["lut"], inp["fleet"]
        d = lambda a, t: _dev(a, t, device)
        self.t = {
            "freq_level": d(lut["freq_level"], np.float32), "sm_level": d(lut["sm_level"], np.float32),
            "pf": d(lut["pf"], np.float32), "dc": d(lut["dc"], np.float32),
        }
        for k in ("n_inst", "inst_model", "inst_prompt_tokens", "inst_batch", "inst_sm", "hbm_mib", "sm_permille"):
            self.t[k] = d(fl[k], np.int32)
        for k in ("inst_slo_ttft_ms", "inst_slo_tbt_ms", "util", "k_dyn_w"):
            self.t[k] = d(fl[k], np.float32)
        t = self.t
        self.lut = festina_lut(int(lut["n_models"]), int(lut["n_rows"]), int(lut["n_sm"]), int(lut["n_freq"]),
                               _ptr(t["sm_level"]), _ptr(t["freq_level"]), _ptr(t["pf"]), _ptr(t["dc"]),
                               float(lut["p0_w"]))
        self.G = int(fl["n_gpus"])
        self.fleet = festina_fleet(self.G, int(fl["max_inst"]), _ptr(t["n_inst"]), _ptr(t["inst_model"]),
                                   _ptr(t["inst_prompt_tokens"]), _ptr(t["inst_batch"]), _ptr(t["inst_sm"]),
                                   _ptr(t["inst_slo_ttft_ms"]), _ptr(t["inst_slo_tbt_ms"]), _ptr(t["hbm_mib"]),
                                   _ptr(t["sm_permille"]), _ptr(t["util"]), _ptr(t["k_dyn_w"]),
                                   int(fl["hbm_cap_mib"]), int(fl["sm_cap_permille"]))
        self.best_dst = torch.empty(self.G, dtype=torch.int32, device=device)
        self.saving = torch.empty(self.G, dtype=torch.float32, device=device)
        self.level = torch.empty(self.G, dtype=torch.int32, device=device)
        self.out = festina_migrations(_ptr(self.best_dst), _ptr(self.saving), _ptr(self.level))
        self.ws_bytes = festina_migrations_workspace_bytes(self.lut, self.fleet)
        self.workspace = torch.empty(max(self.ws_bytes, 256), dtype=torch.uint8, device=device)

    def run(self, stream=None, events=None):
        """One search; `events` = (begin, end) raw hipEvent_t handles recorded around the
        pair-scoring kernel (the timed entry point), else None."""
        festina_score_migrations(self.lut, self.fleet, self.out, self.workspace, self.ws_bytes, stream, events)

    def results(self):
        return self.best_dst.cpu().numpy(), self.saving.cpu().numpy(), self.level.cpu().numpy()


class DeviceSweep:
    """Local-scheduler task batches copied to device memory once, with the ABI structs."""

    def __init__(self, inp: dict, device="cuda"):
        import torch
        lut, bt = inp["lut"], inp["batches"]
        d = lambda a, t: _dev(a, t, device)
        self.t = {
            "freq_level": d(lut["freq_level"], np.float32), "sm_level": d(lut["sm_level"], np.float32),
            "pf": d(lut["pf"], np.float32), "dc": d(lut["dc"], np.float32),
        }
        for k in ("n_tasks", "task_model", "task_phase", "task_tokens", "sm_units"):
            self.t[k] = d(bt[k], np.int32)
        for k in ("task_slack_ms", "k_dyn_w", "util"):
            self.t[k] = d(bt[k], np.float32)
        t = self.t
        self.lut = festina_lut(int(lut["n_models"]), int(lut["n_rows"]), int(lut["n_sm"]), int(lut["n_freq"]),
                               _ptr(t["sm_level"]), _ptr(t["freq_level"]), _ptr(t["pf"]), _ptr(t["dc"]),
                               float(lut["p0_w"]))
        self.B, self.T = int(bt["n_batches"]), int(bt["max_tasks"])
        self.batches = festina_batches(self.B, self.T, _ptr(t["n_tasks"]), _ptr(t["task_model"]),
                                       _ptr(t["task_phase"]), _ptr(t["task_tokens"]), _ptr(t["task_slack_ms"]),
                                       _ptr(t["k_dyn_w"]), _ptr(t["util"]), _ptr(t["sm_units"]),
                                       int(bt["sm_budget"]), int(bt.get("static_power", 0)))
        n = max(self.B, 1)
        self.level = torch.empty(n, dtype=torch.int32, device=device)
        self.feasible = torch.empty(n, dtype=torch.uint8, device=device)
        self.energy = torch.empty(n, dtype=torch.float32, device=device)
        self.task_sm = torch.empty((n, self.T), dtype=torch.int32, device=device)
        self.out = festina_sweep_result(_ptr(self.level), _ptr(self.feasible), _ptr(self.energy),
                                        _ptr(self.task_sm))

    def run(self, stream=None):
        festina_sweep_batches(self.lut, self.batches, self.out, stream)

    def results(self):
        B = self.B
        return (self.level[:B].cpu().numpy(), self.feasible[:B].cpu().numpy(), self.energy[:B].cpu().numpy(),
                self.task_sm[:B].cpu().numpy())


PREF_INT = ("sm_p", "f_p", "sm_d", "f_d")
PREF_FLOAT = ("t_p_ms", "t_d_ms", "p_p_w", "p_d_w", "t_ms", "sm_pref", "f_pref")


class DevicePreferred:
    """Active LLM instances copied to device memory once; run() computes every preferred
    configuration and then the fleet's EWR from them (execution time t_ms = t_p + t_d)."""

    def __init__(self, inp: dict, device="cuda"):
        import torch
        lut, q = inp["lut"], inp["llms"]
        d = lambda a, t: _dev(a, t, device)
        self.t = {
            "freq_level": d(lut["freq_level"], np.float32), "sm_level": d(lut["sm_level"], np.float32),
            "pf": d(lut["pf"], np.float32), "dc": d(lut["dc"], np.float32),
        }
        for k in ("n_inst", "model", "avg_in_tokens", "avg_out_tokens", "batch"):
            self.t[k] = d(q[k], np.int32)
        for k in ("slo_ttft_ms", "slo_tbt_ms", "k_dyn_w"):
            self.t[k] = d(q[k], np.float32)
        t = self.t
        self.lut = festina_lut(int(lut["n_models"]), int(lut["n_rows"]), int(lut["n_sm"]), int(lut["n_freq"]),
                               _ptr(t["sm_level"]), _ptr(t["freq_level"]), _ptr(t["pf"]), _ptr(t["dc"]),
                               float(lut["p0_w"]))
        self.G, self.K = int(q["n_gpus"]), int(q["max_inst"])
        self.llms = festina_llms(self.G, self.K, _ptr(t["n_inst"]), _ptr(t["model"]), _ptr(t["avg_in_tokens"]),
                                 _ptr(t["avg_out_tokens"]), _ptr(t["batch"]), _ptr(t["slo_ttft_ms"]),
                                 _ptr(t["slo_tbt_ms"]), _ptr(t["k_dyn_w"]))
        n = max(self.G * self.K, 1)
        self.o = {k: torch.empty(n, dtype=torch.int32, device=device) for k in PREF_INT}
        self.o.update({k: torch.empty(n, dtype=torch.float32, device=device) for k in PREF_FLOAT})
        self.o["feasible"] = torch.empty(n, dtype=torch.uint8, device=device)
        self.out = festina_preferred(*(_ptr(self.o[k]) for k in PREF_INT + PREF_FLOAT + ("feasible",)))
        g = max(self.G, 1)
        self.f_gpu = torch.empty(g, dtype=torch.float32, device=device)
        self.waste_gpu = torch.empty(g, dtype=torch.float64, device=device)
        self.totals = torch.empty(3, dtype=torch.float64, device=device)
        self.ewr = festina_ewr(_ptr(self.f_gpu), _ptr(self.waste_gpu), _ptr(self.totals))
        self.ws_bytes = festina_ewr_workspace_bytes(self.G)
        self.workspace = torch.empty(max(self.ws_bytes, 256), dtype=torch.uint8, device=device)

    def run_preferred(self, stream=None):
        festina_preferred_configs(self.lut, self.llms, self.out, stream)

    def run_ewr(self, f_pref=None, t_ms=None, stream=None):
        """EWR from device tensors f_pref/t_ms [G*K] (default: this object's own results)."""
        if f_pref is None:
            f_pref = self.o["f_pref"]
            t_ms = self.o["t_ms"]
        festina_fleet_ewr(self.G, self.K, self.t["n_inst"], f_pref, t_ms, self.ewr, self.workspace,
                          self.ws_bytes, stream)

    def run(self, stream=None):
        """Preferred configurations, then the EWR of the fleet from them."""
        self.run_preferred(stream)
        self.run_ewr(stream=stream)

    def results(self):
        G, K = self.G, self.K
        r = {k: self.o[k][:G * K].cpu().numpy().reshape(G, K) for k in PREF_INT + PREF_FLOAT + ("feasible",)}
        return r

    def ewr_results(self):
        return self.f_gpu[:self.G].cpu().numpy(), self.waste_gpu[:self.G].cpu().numpy(), self.totals.cpu().numpy()


class DeviceDispatch:
    """Requests and the GPUs' answers for the paper's own dispatcher, on the device."""

    def __init__(self, inp: dict, device="cuda"):
        import torch
        lut, av, rq = inp["lut"], inp["avail"], inp["requests"]
        d = lambda a, t: _dev(a, t, device)
        self.t = {
            "sm_level": d(lut["sm_level"], np.float32), "freq_level": d(lut["freq_level"], np.float32),
            "pf": d(lut["pf"], np.float32), "dc": d(lut["dc"], np.float32),
            "resident": d(np.asarray(av["resident"], np.uint32).view(np.int32), np.int32),
        }
        for k in ("freq_cur", "batch", "mem_free_mib", "sm_free", "kv_kib_per_token"):
            self.t[k] = d(av[k], np.int32)
        for k in ("k_dyn_w", "t_avail_ms"):
            self.t[k] = d(av[k], np.float32)
        for k in ("model", "prompt_tokens", "pred_out_tokens"):
            self.t[k] = d(rq[k], np.int32)
        for k in ("slo_ttft_ms", "slo_tbt_ms"):
            self.t[k] = d(rq[k], np.float32)
        t = self.t
        self.lut = festina_lut(int(lut["n_models"]), int(lut["n_rows"]), int(lut["n_sm"]), int(lut["n_freq"]),
                               _ptr(t["sm_level"]), _ptr(t["freq_level"]), _ptr(t["pf"]), _ptr(t["dc"]),
                               float(lut["p0_w"]))
        self.avail = festina_gpu_avail(int(av["n_gpus"]), int(av["n_steps"]), _ptr(t["freq_cur"]), _ptr(t["batch"]),
                                       _ptr(t["k_dyn_w"]), _ptr(t["resident"]), _ptr(t["t_avail_ms"]),
                                       _ptr(t["mem_free_mib"]), _ptr(t["sm_free"]), _ptr(t["kv_kib_per_token"]),
                                       float(av["k_new_w"]))
        self.R = int(rq["n_requests"])
        self.req = festina_requests(self.R, _ptr(t["model"]), None, _ptr(t["prompt_tokens"]),
                                    _ptr(t["pred_out_tokens"]), _ptr(t["slo_ttft_ms"]), _ptr(t["slo_tbt_ms"]))
        n = max(self.R, 1)
        self.o = {k: torch.empty(n, dtype=torch.int32, device=device) for k in ("gpu", "freq_level", "sm_level")}
        self.o["phase"] = torch.empty(n, dtype=torch.uint8, device=device)
        self.o["energy_mj"] = torch.empty(n, dtype=torch.float32, device=device)
        self.out = festina_dispatches(*(_ptr(self.o[k]) for k in ("gpu", "freq_level", "sm_level", "phase",
                                                                  "energy_mj")))
        self.ws_bytes = festina_dispatch_workspace_bytes(self.lut, self.avail)
        self.workspace = torch.empty(max(self.ws_bytes, 256), dtype=torch.uint8, device=device)

    def run(self, stream=None):
        festina_dispatch_requests(self.lut, self.avail, self.req, self.out, self.workspace, self.ws_bytes, stream)

    def run_waves(self, wave_start, stream=None):
        """Dispatch wave by wave (requests ordered by wave), committing each wave; the
        carried state lands in self.state_t."""
        import torch
        if not hasattr(self, "state_t"):
            dev = self.t["batch"].device
            G, S = int(self.avail.n_gpus), int(self.avail.n_steps)
            self.state_t = {"freq_cur": torch.empty(G, dtype=torch.int32, device=dev),
                            "batch": torch.empty(G, dtype=torch.int32, device=dev),
                            "mem_free_mib": torch.empty(G * S, dtype=torch.int32, device=dev)}
            self.state = festina_gpu_state(*(_ptr(self.state_t[k]) for k in ("freq_cur", "batch", "mem_free_mib")))
            self.wws_bytes = festina_dispatch_waves_workspace_bytes(self.lut, self.avail)
            self.wworkspace = torch.empty(max(self.wws_bytes, 256), dtype=torch.uint8, device=dev)
        festina_dispatch_waves(self.lut, self.avail, self.req, wave_start, self.state, self.out, self.wworkspace,
                               self.wws_bytes, stream)

    def results(self):
        R = self.R
        return tuple(self.o[k][:R].cpu().numpy() for k in ("gpu", "freq_level", "sm_level", "phase", "energy_mj"))

    def state_results(self):
        G, S = int(self.avail.n_gpus), int(self.avail.n_steps)
        return {"freq_cur": self.state_t["freq_cur"].cpu().numpy(), "batch": self.state_t["batch"].cpu().numpy(),
                "mem_free_mib": self.state_t["mem_free_mib"].cpu().numpy().reshape(G, S)}


class DeviceTransfer:
    """A reconfiguring fleet on the device: the device-mapping cost matrix and the
    in-flight requests' finish-or-move decisions."""

    def __init__(self, inp: dict, device="cuda"):
        import torch
        lut, tr, pl, mv = inp["lut"], inp["transfer"], inp["plan"], inp["moves"]
        d = lambda a, t: _dev(a, t, device)
        self.t = {"sm_level": d(lut["sm_level"], np.float32), "freq_level": d(lut["freq_level"], np.float32),
                  "pf": d(lut["pf"], np.float32), "dc": d(lut["dc"], np.float32),
                  "resident": d(np.asarray(tr["resident"], np.uint32).view(np.int32), np.int32)}
        for k in ("weights_mib", "state_mib", "node"):
            self.t[k] = d(tr[k], np.int32)
        for k in ("dest", "freq_cur", "sm_cur", "batch"):
            self.t["plan_" + k] = d(pl[k], np.int32)
        for k in ("src", "model", "context_tokens", "remaining_tokens", "kv_kib", "token_kib"):
            self.t["req_" + k] = d(mv[k], np.int32)
        t = self.t
        self.lut = festina_lut(int(lut["n_models"]), int(lut["n_rows"]), int(lut["n_sm"]), int(lut["n_freq"]),
                               _ptr(t["sm_level"]), _ptr(t["freq_level"]), _ptr(t["pf"]), _ptr(t["dc"]),
                               float(lut["p0_w"]))
        self.G = int(tr["n_gpus"])
        self.transfer = festina_transfer(self.G, int(inp["n_models"]), _ptr(t["resident"]), _ptr(t["weights_mib"]),
                                         _ptr(t["state_mib"]), _ptr(t["node"]), float(tr["bw_intra_gbs"]),
                                         float(tr["bw_inter_gbs"]))
        self.plan = festina_plan(_ptr(t["plan_dest"]), _ptr(t["plan_freq_cur"]), _ptr(t["plan_sm_cur"]),
                                 _ptr(t["plan_batch"]))
        self.Q = int(mv["n_requests"])
        self.req = festina_inflight(self.Q, *(_ptr(t["req_" + k]) for k in ("src", "model", "context_tokens",
                                                                           "remaining_tokens", "kv_kib",
                                                                           "token_kib")))
        self.cost = torch.empty((self.G, self.G), dtype=torch.float32, device=device)
        n = max(self.Q, 1)
        self.decision = torch.empty(n, dtype=torch.int32, device=device)
        self.remaining = torch.empty(n, dtype=torch.float32, device=device)
        self.migrate = torch.empty(n, dtype=torch.float32, device=device)
        self.moves = festina_moves(_ptr(self.decision), _ptr(self.remaining), _ptr(self.migrate))

    def run_costs(self, stream=None):
        festina_transfer_costs(self.transfer, self.cost, stream)

    def run_moves(self, stream=None):
        festina_request_moves(self.lut, self.transfer, self.plan, self.req, self.moves, stream)

    def results(self):
        Q = self.Q
        return (self.cost.cpu().numpy(), self.decision[:Q].cpu().numpy(), self.remaining[:Q].cpu().numpy(),
                self.migrate[:Q].cpu().numpy())


def _check(t, name, dtypes, shape=None):
    """A device tensor of one of these types (and of this shape, contiguous, if one is given)."""
    import torch
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise ValueError(f"{name}: a tensor in device memory is needed")
    if t.dtype not in dtypes:
        raise ValueError(f"{name}: dtype {t.dtype}, not {' or '.join(str(d) for d in dtypes)}")
    if shape is not None and (t.shape != shape or not t.is_contiguous()):
        raise ValueError(f"{name}: a contiguous tensor of shape {tuple(shape)} is needed, not {tuple(t.shape)}")


def _on(stream, device):
    """A context in which torch allocates for `stream` (None: the current one)."""
    import contextlib
    import torch
    if stream is None:
        return contextlib.nullcontext()
    if isinstance(stream, int):
        stream = torch.cuda.ExternalStream(stream, device=device)
    return torch.cuda.stream(stream)


def _capturing(stream, device):
    """Whether `stream` (None: the current one) is being captured into a graph."""
    import torch
    if stream is None:
        return torch.cuda.is_current_stream_capturing()
    with _on(stream, device):
        return torch.cuda.is_current_stream_capturing()


def _used_on(stream, *tensors):
    """Tell torch that work on `stream` (a torch stream) reads or writes these tensors: their memory is not given to others
    before that work is done, also where the caller drops them right after the call.  Not for a raw handle: its owner
    may end that stream at any time, so the owner keeps the tensors too."""
    if not isinstance(stream, int):
        for t in tensors:
            t.record_stream(stream)


def _dual_levels():
    """What has _current_level, of forward-mode differentiation: -1 where there is none (torch's own name; without it every
    call looks)."""
    import types
    from torch.autograd import forward_ad
    return forward_ad if hasattr(forward_ad, "_current_level") else types.SimpleNamespace(_current_level=0)


def _tangents(*tensors) -> bool:
    """Whether one of them has a forward-mode tangent."""
    from torch.autograd import forward_ad
    return any(forward_ad.unpack_dual(t).tangent is not None for t in tensors)


class _Here:
    """Where calls run, in few attribute reads: the kernels of these calls take about as long as their host work."""

    def __init__(self):
        import torch
        # (torch's own names, without which it takes the public way)
        self.device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
        self.raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
        self.int32 = torch.int32

    def stream(self, stream, now):
        """The handle of `stream` (None: the current one of device `now`), which has to be a stream of that device."""
        if stream is None:
            return self.raw(now) if self.raw is not None else _stream_handle(None)
        if not isinstance(stream, int) and stream.device_index != now:
            raise ValueError(f"stream: one of device {stream.device_index}, not of the current device {now}")
        return _stream_handle(stream)

    def ints(self, t, name, n, now):
        """The address of a contiguous int32 tensor of n entries on device `now`."""
        if t.dtype is not self.int32 or t.get_device() != now or t.dim() != 1 or t.numel() != n or not t.is_contiguous():
            _check(t, name, (self.int32,), (n,))
            _on_device(t, name, now)
        return t.data_ptr()


def _on_device(t, name, now):
    if t.get_device() != now:
        raise ValueError(f"{name}: on device {t.get_device()}, not on device {now} (that of the call)")


class _Workspaces:
    """Device scratch, one for each stream that calls come on, so that they may overlap.  A call that is captured gets
    its own from the graph's memory: a graph keeps the address that it captured, while a stream's scratch is replaced
    when a call needs more, and graphs captured on one stream may be replayed on several."""

    def __init__(self):
        self.by_stream = {}

    def get(self, n, stream, device):
        """(at least n bytes for calls on `stream`, to be held until the launch; their address; the stream's handle)."""
        handle = _stream_handle(stream).value or 0
        if handle and _capturing(stream, device):            # (the null stream cannot be captured; asking takes 1 us)
            ws = self._make(n, stream, device)
            return ws, ws.data_ptr(), handle
        ws, at, size = self.by_stream.get(handle, (None, 0, -1))
        if size < n:
            ws = self._make(n, stream, device)
            at = ws.data_ptr()
            self.by_stream[handle] = ws, at, ws.numel()
        return ws, at, handle

    @staticmethod
    def _make(n, stream, device):
        import torch
        with _on(stream, device):
            return torch.empty(max(n, 256), dtype=torch.uint8, device=device)


class DeviceBlocks:
    """The cache blocks of one GPU's requests: int32 device tensors held [R], add [R], table
    [R][max_blocks], free_ids [n_blocks], n_free [1] (festina_kv_requests), used in place.

    extend() gives every request blocks and slots for its add new tokens: table, and first [R+1],
    slot [max_tokens], length [R], served [R], n_free_out [1].  release(done) returns the blocks of the
    requests whose uint8 done is not 0: free_ids, length, n_free_out; trim(keep) those behind the tokens that each request
    keeps.  advance() makes length and n_free_out
    the next step's held and n_free (no work on the device).

    A call with stream= (a torch stream, or a raw handle) comes after what is on that stream, and waits for no other.
    With a raw handle the tensors have to outlive the call's work."""

    def __init__(self, held, add, table, free_ids, n_free, block_tokens: int, max_tokens: int):
        import torch
        if not isinstance(table, torch.Tensor) or table.dim() != 2:
            raise ValueError("table: a tensor of two dimensions is needed")
        R = int(table.shape[0])
        for name, t, shape in (("held", held, (R,)), ("add", add, (R,)), ("table", table, table.shape),
                               ("free_ids", free_ids, (free_ids.numel(),)), ("n_free", n_free, (1,))):
            _check(t, name, (torch.int32,), shape)
        device = table.device
        self.held, self.add, self.table, self.free_ids, self.n_free = held, add, table, free_ids, n_free
        self.block_tokens, self.max_tokens = int(block_tokens), int(max_tokens)
        i32 = lambda n: torch.empty(n, dtype=torch.int32, device=device)
        self.first, self.slot, self.length, self.n_free_out = i32(R + 1), i32(max(self.max_tokens, 0)), i32(R), i32(1)
        self.served = torch.empty(R, dtype=torch.uint8, device=device)
        self.ws_bytes = festina_blocks_workspace_bytes(R, self.max_tokens)
        self._ws, self._here, self._trim = _Workspaces(), _Here(), lib().festina_trim_blocks
        self._structs()

    def _structs(self):
        self.req = festina_kv_requests(int(self.table.shape[0]), int(self.table.shape[1]), self.block_tokens,
                                       int(self.free_ids.numel()), _ptr(self.held), _ptr(self.add), _ptr(self.table),
                                       _ptr(self.free_ids), _ptr(self.n_free))
        self.out = festina_kv_step(self.max_tokens, _ptr(self.first), _ptr(self.slot), _ptr(self.length),
                                   _ptr(self.served), _ptr(self.n_free_out))

    def extend(self, stream=None):
        held, ws, handle = self._ws.get(self.ws_bytes, stream, self.table.device)
        festina_extend_blocks(self.req, self.out, ws, self.ws_bytes, handle)
        if stream is not None:
            _used_on(stream, *self._tensors())

    def release(self, done, stream=None):
        import torch
        _check(done, "done", (torch.uint8, torch.bool), self.held.shape)
        held, ws, handle = self._ws.get(self.ws_bytes, stream, self.table.device)
        festina_release_blocks(self.req, done, self.out, ws, self.ws_bytes, handle)
        if stream is not None:
            _used_on(stream, done, *self._tensors())

    def trim(self, keep, stream=None):
        """Give back the blocks behind the first keep[r] (int32, device) tokens of every request: free_ids, length (keep),
        n_free_out."""
        here = self._here
        now = here.device()
        at = here.ints(keep, "keep", self.held.numel(), now)
        if self.table.get_device() != now:
            _on_device(self.table, "table", now)
        if stream is not None:
            here.stream(stream, now)
        held, ws, handle = self._ws.get(self.ws_bytes, stream, self.table.device)
        st = self._trim(C.byref(self.req), at, C.byref(self.out), ws, self.ws_bytes, handle)
        if st != FESTINA_OK:
            raise FestinaError(st, "festina_trim_blocks")
        if stream is not None:
            _used_on(stream, keep, *self._tensors())

    def _tensors(self):
        return (self.held, self.add, self.table, self.free_ids, self.n_free, self.first, self.slot, self.length, self.served,
                self.n_free_out)

    def advance(self):
        self.held, self.length = self.length, self.held
        self.n_free, self.n_free_out = self.n_free_out, self.n_free
        self._structs()


class DeviceCache:
    """One layer's key/value cache in 8 bits (festina_kv_cache): uint8 codes k [n_blocks][kv heads][block tokens]
    [dim], v [n_blocks][kv heads][dim][block tokens] and float32 scales k_scale, v_scale [n_blocks][kv heads],
    device tensors used in place (``DeviceCache.empty`` makes them).  Scratch is the object's own, or shared with that of
    the cache given as scratch_of (another layer's), one for each stream; what torch.cuda.graph captures has scratch of its graph's memory (a graph captured by other means: festina_attend
    with a workspace that the caller keeps).  stream= as for DeviceBlocks."""

    def __init__(self, k, v, k_scale, v_scale, scratch_of=None):
        import torch
        _check(k, "k", (torch.uint8,), k.shape)
        if k.dim() != 4:
            raise ValueError("k: [blocks][kv heads][block tokens][dim]")
        n, h, bt, d = (int(x) for x in k.shape)
        _check(v, "v", (torch.uint8,), (n, h, d, bt))
        _check(k_scale, "k_scale", (torch.float32,), (n, h))
        _check(v_scale, "v_scale", (torch.float32,), (n, h))
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        self.cache = festina_kv_cache(n, bt, h, d, _ptr(k), _ptr(v), _ptr(k_scale), _ptr(v_scale))
        self._ws, self._ws_bytes = scratch_of._ws if scratch_of is not None else _Workspaces(), {}
        self._halves = {torch.bfloat16: FESTINA_BF16, torch.float16: FESTINA_F16}
        self._types = {**self._halves, torch.float32: FESTINA_F32}
        self._int32, self._f32, self._rows, self._scale = (torch.int32,), torch.float32, (h, d), d ** -0.5
        self._empty, self._attend, self._cache_ref = torch.empty, lib().festina_attend, C.byref(self.cache)
        self._attend_drafts, self._int64, self._here = lib().festina_attend_drafts, (torch.int64,), _Here()
        self._keep, self._struct, self._device = lib().festina_keep_tokens, bytes(self.cache), k.get_device()
        self._graded, self._dual = torch.is_grad_enabled, _dual_levels()

    @classmethod
    def empty(cls, n_blocks: int, block_tokens: int, n_kv_heads: int, head_dim: int, device="cuda", scratch_of=None):
        import torch
        u8 = lambda *s: torch.empty(s, dtype=torch.uint8, device=device)
        f32 = lambda: torch.zeros((n_blocks, n_kv_heads), dtype=torch.float32, device=device)
        return cls(u8(n_blocks, n_kv_heads, block_tokens, head_dim), u8(n_blocks, n_kv_heads, head_dim, block_tokens),
                   f32(), f32(), scratch_of)

    def store(self, k, v, slot, stream=None):
        """Store keys and values [tokens][kv heads][dim] (bfloat16, half or float32; any strides but the last)
        at the int32 slots [tokens].  What is held has no gradient."""
        for name, x in (("k", k), ("v", v)):
            _check(x, name, self._types)
            if x.dim() != 3 or x.shape[1:] != self._rows or (x.stride(2) != 1 and x.numel()):
                raise ValueError(f"{name}: [tokens][{self._rows[0]}][{self._rows[1]}] with its last axis contiguous")
        T = k.shape[0]
        if k.dtype != v.dtype or v.shape[0] != T:
            raise ValueError("k and v: one type and number of tokens")
        _check(slot, "slot", self._int32, (T,))
        (kt, kh, _), (vt, vh, _) = k.stride(), v.stride()
        festina_store_kv(self.cache, festina_kv_tokens(T, self._types[k.dtype], k.data_ptr(), v.data_ptr(), kt, kh, vt,
                                                       vh, slot.data_ptr()), stream)
        if stream is not None:
            _used_on(stream, k, v, slot, self.k, self.v, self.k_scale, self.v_scale)

    def attend(self, q, table, length, first, max_new: int, scale=None, window: int = 0, out=None, lse=None,
               stream=None, seen=None):
        """Attention of the queries [tokens][heads][dim] (bfloat16 or half) over the cache: (out, lse).  table
        [requests][columns], length [requests] (new tokens included) and first [requests+1] are a step's
        (DeviceBlocks); max_new bounds the new tokens of one request.  out and lse are made where not given.  seen
        [tokens] (int64, DeviceDrafts.plan) says which of its request's new tokens each sees, where they are drafts.  For
        serving: queries that ask for a gradient or carry a tangent are refused."""
        # every check by itself: _check() where one fails names what is wrong (a decode step's kernels take about as
        # long as this function's host work, so it keeps to a few attribute reads a tensor)
        dim = self._rows[1]
        dtype = q.dtype
        kind = self._halves.get(dtype)
        i32 = self._int32[0]
        if kind is None or not q.is_cuda:
            _check(q, "q", self._halves)
        if (q.requires_grad and self._graded()) or (self._dual._current_level >= 0 and _tangents(q)):
            raise ValueError("q: no gradient passes through a cache in 8 bits (call under torch.no_grad(), without tangents)")
        if q.dim() != 3 or q.shape[2] != dim or (q.stride(2) != 1 and q.numel()):
            raise ValueError(f"q: [tokens][heads][{dim}] with its last axis contiguous")
        if table.dtype is not i32 or not table.is_cuda:
            _check(table, "table", self._int32)
        if table.dim() != 2 or not table.is_contiguous():
            raise ValueError("table: a contiguous tensor of two dimensions is needed")
        T, heads, _ = q.shape
        R, columns = table.shape
        if length.dtype is not i32 or not length.is_cuda or length.dim() != 1 or len(length) != R or \
                not length.is_contiguous():
            _check(length, "length", self._int32, (R,))
        if first.dtype is not i32 or not first.is_cuda or first.dim() != 1 or len(first) != R + 1 or \
                not first.is_contiguous():
            _check(first, "first", self._int32, (R + 1,))
        if stream is None:
            if out is None:
                out = self._empty((T, heads, dim), dtype=dtype, device=q.device)
            if lse is None:
                lse = self._empty((T, heads), dtype=self._f32, device=q.device)
        elif out is None or lse is None:
            with _on(stream, q.device):
                return self.attend(q, table, length, first, max_new, scale, window,
                                   self._empty((T, heads, dim), dtype=dtype, device=q.device) if out is None else out,
                                   self._empty((T, heads), dtype=self._f32, device=q.device) if lse is None else lse,
                                   stream, seen)
        if out.dtype is not dtype or not out.is_cuda:
            _check(out, "out", (dtype,))
        if out.shape != q.shape or (out.stride(2) != 1 and out.numel()):
            raise ValueError("out: q's shape with its last axis contiguous")
        if lse.dtype is not self._f32 or not lse.is_cuda or lse.dim() != 2 or not lse.is_contiguous() or \
                lse.shape[0] != T or lse.shape[1] != heads:
            _check(lse, "lse", (self._f32,), (T, heads))
        if max_new >> 31 or window >> 31:                    # past the struct's 32 bits, where ctypes would cut them off
            max_new, window = max(-1, min(max_new, 0x7FFFFFFF)), max(-1, min(window, 0x7FFFFFFF))
        qt, qh, _ = q.stride()
        ot, oh, _ = out.stride()
        att = festina_attention(R, columns, T, heads, max_new, kind, window, self._scale if scale is None else scale,
                                table.data_ptr(), length.data_ptr(), first.data_ptr(), q.data_ptr(), qt, qh,
                                out.data_ptr(), ot, oh, lse.data_ptr())
        if seen is not None:
            return self._over_drafts(att, (R, columns, T, heads, max_new, 1), seen, q, table, length, first, out, lse, stream)
        sizes = (R, columns, T, heads, max_new)
        n = self._ws_bytes.get(sizes)
        if n is None:
            if len(self._ws_bytes) > 1024:
                self._ws_bytes.clear()
            n = festina_attend_workspace_bytes(self.cache, att)
            if n:                                            # 0: refused below, for something that may not be a size
                self._ws_bytes[sizes] = n
        held, ws, handle = self._ws.get(n, stream, q.device)
        st = self._attend(self._cache_ref, C.byref(att), ws, n, handle)
        if st != FESTINA_OK:
            raise FestinaError(st, "festina_attend")
        if stream is not None:
            _used_on(stream, q, table, length, first, out, lse, self.k, self.v, self.k_scale, self.v_scale)
        return out, lse

    def _over_drafts(self, att, sizes, seen, q, table, length, first, out, lse, stream):
        """The rest of attend() where new tokens are drafts."""
        now = q.get_device()
        if seen.dtype is not self._int64[0] or seen.get_device() != now or seen.dim() != 1 or seen.numel() != att.n_tokens or \
                not seen.is_contiguous():
            _check(seen, "seen", self._int64, (att.n_tokens,))
        here = self._here
        if here.device() != now or seen.get_device() != now or self.k.get_device() != now:
            raise ValueError("q, seen, cache: on the current device")
        if stream is not None:
            here.stream(stream, now)
        n = self._ws_bytes.get(sizes)
        if n is None:
            if len(self._ws_bytes) > 1024:
                self._ws_bytes.clear()
            n = festina_attend_drafts_workspace_bytes(self.cache, att)
            if n:
                self._ws_bytes[sizes] = n
        held, ws, handle = self._ws.get(n, stream, q.device)
        st = self._attend_drafts(self._cache_ref, C.byref(att), seen.data_ptr(), ws, n, handle)
        if st != FESTINA_OK:
            raise FestinaError(st, "festina_attend_drafts")
        if stream is not None:
            _used_on(stream, q, table, length, first, seen, out, lse, self.k, self.v, self.k_scale, self.v_scale)
        return out, lse

    def keep(self, table, length, first, path, kept, also=(), stream=None):
        """Move the kept tokens of a step together, here and in the caches `also` (the other layers', of the same sizes): table,
        length (new tokens included) and first are the step's, path [tokens] and kept [requests] (int32) as from
        DeviceDrafts.accept."""
        here = self._here
        now = here.device()
        if table.dim() != 2 or table.dtype is not here.int32 or table.get_device() != now or not table.is_contiguous():
            _check(table, "table", self._int32, table.shape)
            raise ValueError(f"table: a contiguous tensor of two dimensions on the current device {now} is needed")
        R, columns = table.shape
        T = path.numel()
        q = festina_kept(R, columns, T, table.data_ptr(), here.ints(length, "length", R, now),
                         here.ints(first, "first", R + 1, now), here.ints(path, "path", T, now),
                         here.ints(kept, "kept", R, now))
        caches = (self, *also)
        structs = [c._struct for c in caches]
        for c in caches:
            if c._device != now:
                _on_device(c.k, "cache", now)
        if len(set(structs)) != len(structs):
            raise ValueError("also: each cache once (its tokens would be moved twice)")
        st = self._keep(b"".join(structs), len(structs), C.byref(q), here.stream(stream, now))
        if st != FESTINA_OK:
            raise FestinaError(st, "festina_keep_tokens")
        if stream is not None:
            _used_on(stream, table, length, first, path, kept, *(x for c in caches for x in (c.k, c.v, c.k_scale, c.v_scale)))


class DeviceDrafts:
    """The draft trees of a step (festina_drafts): int32 device tensors parent [tokens] (an index among its request's new
    tokens, -1 for node 0; None: each token's is the one before it) and, for accept(), token [tokens], used in place; tokens is
    the most that a step may have.

    plan() makes seen [tokens] (int64: bit j for node j; DeviceCache.attend) and position [tokens] (int32: DeviceRotary),
    accept() path [tokens], kept [n_requests], next [n_requests] and length [n_requests].  stream= as for DeviceBlocks.

    A request's new tokens are guesses but for node 0, and those that the model did not choose are not accepted.  The rest of
    a prompt stays where its tokens are a chain and choice holds each next one's token in the model's place (Server.verify's
    known does so); more than 64 new tokens are a run, kept whole, whose parents are not read."""

    def __init__(self, parent, token, n_requests: int, max_tokens=None, device=None):
        import torch
        given = [t for t in (parent, token) if t is not None]
        if max_tokens is None or device is None:
            if not given or not isinstance(given[0], torch.Tensor):
                raise ValueError("parent, token: a tensor is needed, or max_tokens and device")
            max_tokens = given[0].numel() if max_tokens is None else max_tokens
            device = given[0].device if device is None else device
        self.max_tokens, self.n_requests = int(max_tokens), int(n_requests)
        if self.max_tokens < 0 or self.n_requests < 0:
            raise ValueError("max_tokens and n_requests: not negative")
        for name, t in (("parent", parent), ("token", token)):
            if t is not None:
                _check(t, name, (torch.int32,), (self.max_tokens,))
        self.parent, self.token = parent, token
        i32 = lambda n: torch.empty(n, dtype=torch.int32, device=device)
        self.seen = torch.empty(self.max_tokens, dtype=torch.int64, device=device)
        for name, t in (("parent", parent), ("token", token)):
            if t is not None:
                _on_device(t, name, self.seen.get_device())
        self.position, self.path = i32(self.max_tokens), i32(self.max_tokens)
        self.kept, self.next, self.length = (i32(self.n_requests) for _ in range(3))
        self.accepted = festina_accepted(_ptr(self.path), _ptr(self.kept), _ptr(self.next), _ptr(self.length))
        self._here, self._plan, self._accept = _Here(), lib().festina_plan_drafts, lib().festina_accept_drafts

    def _drafts(self, first, length, now):
        if self.kept.get_device() != now:
            _on_device(self.kept, "the drafts", now)
        here = self._here
        return festina_drafts(self.n_requests, self.max_tokens, here.ints(first, "first", self.n_requests + 1, now),
                              here.ints(length, "length", self.n_requests, now),
                              None if self.parent is None else self.parent.data_ptr())

    def plan(self, first, length, stream=None):
        """What the nodes see and where they stand; first and length are the step's (DeviceBlocks)."""
        now = self._here.device()
        st = self._plan(C.byref(self._drafts(first, length, now)), self.seen.data_ptr(), self.position.data_ptr(),
                        self._here.stream(stream, now))
        if st != FESTINA_OK:
            raise FestinaError(st, "festina_plan_drafts")
        if stream is not None:
            _used_on(stream, first, length, *self._tensors())

    def accept(self, first, length, choice, stream=None):
        """The nodes that the model's choice [max_tokens] (int32: the token chosen behind each) accepts."""
        if self.token is None:
            raise ValueError("token: the drafted tokens are needed")
        now = self._here.device()
        st = self._accept(C.byref(self._drafts(first, length, now)), self.token.data_ptr(),
                          self._here.ints(choice, "choice", self.max_tokens, now), C.byref(self.accepted),
                          self._here.stream(stream, now))
        if st != FESTINA_OK:
            raise FestinaError(st, "festina_accept_drafts")
        if stream is not None:
            _used_on(stream, first, length, choice, *self._tensors())

    def _tensors(self):
        return [t for t in (self.parent, self.token, self.seen, self.position, self.path, self.kept, self.next, self.length)
                if t is not None]


class DeviceRotary:
    """Norm and rotation of queries and keys (festina_rotary): freq, radians per position of each rotated pair (host numbers,
    at most head_dim / 2), weights of the heads' norms or None (copied), and whether pairs are neighbours (interleaved) or half of the
    rotated elements apart.  What a model's layers share of these is kept once and may be used by all."""

    def __init__(self, freq, head_dim: int, q_weight=None, k_weight=None, eps: float = 1e-6, interleaved: bool = False,
                 device="cuda"):
        import torch
        turn = np.array([_turn(float(f)) for f in np.asarray(freq, np.float64).reshape(-1)], np.uint64)
        self.turn = torch.from_numpy(turn.view(np.int64)).to(device)
        self.weights = []
        for name, w in (("q_weight", q_weight), ("k_weight", k_weight)):
            if w is not None and tuple(w.shape) != (int(head_dim),):
                raise ValueError(f"{name}: shape ({int(head_dim)},), not {tuple(w.shape)}")
            self.weights.append(None if w is None else w.detach().to(device=device, dtype=torch.float32).contiguous().clone())
        self.head_dim = int(head_dim)
        self.rotary = festina_rotary(self.head_dim, 2 * len(turn), 1 if interleaved else 0, float(eps), _ptr(self.turn),
                                     *(_ptr(w) for w in self.weights))
        self._types = {torch.bfloat16: FESTINA_BF16, torch.float16: FESTINA_F16, torch.float32: FESTINA_F32}
        self._here, self._empty, self._graded, self._dual = _Here(), torch.empty, torch.is_grad_enabled, _dual_levels()
        self._rotate, self._ref = lib().festina_rotate_heads, C.byref(self.rotary)

    def apply(self, q, k, position, q_out=None, k_out=None, stream=None):
        """(q_out, k_out): queries and keys [tokens][heads][head_dim] of one type (any strides but the last) at the int32
        positions [tokens].  Outputs are made where not given, and may be q and k themselves, else they share no memory with either
        nor with each other.  For serving: inputs that ask for a gradient or carry a tangent are refused."""
        return self._apply(q, k, position, q_out, k_out, stream, q_out, k_out)

    def _apply(self, q, k, position, q_out, k_out, stream, q_given, k_given):
        here, D, dtype = self._here, self.head_dim, q.dtype
        now, kind = here.device(), self._types.get(dtype)
        if stream is not None and (q_out is None or k_out is None):
            with _on(stream, q.device):
                return self._apply(q, k, position, self._empty(q.shape, dtype=dtype, device=q.device) if q_out is None else q_out,
                                   self._empty(k.shape, dtype=k.dtype, device=k.device) if k_out is None else k_out, stream,
                                   q_given, k_given)
        if q.dim() != 3 or k.dim() != 3:
            raise ValueError("q and k: [tokens][heads][dim]")
        T, heads, qd = q.shape
        tokens, kv_heads, kd = k.shape
        qt, qh, qs = q.stride()
        kt, kh, ks = k.stride()
        if kind is None or k.dtype is not dtype or q.get_device() != now or k.get_device() != now or tokens != T or qd != D or \
                kd != D or (qs != 1 and q.numel()) or (ks != 1 and k.numel()):
            _check(q, "q", self._types)
            _check(k, "k", (dtype,))
            _on_device(q, "q", now)
            _on_device(k, "k", now)
            raise ValueError(f"q and k: [{T}][heads][{D}] with their last axis contiguous")
        if ((q.requires_grad or k.requires_grad) and self._graded()) or (self._dual._current_level >= 0 and _tangents(q, k)):
            raise ValueError("q, k: no gradient passes through (call under torch.no_grad(), without tangents)")
        if q_given is not None or k_given is not None:
            self._given(q, k, q_given, k_given, now)
        if q_out is None:
            q_out = self._empty((T, heads, D), dtype=dtype, device=q.device)
            ot, oh = heads * D, D
        else:
            ot, oh, _ = q_out.stride()
        if k_out is None:
            k_out = self._empty((T, kv_heads, D), dtype=dtype, device=q.device)
            pt, ph = kv_heads * D, D
        else:
            pt, ph, _ = k_out.stride()
        if self.turn.get_device() != now:
            _on_device(self.turn, "the rotary", now)
        st = self._rotate(self._ref, C.byref(festina_heads(
            T, heads, kv_heads, kind, here.ints(position, "position", T, now), q.data_ptr(), k.data_ptr(), qt, qh, kt, kh,
            q_out.data_ptr(), k_out.data_ptr(), ot, oh, pt, ph)), here.stream(stream, now))
        if st != FESTINA_OK:
            raise FestinaError(st, "festina_rotate_heads")
        if stream is not None:
            _used_on(stream, q, k, position, q_out, k_out, self.turn, *(w for w in self.weights if w is not None))
        return q_out, k_out

    def _given(self, q, k, q_out, k_out, now):
        """Outputs that the caller brings: a token's heads are several waves' work, so what one writes no other may read or write."""
        D = self.head_dim
        x, y = _place(q, D), _place(k, D)
        places = []
        for out, name, t, own, other in ((q_out, "q_out", q, x, y), (k_out, "k_out", k, y, x)):
            if out is None:
                continue
            at = own
            if out is not t:
                if out.dtype is not t.dtype or out.get_device() != now:
                    _check(out, name, (t.dtype,))
                    _on_device(out, name, now)
                if out.shape != t.shape or (out.stride(2) != 1 and out.numel()):
                    raise ValueError(f"{name}: the shape {tuple(t.shape)} with its last axis contiguous")
                if (out.requires_grad and self._graded()) or (self._dual._current_level >= 0 and _tangents(out)):
                    raise ValueError(f"{name}: no gradient passes through (call under torch.no_grad(), without tangents)")
                at = _place(out, D)
                if at != own and at[1] > own[0] and own[1] > at[0] and _meet(at, own, D):
                    raise ValueError(f"{name}: the input's own memory with its strides, or other memory")
            if not _once(at, D):
                raise ValueError(f"{name}: an element of its own for each of the input")
            if at[1] > other[0] and other[1] > at[0] and _meet(at, other, D):
                raise ValueError(f"{name}: shares memory with the other input")
            places.append(at)
            if q_out is q and k_out is k:                    # in place: all has been looked at
                if not _once(y, D):
                    raise ValueError("k_out: an element of its own for each of the input")
                return
        if len(places) == 2 and _meet(*places, D):
            raise ValueError("q_out and k_out: share memory")


def _place(t, D):
    """Where a tensor [tokens][heads][D] lies, in elements: its begin and end, sizes, and strides (0 where they do not count)."""
    (T, H, _), (s, p, _) = t.shape, t.stride()
    if T <= 1:
        s = 0
    if H <= 1:
        p = 0
    a = t.data_ptr() // t.element_size()
    return a, a + (T - 1) * s + (H - 1) * p + D, T, H, s, p


def _starts(x):
    a, _, T, H, s, p = x
    return np.sort((a + np.arange(T, dtype=np.int64)[:, None] * s + np.arange(H, dtype=np.int64) * p).ravel())


def _meet(x, y, D) -> bool:
    """Whether two tensors [tokens][heads][D] of one type with contiguous last axes (their _place) share an element."""
    (a, a_end, T, H, s, p), (b, b_end, U, K, r, q) = x, y
    if a_end <= b or b_end <= a or not (T * H and U * K and D):
        return False
    if s == r and s:                                         # side by side in each token
        width, other, d = (H - 1) * p + D, (K - 1) * q + D, (b - a) % s
        if width <= d and d + other <= s:
            return False
    step = math.gcd(s, p, r, q)                              # or in each head
    if step and D <= (b - a) % step <= step - D:
        return False
    starts, at = _starts(y), _starts(x)
    return bool((np.searchsorted(starts, at - D, "right") < np.searchsorted(starts, at + D, "left")).any())


def _once(x, D) -> bool:
    """Whether such a tensor has each of its elements at a place of its own."""
    _, _, T, H, s, p = x
    if not (T * H and D):
        return True
    (inner, n), (outer, m) = ((s, T), (p, H)) if (T > 1 and s <= p) or H <= 1 else ((p, H), (s, T))
    if (n <= 1 or inner >= D) and (m <= 1 or outer >= (n - 1) * inner + D):
        return True
    starts = _starts(x)
    return bool((starts[1:] - starts[:-1] >= D).all())


def _turn(radians: float) -> int:
    """Radians as a part of a turn times 2^64, rounded to a whole number (the float taken as it is, pi to 60 digits)."""
    from fractions import Fraction
    if not np.isfinite(radians):
        raise ValueError("freq: finite numbers")
    turn = Fraction(radians) / (2 * Fraction(314159265358979323846264338327950288419716939937510582097494, 10 ** 59))
    return round(turn * 2 ** 64) % 2 ** 64


# ------------------------------------------------------------------ the ABI calls
def festina_placements_workspace_bytes(lut, gpus, req) -> int:
    return int(lib().festina_placements_workspace_bytes(C.byref(lut), C.byref(gpus), C.byref(req)))


def _events(events):
    b, e = events
    return (C.c_void_p(b) if b else None), (C.c_void_p(e) if e else None)


def festina_score_placements(lut, gpus, req, out, workspace, workspace_bytes, stream=None, events=None) -> None:
    """festina_score_placements, or festina_score_placements_timed when `events` = (begin, end)
    raw hipEvent_t handles."""
    ws = None if workspace is None else C.c_void_p(workspace.data_ptr())
    args = (C.byref(lut), C.byref(gpus), C.byref(req), C.byref(out), ws, int(workspace_bytes),
            _stream_handle(stream))
    if events is None:
        st = lib().festina_score_placements(*args)
    else:
        st = lib().festina_score_placements_timed(*args, *_events(events))
    if st != FESTINA_OK:
        raise FestinaError(st, "festina_score_placements")


def festina_score_placements_noalloc(lut, gpus, req, out, stream=None) -> None:
    st = lib().festina_score_placements_noalloc(C.byref(lut), C.byref(gpus), C.byref(req), C.byref(out),
                                                _stream_handle(stream))
    if st != FESTINA_OK:
        raise FestinaError(st, "festina_score_placements_noalloc")


def festina_migrations_workspace_bytes(lut, fleet) -> int:
    return int(lib().festina_migrations_workspace_bytes(C.byref(lut), C.byref(fleet)))


def festina_score_migrations(lut, fleet, out, workspace, workspace_bytes, stream=None, events=None) -> None:
    """festina_score_migrations, or festina_score_migrations_timed when `events` = (begin, end)
    raw hipEvent_t handles."""
    ws = None if workspace is None else C.c_void_p(workspace.data_ptr())
    args = (C.byref(lut), C.byref(fleet), C.byref(out), ws, int(workspace_bytes), _stream_handle(stream))
    if events is None:
        st = lib().festina_score_migrations(*args)
    else:
        st = lib().festina_score_migrations_timed(*args, *_events(events))
    if st != FESTINA_OK:
        raise FestinaError(st, "festina_score_migrations")


def festina_sweep_batches(lut, batches, out, stream=None) -> None:
    st = lib().festina_sweep_batches(C.byref(lut), C.byref(batches), C.byref(out), _stream_handle(stream))
    if st != FESTINA_OK:
        raise FestinaError(st, "festina_sweep_batches")


def festina_preferred_configs(lut, llms, out, stream=None) -> None:
    st = lib().festina_preferred_configs(C.byref(lut), C.byref(llms), C.byref(out), _stream_handle(stream))
    if st != FESTINA_OK:
        raise FestinaError(st, "festina_preferred_configs")


def festina_ewr_workspace_bytes(n_gpus: int) -> int:
    return int(lib().festina_ewr_workspace_bytes(int(n_gpus)))


def festina_fleet_ewr(n_gpus, max_inst, n_inst, f_pref, t_ms, out, workspace, workspace_bytes, stream=None) -> None:
    ws = None if workspace is None else C.c_void_p(workspace.data_ptr())
    st = lib().festina_fleet_ewr(int(n_gpus), int(max_inst), _ptr(n_inst), _ptr(f_pref), _ptr(t_ms), C.byref(out),
                                 ws, int(workspace_bytes), _stream_handle(stream))
    if st != FESTINA_OK:
        raise FestinaError(st, "festina_fleet_ewr")


def festina_dispatch_workspace_bytes(lut, avail) -> int:
    return int(lib().festina_dispatch_workspace_bytes(C.byref(lut), C.byref(avail)))


def festina_dispatch_requests(lut, avail, req, out, workspace, workspace_bytes, stream=None) -> None:
    ws = None if workspace is None else C.c_void_p(workspace.data_ptr())
    st = lib().festina_dispatch_requests(C.byref(lut), C.byref(avail), C.byref(req), C.byref(out), ws,
                                         int(workspace_bytes), _stream_handle(stream))
    if st != FESTINA_OK:
        raise FestinaError(st, "festina_dispatch_requests")


def festina_dispatch_waves_workspace_bytes(lut, avail) -> int:
    return int(lib().festina_dispatch_waves_workspace_bytes(C.byref(lut), C.byref(avail)))


def festina_dispatch_waves(lut, avail, req, wave_start, state, out, workspace, workspace_bytes, stream=None) -> None:
    """wave_start: host sequence of n_waves + 1 request offsets."""
    ws = None if workspace is None else C.c_void_p(workspace.data_ptr())
    bounds = np.ascontiguousarray(wave_start, dtype=np.int32)
    st = lib().festina_dispatch_waves(C.byref(lut), C.byref(avail), C.byref(req), int(bounds.size) - 1,
                                      bounds.ctypes.data if bounds.size else None, C.byref(state), C.byref(out), ws,
                                      int(workspace_bytes), _stream_handle(stream))
    if st != FESTINA_OK:
        raise FestinaError(st, "festina_dispatch_waves")


def festina_transfer_costs(transfer, cost, stream=None) -> None:
    st = lib().festina_transfer_costs(C.byref(transfer), _ptr(cost), _stream_handle(stream))
    if st != FESTINA_OK:
        raise FestinaError(st, "festina_transfer_costs")


def festina_request_moves(lut, transfer, plan, req, out, stream=None) -> None:
    st = lib().festina_request_moves(C.byref(lut), C.byref(transfer), C.byref(plan), C.byref(req), C.byref(out),
                                     _stream_handle(stream))
    if st != FESTINA_OK:
        raise FestinaError(st, "festina_request_moves")


def festina_blocks_workspace_bytes(n_requests: int, max_tokens: int) -> int:
    return int(lib().festina_blocks_workspace_bytes(int(n_requests), int(max_tokens)))


def festina_extend_blocks(req, out, workspace, workspace_bytes, stream=None) -> None:
    """workspace: the address of device memory (here and in the calls below)."""
    st = lib().festina_extend_blocks(C.byref(req), C.byref(out), workspace, int(workspace_bytes),
                                     _stream_handle(stream))
    if st != FESTINA_OK:
        raise FestinaError(st, "festina_extend_blocks")


def festina_release_blocks(req, done, out, workspace, workspace_bytes, stream=None) -> None:
    st = lib().festina_release_blocks(C.byref(req), _ptr(done), C.byref(out), workspace, int(workspace_bytes),
                                      _stream_handle(stream))
    if st != FESTINA_OK:
        raise FestinaError(st, "festina_release_blocks")


def festina_store_kv(cache, tokens, stream=None) -> None:
    st = lib().festina_store_kv(C.byref(cache), C.byref(tokens), _stream_handle(stream))
    if st != FESTINA_OK:
        raise FestinaError(st, "festina_store_kv")


def festina_attend_workspace_bytes(cache, att) -> int:
    return int(lib().festina_attend_workspace_bytes(C.byref(cache), C.byref(att)))


def festina_attend(cache, att, workspace, workspace_bytes, stream=None) -> None:
    st = lib().festina_attend(C.byref(cache), C.byref(att), workspace, int(workspace_bytes),
                              _stream_handle(stream))
    if st != FESTINA_OK:
        raise FestinaError(st, "festina_attend")


def festina_trim_blocks(req, keep, out, workspace, workspace_bytes, stream=None) -> None:
    st = lib().festina_trim_blocks(C.byref(req), _ptr(keep), C.byref(out), workspace, int(workspace_bytes),
                                   _stream_handle(stream))
    if st != FESTINA_OK:
        raise FestinaError(st, "festina_trim_blocks")


def festina_plan_drafts(drafts, seen, position, stream=None) -> None:
    st = lib().festina_plan_drafts(C.byref(drafts), _ptr(seen), _ptr(position), _stream_handle(stream))
    if st != FESTINA_OK:
        raise FestinaError(st, "festina_plan_drafts")


def festina_accept_drafts(drafts, token, choice, out, stream=None) -> None:
    st = lib().festina_accept_drafts(C.byref(drafts), _ptr(token), _ptr(choice), C.byref(out), _stream_handle(stream))
    if st != FESTINA_OK:
        raise FestinaError(st, "festina_accept_drafts")


def festina_attend_drafts_workspace_bytes(cache, att) -> int:
    return int(lib().festina_attend_drafts_workspace_bytes(C.byref(cache), C.byref(att)))


def festina_attend_drafts(cache, att, seen, workspace, workspace_bytes, stream=None) -> None:
    st = lib().festina_attend_drafts(C.byref(cache), C.byref(att), _ptr(seen), workspace, int(workspace_bytes),
                                     _stream_handle(stream))
    if st != FESTINA_OK:
        raise FestinaError(st, "festina_attend_drafts")


def festina_keep_tokens(caches, n_caches: int, kept, stream=None) -> None:
    """caches: a ctypes array of festina_kv_cache."""
    st = lib().festina_keep_tokens(caches, int(n_caches), C.byref(kept), _stream_handle(stream))
    if st != FESTINA_OK:
        raise FestinaError(st, "festina_keep_tokens")


def festina_rotate_heads(rotary, heads, stream=None) -> None:
    st = lib().festina_rotate_heads(C.byref(rotary), C.byref(heads), _stream_handle(stream))
    if st != FESTINA_OK:
        raise FestinaError(st, "festina_rotate_heads")
