"""Python binding of librubick.so (include/rubick.h): argument marshalling only.

Every computation runs in the HIP library; PyTorch supplies device memory and
the stream.  Importing the module does not need a GPU; loading the library
does, and fails loudly when the library has not been built.
"""
from __future__ import annotations

import ctypes as C
import os

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "librubick.so")

RK_OK, RK_ERR_INVALID_ARG, RK_ERR_CAPACITY, RK_ERR_DEVICE, RK_ERR_UNSUPPORTED = 0, -1, -2, -3, -4
RK_NO_PLAN = 0xFFFFFFFF
RK_MAX_CPU_LEVELS, RK_MAX_MEM_LEVELS = 64, 16
RK_MAX_JOBS_PER_ROUND = 12288
RK_STATIC_MAX_STEPS = 524288
RK_MAX_TENANTS = 256
RK_FIT_PARAMS, RK_FIT_MAX_STARTS, RK_FIT_MAX_SAMPLES, RK_FIT_K_MAX = 7, 8, 64, 32.0
FIT_FIELDS = ("k_bwd", "k_sync", "k_opt", "k_opt_off", "k_off", "k_swap", "k_const")

EXPORTS = ("rk_create", "rk_destroy", "rk_sync", "rk_workspace_bytes", "rk_last_error", "rk_enumerate_plans", "rk_eval_candidates",
           "rk_best_plan", "rk_curves", "rk_job_curves", "rk_allocate", "rk_schedule_round", "rk_schedule_rounds",
           "rk_eval_points", "rk_min_res", "rk_allocate_sla", "rk_schedule_round_sla", "rk_fit_models", "rk_simulate", "rk_schedule_rounds_shared", "rk_place", "rk_allocate_static", "rk_place_plans",
           "rk_schedule_round_placed", "rk_reschedule", "rk_probe_stream", "rk_eval_best_plan", "rk_reschedule_nodes", "rk_best_plan_placed", "rk_reschedule_rounds", "rk_schedule_round_nodes", "rk_privileged", "rk_curve_slopes",
           "rk_norm_forward", "rk_norm_backward", "rk_route_forward", "rk_route_backward", "rk_distill_loss",
           "rk_distill_backward", "rk_distill_loss_backward",
           "rk_recur_forward", "rk_recur_backward", "rk_dropout_forward", "rk_dropout_backward", "rk_head_loss", "rk_head_backward",
           "rk_head_loss_backward")

_JOB_F32 = ("P_bytes", "seq", "hidden", "elem_bytes", "t_fwd_sample", "k_bwd", "k_sync", "k_opt", "k_opt_off",
            "k_off", "k_swap", "k_const", "mem_state", "mem_act", "mem_act_gc", "mem_const", "ref_thr")
_JOB_U32 = ("layers", "gbatch", "mbatch")


class rk_jobs(C.Structure):
    _fields_ = [("n_jobs", C.c_uint32)] + [(n, C.c_void_p) for n in _JOB_F32 + _JOB_U32]


class rk_plan_bounds(C.Structure):
    _fields_ = [(n, C.c_uint32) for n in ("g_max", "tp_max", "pp_max", "zero_mask", "gc_mask", "off_mask", "mu_mask")]


class rk_plan_table(C.Structure):
    _fields_ = [("triple_off", C.c_void_p), ("triples", C.c_void_p), ("seg_off", C.c_void_p),
                ("seg_g", C.c_void_p), ("seg_first", C.c_void_p),
                ("cap_triples", C.c_uint64), ("cap_segs", C.c_uint64),
                ("h_triple_off", C.c_void_p), ("h_seg_off", C.c_void_p),
                ("n_triples", C.c_uint64), ("n_segs", C.c_uint64), ("n_jobs", C.c_uint32),
                ("max_triples_per_job", C.c_uint32), ("max_segs_per_job", C.c_uint32),
                ("option_mask", C.c_uint32)]


class rk_alloc_grid(C.Structure):
    _fields_ = [("n_cpu", C.c_uint32), ("cpu_levels", C.c_uint32 * RK_MAX_CPU_LEVELS), ("cpu_mode", C.c_uint32),
                ("n_mem", C.c_uint32), ("mem_levels_gb", C.c_float * RK_MAX_MEM_LEVELS), ("mem_mode", C.c_uint32)]


class rk_env(C.Structure):
    _fields_ = [("B_intra", C.c_float), ("B_inter", C.c_float), ("B_pcie", C.c_float),
                ("gpu_mem_cap", C.c_float), ("gpus_per_node", C.c_uint32)]


class rk_cluster(C.Structure):
    _fields_ = [("G", C.c_uint32), ("C", C.c_uint32), ("host_mem_gb", C.c_float)]


class rk_sla(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("guaranteed", "tenant", "req_g", "req_c", "req_m", "base_thr")] + \
               [("n_tenants", C.c_uint32), ("quota_g", C.c_void_p), ("quota_c", C.c_void_p)]


class rk_samples(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("sample_off", "triple", "option", "cpus", "thr")] + [("max_samples", C.c_uint32)]


class rk_fit_options(C.Structure):
    _fields_ = [("max_iter", C.c_uint32), ("refit_threshold", C.c_float), ("n_starts", C.c_uint32),
                ("start_offsets", C.c_void_p)]


class rk_fit_result(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in FIT_FIELDS + ("theta", "rmsle_before", "rmsle_after", "iters")]


class rk_trace(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("arrival", "work", "delta")]


class rk_sim_options(C.Structure):
    _fields_ = [("dt", C.c_double), ("n_ticks", C.c_uint32), ("policy", C.c_uint32), ("gate", C.c_double),
                ("nodes", C.c_void_p)]


class rk_sim_result(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("finish", "n_reconf", "progress", "held", "gpus_in_use", "totals", "frozen")]


ASSIGN_DTYPE = np.dtype([("g", np.uint32), ("c", np.uint32), ("mem_gb", np.float32),
                         ("plan", np.uint32), ("thr", np.float32)])


class RkError(RuntimeError):
    def __init__(self, code, text):
        super().__init__(f"librubick error {code}: {text}")
        self.code = code


_lib = None


def load_library():
    """Load librubick.so; raises if it has not been built (no CPU fallback exists)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_2408_08586_amd.build`")
        lib = C.CDLL(LIB_PATH)
        for name in EXPORTS:
            getattr(lib, name).restype = C.c_int32
        lib.rk_last_error.restype = C.c_char_p
        _lib = lib
    return _lib


# ------------------------------------------------------------------ marshalling helpers
def make_bounds(b) -> rk_plan_bounds:
    return rk_plan_bounds(b.g_max, b.tp_max, b.pp_max, b.zero_mask, b.gc_mask, b.off_mask, getattr(b, "mu_mask", 1))


def make_grid(g) -> rk_alloc_grid:
    out = rk_alloc_grid()
    cpu = [int(v) for v in g.cpu_levels]
    mem = [float(v) for v in g.mem_levels_gb]
    out.n_cpu, out.cpu_mode, out.n_mem, out.mem_mode = len(cpu), int(g.cpu_mode), len(mem), int(g.mem_mode)
    for i, v in enumerate(cpu[:RK_MAX_CPU_LEVELS]):
        out.cpu_levels[i] = v
    for i, v in enumerate(mem[:RK_MAX_MEM_LEVELS]):
        out.mem_levels_gb[i] = v
    return out


def make_env(e) -> rk_env:
    return rk_env(e.B_intra, e.B_inter, e.B_pcie, e.gpu_mem_cap, e.gpus_per_node)


def make_cluster(c) -> rk_cluster:
    return rk_cluster(int(c.G), int(c.C), float(c.host_mem_gb))


def _ptr(t):
    return C.c_void_p(0 if t is None else t.data_ptr())


def _check(ctx, rc):
    if rc != RK_OK:
        raise RkError(rc, rk_last_error(ctx))


class Jobs:
    """Job descriptors on the device, struct of arrays."""

    def __init__(self, coef: np.ndarray, ints: np.ndarray, device="cuda:0"):
        import torch
        coef = np.ascontiguousarray(coef, dtype=np.float32)
        ints = np.ascontiguousarray(ints, dtype=np.uint32)
        assert coef.ndim == 2 and coef.shape[1] == len(_JOB_F32) and ints.shape == (coef.shape[0], len(_JOB_U32))
        self.n_jobs = coef.shape[0]
        self.f32 = torch.from_numpy(np.ascontiguousarray(coef.T)).to(device)                       # [17, J]
        self.u32 = torch.from_numpy(np.ascontiguousarray(ints.T).view(np.int32)).to(device)        # [3, J]
        self.c = rk_jobs()
        self.c.n_jobs = self.n_jobs
        stride = self.n_jobs * 4
        for k, name in enumerate(_JOB_F32):
            setattr(self.c, name, self.f32.data_ptr() + k * stride)
        for k, name in enumerate(_JOB_U32):
            setattr(self.c, name, self.u32.data_ptr() + k * stride)

    @property
    def ref_thr(self):
        return self.f32[len(_JOB_F32) - 1]


class PlanTable:
    """Device buffers of a plan table plus the C struct that points at them."""

    def __init__(self, n_jobs, cap_triples, cap_segs, device="cuda:0"):
        import torch
        i32 = dict(dtype=torch.int32, device=device)
        self.triple_off = torch.zeros(n_jobs + 1, **i32)
        self.seg_off = torch.zeros(n_jobs + 1, **i32)
        self.triples = torch.zeros(max(cap_triples, 1), **i32)
        self.seg_g = torch.zeros(max(cap_segs, 1), **i32)
        self.seg_first = torch.zeros(max(cap_segs, 1), **i32)
        self.h_triple_off = np.zeros(n_jobs + 1, np.uint32)
        self.h_seg_off = np.zeros(n_jobs + 1, np.uint32)
        self.c = rk_plan_table()
        self.c.triple_off, self.c.triples = self.triple_off.data_ptr(), self.triples.data_ptr()
        self.c.seg_off, self.c.seg_g, self.c.seg_first = (self.seg_off.data_ptr(), self.seg_g.data_ptr(),
                                                          self.seg_first.data_ptr())
        self.c.cap_triples, self.c.cap_segs = cap_triples, cap_segs
        self.c.h_triple_off = self.h_triple_off.ctypes.data
        self.c.h_seg_off = self.h_seg_off.ctypes.data
        self.c.n_jobs = n_jobs

    n_triples = property(lambda self: int(self.c.n_triples))
    n_segs = property(lambda self: int(self.c.n_segs))
    n_jobs = property(lambda self: int(self.c.n_jobs))

    def n_candidates(self, n_rows, jb=0, je=None):
        je = self.n_jobs if je is None else je
        return 16 * n_rows * int(self.h_triple_off[je] - self.h_triple_off[jb])

    def n_segments(self, n_rows, jb=0, je=None):
        je = self.n_jobs if je is None else je
        return n_rows * int(self.h_seg_off[je] - self.h_seg_off[jb])

    def unpack_triples(self) -> np.ndarray:
        """Host copy of the triples as (d, t, p) rows."""
        x = self.triples[:self.n_triples].cpu().numpy().view(np.uint32)
        return np.stack([x & 0xFFFF, 1 << ((x >> 16) & 3), (x >> 18) & 0xFFF, x >> 30], axis=1).astype(np.uint32)


# ------------------------------------------------------------------ the C ABI, same names
def rk_create(device_id=0, stream=None):
    """stream: a torch.cuda.Stream, a raw hipStream_t value, or None for the current torch stream."""
    import torch
    lib = load_library()
    if stream is None:
        stream = torch.cuda.current_stream(device_id).cuda_stream
    elif hasattr(stream, "cuda_stream"):
        stream = stream.cuda_stream
    ctx = C.c_void_p()
    rc = lib.rk_create(C.byref(ctx), C.c_int32(device_id), C.c_void_p(stream))
    if rc != RK_OK:
        raise RkError(rc, "rk_create failed")
    return ctx


def rk_destroy(ctx):
    return load_library().rk_destroy(ctx)


def rk_sync(ctx):
    _check(ctx, load_library().rk_sync(ctx))


def rk_workspace_bytes(ctx) -> int:
    """Bytes of device memory in the context's working buffers."""
    bytes_ = C.c_uint64()
    rc = load_library().rk_workspace_bytes(ctx, C.byref(bytes_))
    if rc != RK_OK:
        raise RkError(rc, "rk_workspace_bytes failed")
    return bytes_.value


def rk_last_error(ctx) -> str:
    return load_library().rk_last_error(ctx).decode()


def rk_enumerate_plans(ctx, jobs: Jobs, bounds: rk_plan_bounds, table: rk_plan_table):
    _check(ctx, load_library().rk_enumerate_plans(ctx, C.byref(jobs.c), C.byref(bounds), C.byref(table)))


def rk_eval_candidates(ctx, jobs: Jobs, table: rk_plan_table, grid: rk_alloc_grid, env: rk_env,
                       job_begin, job_end, thr, feas=None):
    need = C.c_uint64(0)
    _check(ctx, load_library().rk_eval_candidates(ctx, C.byref(jobs.c), C.byref(table), C.byref(grid), C.byref(env),
                                                  C.c_uint32(job_begin), C.c_uint32(job_end), _ptr(thr), _ptr(feas),
                                                  C.c_uint64(0 if thr is None else thr.numel()), C.byref(need)))
    return need.value


def rk_best_plan(ctx, table: rk_plan_table, grid: rk_alloc_grid, job_begin, job_end, thr, best_thr, best_plan):
    need = C.c_uint64(0)
    _check(ctx, load_library().rk_best_plan(ctx, C.byref(table), C.byref(grid), C.c_uint32(job_begin),
                                            C.c_uint32(job_end), _ptr(thr), _ptr(best_thr), _ptr(best_plan),
                                            C.c_uint64(0 if best_thr is None else best_thr.numel()), C.byref(need)))
    return need.value


def rk_eval_best_plan(ctx, jobs: Jobs, table: rk_plan_table, grid: rk_alloc_grid, env: rk_env, job_begin, job_end, thr,
                      best_thr, best_plan, feas=None):
    _check(ctx, load_library().rk_eval_best_plan(ctx, C.byref(jobs.c), C.byref(table), C.byref(grid), C.byref(env),
                                                 C.c_uint32(job_begin), C.c_uint32(job_end), _ptr(thr), _ptr(feas),
                                                 C.c_uint64(0 if thr is None else thr.numel()), _ptr(best_thr),
                                                 _ptr(best_plan), C.c_uint64(0 if best_thr is None else best_thr.numel())))


def rk_curves(ctx, table, grid, job_begin, job_end, best_thr, best_plan, curve_thr, curve_plan, curve_g):
    _check(ctx, load_library().rk_curves(ctx, C.byref(table), C.byref(grid), C.c_uint32(job_begin),
                                         C.c_uint32(job_end), _ptr(best_thr), _ptr(best_plan), _ptr(curve_thr),
                                         _ptr(curve_plan), _ptr(curve_g), C.c_uint64(curve_thr.numel())))


def rk_job_curves(ctx, jobs: Jobs, table, grid, env, job_begin, job_end, best_thr, best_plan,
                  curve_thr, curve_plan, curve_g):
    _check(ctx, load_library().rk_job_curves(ctx, C.byref(jobs.c), C.byref(table), C.byref(grid), C.byref(env),
                                             C.c_uint32(job_begin), C.c_uint32(job_end), _ptr(best_thr),
                                             _ptr(best_plan), _ptr(curve_thr), _ptr(curve_plan), _ptr(curve_g),
                                             C.c_uint64(curve_thr.numel())))


def rk_allocate(ctx, ref_thr, table, grid, cluster: rk_cluster, job_begin, job_end, best_thr, best_plan,
                curve_thr, assign, total):
    _check(ctx, load_library().rk_allocate(ctx, _ptr(ref_thr), C.byref(table), C.byref(grid), C.byref(cluster),
                                           C.c_uint32(job_begin), C.c_uint32(job_end), _ptr(best_thr),
                                           _ptr(best_plan), _ptr(curve_thr), _ptr(assign), _ptr(total)))


def rk_allocate_static(ctx, ref_thr, table, grid, cluster: rk_cluster, job_begin, job_end, best_thr, best_plan,
                       curve_thr, assign, total):
    _check(ctx, load_library().rk_allocate_static(ctx, _ptr(ref_thr), C.byref(table), C.byref(grid), C.byref(cluster),
                                                  C.c_uint32(job_begin), C.c_uint32(job_end), _ptr(best_thr),
                                                  _ptr(best_plan), _ptr(curve_thr), _ptr(assign), _ptr(total)))


class rk_job_state(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("state", "cur_seg", "cur_c", "floor_seg", "floor_c")]


def rk_reschedule(ctx, ref_thr, table, grid, cluster: rk_cluster, best_thr, best_plan, curve_thr, cur_seg, cur_c, assign,
                  total, state=None, floor_seg=None, floor_c=None, n_moves=None):
    """Algorithm 1's Schedule loop from the jobs' present state (device tensors; state is uint8, cur_seg / floor_seg int32)."""
    js = rk_job_state(_ptr(state), _ptr(cur_seg), _ptr(cur_c), _ptr(floor_seg), _ptr(floor_c))
    _check(ctx, load_library().rk_reschedule(ctx, _ptr(ref_thr), C.byref(table), C.byref(grid), C.byref(cluster),
                                             _ptr(best_thr), _ptr(best_plan), _ptr(curve_thr), C.byref(js), _ptr(assign),
                                             _ptr(total), _ptr(n_moves)))


def rk_curve_slopes(ctx, ref_thr, table, grid, job_begin, job_end, best_thr, curve_thr, gpu_slope, gpu_next, from0_slope,
                    from0_next, cpu_slope, cpu_next):
    """The slope table of the curves (device tensors; capacity = size of gpu_slope)."""
    _check(ctx, load_library().rk_curve_slopes(ctx, _ptr(ref_thr), C.byref(table), C.byref(grid), C.c_uint32(job_begin),
                                               C.c_uint32(job_end), _ptr(best_thr), _ptr(curve_thr), _ptr(gpu_slope),
                                               _ptr(gpu_next), _ptr(from0_slope), _ptr(from0_next), _ptr(cpu_slope),
                                               _ptr(cpu_next), C.c_uint64(gpu_slope.numel())))


def rk_privileged(ctx, table, grid, sla: "Sla", min_seg, min_c, cur_seg, cur_c, floor_seg, floor_c, state_out, state=None):
    """Floors and states for the Schedule loops from the service levels (device tensors; state tensors are uint8)."""
    held = rk_job_state(_ptr(state), _ptr(cur_seg), _ptr(cur_c), None, None)
    _check(ctx, load_library().rk_privileged(ctx, C.byref(table), C.byref(grid), C.byref(sla.c), _ptr(min_seg), _ptr(min_c),
                                             C.byref(held), _ptr(floor_seg), _ptr(floor_c), _ptr(state_out)))


def rk_reschedule_rounds(ctx, ref_thr, table, grid, clusters, best_thr, best_plan, curve_thr, cur_seg, cur_c, assign, totals,
                         state_stride=0, state=None, floor_seg=None, floor_c=None, stats=None):
    """Many rounds of Algorithm 1's Schedule loop over the same jobs at once (clusters: list of rk_cluster; the state
    tensors hold one state for all rounds, or one per round when state_stride is the number of jobs)."""
    n_rounds = len(clusters)
    arr = (rk_cluster * n_rounds)(*clusters)
    js = rk_job_state(_ptr(state), _ptr(cur_seg), _ptr(cur_c), _ptr(floor_seg), _ptr(floor_c))
    _check(ctx, load_library().rk_reschedule_rounds(ctx, _ptr(ref_thr), C.byref(table), C.byref(grid), C.c_uint32(n_rounds), arr,
                                                    _ptr(best_thr), _ptr(best_plan), _ptr(curve_thr), C.byref(js),
                                                    C.c_uint32(state_stride), _ptr(assign), _ptr(totals), _ptr(stats)))


def rk_schedule_round_nodes(ctx, jobs: Jobs, bounds, grid, env, nodes, cur_seg, cur_c, assign, placed, place_off, entries,
                            cap_entries, total, prev_off=None, prev_entries=None, n_prev_entries=0, state=None, floor_seg=None,
                            floor_c=None, stats=None):
    """A whole round of Algorithm 1 on nodes from the job descriptors (device tensors for the state and the results)."""
    js = rk_job_state(_ptr(state), _ptr(cur_seg), _ptr(cur_c), _ptr(floor_seg), _ptr(floor_c))
    _check(ctx, load_library().rk_schedule_round_nodes(ctx, C.byref(jobs.c), C.byref(bounds), C.byref(grid), C.byref(env),
                                                       C.byref(nodes), C.byref(js), _ptr(prev_off), _ptr(prev_entries),
                                                       C.c_uint64(n_prev_entries), _ptr(assign), _ptr(placed), _ptr(place_off),
                                                       _ptr(entries), C.c_uint64(cap_entries), _ptr(total), _ptr(stats)))


def rk_reschedule_nodes(ctx, ref_thr, table, grid, nodes: "rk_nodes", best_thr, best_plan, curve_thr, cur_seg, cur_c, assign,
                        place_off, entries, cap_entries, total, prev_off=None, prev_entries=None, n_prev_entries=0,
                        state=None, floor_seg=None, floor_c=None, stats=None):
    """Algorithm 1's Schedule loop with the node-by-node search of ScheduleJob, from the jobs' present state and
    placement (device tensors; entries as rk_place_entry records; stats: five words)."""
    js = rk_job_state(_ptr(state), _ptr(cur_seg), _ptr(cur_c), _ptr(floor_seg), _ptr(floor_c))
    _check(ctx, load_library().rk_reschedule_nodes(ctx, _ptr(ref_thr), C.byref(table), C.byref(grid), C.byref(nodes),
                                                   _ptr(best_thr), _ptr(best_plan), _ptr(curve_thr), C.byref(js),
                                                   _ptr(prev_off), _ptr(prev_entries), C.c_uint64(n_prev_entries),
                                                   _ptr(assign), _ptr(place_off), _ptr(entries), C.c_uint64(cap_entries),
                                                   _ptr(total), _ptr(stats)))


def rk_best_plan_placed(ctx, jobs: Jobs, table, grid, env, assign, place_off, entries, placed, total):
    """GetBestPlan(j, placement) for a placement that is there already (device tensors)."""
    _check(ctx, load_library().rk_best_plan_placed(ctx, C.byref(jobs.c), C.byref(table), C.byref(grid), C.byref(env),
                                                   _ptr(assign), _ptr(place_off), _ptr(entries), _ptr(placed), _ptr(total)))


def rk_probe_stream(ctx, buf, n_floats, mode, value=0.0, out=None):
    """Measurement helper: stream-read (modes 0, 3; strided: 2) or fill (modes 1, 4) the first n_floats floats of buf."""
    _check(ctx, load_library().rk_probe_stream(ctx, _ptr(buf), C.c_uint64(n_floats), C.c_int32(mode), C.c_float(value),
                                               _ptr(out)))


def rk_schedule_round(ctx, jobs: Jobs, bounds, grid, env, cluster, assign, total):
    _check(ctx, load_library().rk_schedule_round(ctx, C.byref(jobs.c), C.byref(bounds), C.byref(grid), C.byref(env),
                                                 C.byref(cluster), _ptr(assign), _ptr(total)))


def rk_schedule_rounds(ctx, jobs: Jobs, bounds, grid, env, round_off: np.ndarray, clusters, assign, totals):
    round_off = np.ascontiguousarray(round_off, dtype=np.uint32)
    n_rounds = len(round_off) - 1
    arr = (rk_cluster * n_rounds)(*clusters)
    _check(ctx, load_library().rk_schedule_rounds(ctx, C.byref(jobs.c), C.byref(bounds), C.byref(grid), C.byref(env),
                                                  C.c_uint32(n_rounds), round_off.ctypes.data_as(C.c_void_p), arr,
                                                  _ptr(assign), _ptr(totals)))


class Sla:
    """Service-level inputs on the device (int32 tensors hold the uint32 values)."""

    def __init__(self, guaranteed, tenant, quota_g, quota_c, req_g=None, req_c=None, req_m=None, base_thr=None,
                 device="cuda:0"):
        import torch
        dev_u32 = lambda a: None if a is None else torch.from_numpy(
            np.ascontiguousarray(a, dtype=np.uint32).view(np.int32)).to(device)
        self.guaranteed, self.tenant = dev_u32(guaranteed), dev_u32(tenant)
        self.req_g, self.req_c, self.req_m = dev_u32(req_g), dev_u32(req_c), dev_u32(req_m)
        self.quota_g, self.quota_c = dev_u32(quota_g), dev_u32(quota_c)
        if base_thr is None or hasattr(base_thr, "data_ptr"):
            self.base_thr = base_thr
        else:
            self.base_thr = torch.from_numpy(np.ascontiguousarray(base_thr, dtype=np.float32)).to(device)
        self.c = rk_sla()
        for name in ("guaranteed", "tenant", "req_g", "req_c", "req_m", "base_thr", "quota_g", "quota_c"):
            t = getattr(self, name)
            setattr(self.c, name, None if t is None or t.numel() == 0 else t.data_ptr())
        self.c.n_tenants = 0 if self.quota_g is None else int(self.quota_g.numel())


def rk_eval_points(ctx, jobs: Jobs, table, grid, env, pt_job, pt_plan, pt_c, pt_m, thr, feas=None):
    _check(ctx, load_library().rk_eval_points(ctx, C.byref(jobs.c), C.byref(table), C.byref(grid), C.byref(env),
                                              C.c_uint64(thr.numel()), _ptr(pt_job), _ptr(pt_plan), _ptr(pt_c),
                                              _ptr(pt_m), _ptr(thr), _ptr(feas)))


def rk_min_res(ctx, table, grid, job_begin, job_end, best_thr, sla: Sla, min_seg, min_c, min_m):
    _check(ctx, load_library().rk_min_res(ctx, C.byref(table), C.byref(grid), C.c_uint32(job_begin),
                                          C.c_uint32(job_end), _ptr(best_thr), C.byref(sla.c), _ptr(min_seg),
                                          _ptr(min_c), _ptr(min_m)))


def rk_allocate_sla(ctx, ref_thr, table, grid, cluster: rk_cluster, job_begin, job_end, best_thr, best_plan,
                    curve_thr, sla: Sla, min_seg, min_c, assign, total):
    _check(ctx, load_library().rk_allocate_sla(ctx, _ptr(ref_thr), C.byref(table), C.byref(grid), C.byref(cluster),
                                               C.c_uint32(job_begin), C.c_uint32(job_end), _ptr(best_thr),
                                               _ptr(best_plan), _ptr(curve_thr), C.byref(sla.c), _ptr(min_seg),
                                               _ptr(min_c), _ptr(assign), _ptr(total)))


def rk_schedule_round_sla(ctx, jobs: Jobs, bounds, grid, env, cluster, sla: Sla, assign, total):
    _check(ctx, load_library().rk_schedule_round_sla(ctx, C.byref(jobs.c), C.byref(bounds), C.byref(grid),
                                                     C.byref(env), C.byref(cluster), C.byref(sla.c), _ptr(assign),
                                                     _ptr(total)))


def pack_triples(d, t, p, v=0) -> np.ndarray:
    """(d, t, p, micro-batch shift v) -> the packed form of the plan table (t must be 1, 2, 4 or 8)."""
    d, t, p, v = (np.asarray(a, dtype=np.uint32) for a in (d, t, p, v))
    log2t = np.select([t == 1, t == 2, t == 4, t == 8], [0, 1, 2, 3], default=0).astype(np.uint32)
    return (d | (log2t << np.uint32(16)) | (p << np.uint32(18)) | (v << np.uint32(30))).astype(np.uint32)


class Samples:
    """Measured runs on the device, CSR over the models."""

    def __init__(self, sample_off, triple, option, cpus, thr, device="cuda:0"):
        import torch
        dev_u32 = lambda a: torch.from_numpy(np.ascontiguousarray(a, dtype=np.uint32).view(np.int32)).to(device)
        sample_off = np.ascontiguousarray(sample_off, dtype=np.uint32)
        self.sample_off, self.triple, self.option, self.cpus = (dev_u32(a) for a in (sample_off, triple, option, cpus))
        self.thr = torch.from_numpy(np.ascontiguousarray(thr, dtype=np.float32)).to(device)
        self.c = rk_samples(self.sample_off.data_ptr(), self.triple.data_ptr(), self.option.data_ptr(),
                            self.cpus.data_ptr(), self.thr.data_ptr(),
                            int(np.max(np.diff(sample_off.astype(np.int64)))) if len(sample_off) > 1 else 0)


class FitResult:
    def __init__(self, n_models, device="cuda:0"):
        import torch
        self.params = torch.zeros((len(FIT_FIELDS), max(n_models, 1)), dtype=torch.float32, device=device)
        self.theta = torch.zeros((max(n_models, 1), RK_FIT_PARAMS), dtype=torch.float64, device=device)
        self.rmsle_before = torch.zeros(max(n_models, 1), dtype=torch.float32, device=device)
        self.rmsle_after = torch.zeros(max(n_models, 1), dtype=torch.float32, device=device)
        self.iters = torch.zeros(max(n_models, 1), dtype=torch.int32, device=device)
        self.c = rk_fit_result(*[self.params[i].data_ptr() for i in range(len(FIT_FIELDS))], self.theta.data_ptr(),
                               self.rmsle_before.data_ptr(), self.rmsle_after.data_ptr(), self.iters.data_ptr())


def rk_fit_models(ctx, jobs: Jobs, env, samples: Samples, result: FitResult, max_iter=100, refit_threshold=0.0,
                  start_offsets=None):
    offs = np.zeros((0, RK_FIT_PARAMS)) if start_offsets is None else np.ascontiguousarray(start_offsets, dtype=np.float64)
    opt = rk_fit_options(int(max_iter), float(refit_threshold), int(offs.shape[0]),
                         offs.ctypes.data if offs.size else None)
    _check(ctx, load_library().rk_fit_models(ctx, C.byref(jobs.c), C.byref(env), C.byref(samples.c), C.byref(opt),
                                             C.byref(result.c)))


class SimResult:
    def __init__(self, n_jobs, n_ticks, device="cuda:0"):
        import torch
        nj, nt = max(n_jobs, 1), max(n_ticks, 1)
        self.finish = torch.zeros(nj, dtype=torch.float64, device=device)
        self.n_reconf = torch.zeros(nj, dtype=torch.int32, device=device)
        self.progress = torch.zeros(nj, dtype=torch.float64, device=device)
        self.held = torch.zeros(nj, dtype=torch.float64, device=device)
        self.gpus_in_use = torch.zeros(nt, dtype=torch.int32, device=device)
        self.totals = torch.zeros(nt, dtype=torch.float32, device=device)
        self.frozen = torch.zeros(nt, dtype=torch.int32, device=device)
        self.c = rk_sim_result(*[getattr(self, n).data_ptr() for n in
                                 ("finish", "n_reconf", "progress", "held", "gpus_in_use", "totals", "frozen")])


def rk_simulate(ctx, ref_thr, table, grid, cluster, best_thr, best_plan, curve_thr, arrival, work, delta, dt, n_ticks,
                gate, result: SimResult, policy=0, nodes=None):
    """arrival, work, delta: float64 device tensors.  policy 0: greedy round every tick, 1: Algorithm 1's loop,
    2: that loop over the nodes (nodes: rk_nodes)."""
    tr = rk_trace(arrival.data_ptr(), work.data_ptr(), delta.data_ptr())
    opt = rk_sim_options(float(dt), int(n_ticks), int(policy), float(gate),
                         None if nodes is None else C.cast(C.pointer(nodes), C.c_void_p))
    _check(ctx, load_library().rk_simulate(ctx, _ptr(ref_thr), C.byref(table), C.byref(grid), C.byref(cluster),
                                           _ptr(best_thr), _ptr(best_plan), _ptr(curve_thr), C.byref(tr), C.byref(opt),
                                           C.byref(result.c)))


def rk_schedule_rounds_shared(ctx, jobs: Jobs, bounds, grid, env, round_off: np.ndarray, round_jobs: np.ndarray, clusters,
                              assign, totals):
    round_off = np.ascontiguousarray(round_off, dtype=np.uint32)
    round_jobs = np.ascontiguousarray(round_jobs, dtype=np.uint32)
    n_rounds = len(round_off) - 1
    arr = (rk_cluster * n_rounds)(*clusters)
    _check(ctx, load_library().rk_schedule_rounds_shared(ctx, C.byref(jobs.c), C.byref(bounds), C.byref(grid),
                                                         C.byref(env), C.c_uint32(n_rounds),
                                                         round_off.ctypes.data_as(C.c_void_p),
                                                         round_jobs.ctypes.data_as(C.c_void_p), arr, _ptr(assign),
                                                         _ptr(totals)))


# ------------------------------------------------------------------ allocation helpers (no arithmetic)
def enumerate_to_table(ctx, jobs: Jobs, bounds: rk_plan_bounds, device="cuda:0") -> PlanTable:
    """Sizing call, allocation, fill call."""
    probe = rk_plan_table()
    rk_enumerate_plans(ctx, jobs, bounds, probe)
    table = PlanTable(jobs.n_jobs, int(probe.n_triples), int(probe.n_segs), device)
    rk_enumerate_plans(ctx, jobs, bounds, table.c)
    return table


class rk_nodes(C.Structure):
    _fields_ = [("n_nodes", C.c_uint32), ("gpus_per_node", C.c_uint32), ("cpus_per_node", C.c_uint32),
                ("mem_per_node_gb", C.c_float)]


class rk_place_result(C.Structure):
    _fields_ = [(n, C.c_uint32) for n in ("n_entries", "n_placed", "n_failed", "in_order")]


PLACE_DTYPE = np.dtype([("node", np.uint32), ("g", np.uint32), ("c", np.uint32), ("mem_gb", np.float32)])


def rk_place(ctx, nodes: rk_nodes, n_jobs, assign, place_off, entries, cap_entries, status, want_result=True):
    """Node-level placement of the records in assign; returns rk_place_result (after a wait) or None."""
    res = rk_place_result() if want_result else None
    _check(ctx, load_library().rk_place(ctx, C.byref(nodes), C.c_uint32(n_jobs), _ptr(assign), _ptr(place_off),
                                        _ptr(entries), C.c_uint64(cap_entries), _ptr(status),
                                        C.byref(res) if want_result else None))
    return res


def rk_place_plans(ctx, jobs: Jobs, table, grid, env, nodes: rk_nodes, best_thr, assign, min_seg, placed, place_off, entries,
                   cap_entries, status, total, want_result=True, prev_off=None, prev_entries=None):
    """Placement that feeds the plan; min_seg may be None; prev_off / prev_entries: an earlier placement whose
    unchanged jobs stay on their nodes.  Returns rk_place_result (after a wait) or None."""
    res = rk_place_result() if want_result else None
    _check(ctx, load_library().rk_place_plans(ctx, C.byref(jobs.c), C.byref(table), C.byref(grid), C.byref(env), C.byref(nodes),
                                              _ptr(best_thr), _ptr(assign), _ptr(min_seg), _ptr(prev_off), _ptr(prev_entries),
                                              _ptr(placed), _ptr(place_off),
                                              _ptr(entries), C.c_uint64(cap_entries), _ptr(status), _ptr(total),
                                              C.byref(res) if want_result else None))
    return res


def rk_schedule_round_placed(ctx, jobs: Jobs, bounds, grid, env, nodes: rk_nodes, sla, assign, placed, place_off, entries,
                             cap_entries, status, total, want_result=True):
    """A whole round on nodes; sla may be None."""
    res = rk_place_result() if want_result else None
    _check(ctx, load_library().rk_schedule_round_placed(ctx, C.byref(jobs.c), C.byref(bounds), C.byref(grid), C.byref(env),
                                                        C.byref(nodes), C.byref(sla.c) if sla is not None else None,
                                                        _ptr(assign), _ptr(placed), _ptr(place_off), _ptr(entries),
                                                        C.c_uint64(cap_entries), _ptr(status), _ptr(total),
                                                        C.byref(res) if want_result else None))
    return res


def new_place_entries(cap_entries, device="cuda:0"):
    import torch
    return torch.zeros(max(int(cap_entries), 1) * PLACE_DTYPE.itemsize, dtype=torch.uint8, device=device)


def place_entries_to_numpy(t, n_entries) -> np.ndarray:
    return t.cpu().numpy().view(PLACE_DTYPE)[:int(n_entries)]


def new_assign(n_jobs, device="cuda:0"):
    import torch
    return torch.zeros(n_jobs * ASSIGN_DTYPE.itemsize, dtype=torch.uint8, device=device)


def assign_to_numpy(t) -> np.ndarray:
    return t.cpu().numpy().view(ASSIGN_DTYPE)


def u32(t) -> np.ndarray:
    """Host copy of an int32 device tensor reinterpreted as uint32."""
    return t.cpu().numpy().view(np.uint32)


# ------------------------------------------------------------------ operators of a training step
RK_F32, RK_BF16, RK_F16 = 0, 1, 2
RK_NORM_KINDS = {"none": 0, "rms": 1, "layer": 2}
RK_NORM_MAX_WIDTH, RK_MAX_EXPERTS, RK_MAX_TOP_K, RK_MAX_TEACHER_LOGITS = 32768, 1024, 32, 1024
RK_RECUR_MAX_WIDTH, RK_HEAD_MAX_WIDTH = 1048576, 65536


class rk_matrix(C.Structure):
    _fields_ = [("data", C.c_void_p), ("stride", C.c_uint64), ("type", C.c_uint32)]


class rk_norm_block(C.Structure):
    _fields_ = [("post_kind", C.c_uint32), ("pre_kind", C.c_uint32), ("post_eps", C.c_float), ("pre_eps", C.c_float),
                ("res_scale", C.c_float), ("param_type", C.c_uint32)] + \
               [(n, C.c_void_p) for n in ("post_weight", "post_bias", "pre_weight", "pre_bias", "gate")] + \
               [("gate_rows", C.c_uint64), ("gate_stride", C.c_uint64)]


class rk_norm_grads(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("post_weight", "post_bias", "pre_weight", "pre_bias", "gate")] + \
               [("gate_stride", C.c_uint64), ("gates", C.c_uint64)]


class rk_router(C.Structure):
    _fields_ = [("n_experts", C.c_uint32), ("top_k", C.c_uint32), ("renormalise", C.c_uint32), ("group_tokens", C.c_uint64)]


class rk_distill(C.Structure):
    _fields_ = [("temperature", C.c_float), ("kd_weight", C.c_float), ("ce_weight", C.c_float)]


class rk_teacher(C.Structure):
    _fields_ = [("logits", C.c_void_p), ("index", C.c_void_p), ("top_k", C.c_uint32), ("label", C.c_void_p),
                ("row_weight", C.c_void_p)]


class rk_recur(C.Structure):
    _fields_ = [("coupled", C.c_uint32), ("param_type", C.c_uint32), ("bias", C.c_void_p), ("offsets", C.c_void_p),
                ("n_seqs", C.c_uint32), ("seq_rows", C.c_uint64)]


class rk_dropout(C.Structure):
    _fields_ = [("p", C.c_float), ("rng", C.c_void_p)]


class rk_head(C.Structure):
    _fields_ = [("logit_scale", C.c_float), ("z_weight", C.c_float)]


def _refuse(what):
    raise RkError(RK_ERR_INVALID_ARG, what)


_TYPES = {}                 # element types by torch dtype, and the dtypes by name; filled with the first tensor


def _types():
    if not _TYPES:
        import torch
        _TYPES.update({torch.float32: RK_F32, torch.bfloat16: RK_BF16, torch.float16: RK_F16, "float32": torch.float32,
                       "int32": torch.int32, "int64": torch.int64, "uint8": torch.uint8, "bool": torch.bool})
    return _TYPES


def _type_of(t):
    kind = _types().get(t.dtype)
    return _refuse(f"{t.dtype} is none of float32, bfloat16, float16") if kind is None else kind


def _matrix(t, name, shape=None):
    """A [rows, width] tensor, its rows of consecutive elements, as an rk_matrix; the tensor has to outlive the call."""
    if t is None:
        return None
    size, strides = t.shape, t.stride()
    if len(size) != 2 or (strides[1] != 1 and size[1] > 1):
        _refuse(f"{name} is no matrix of consecutive row elements")
    if shape is not None and size != shape:
        _refuse(f"{name} is {tuple(size)}, not {tuple(shape)}")
    stride, width = strides[0], size[1]
    if stride < width:
        if size[0] > 1:
            _refuse(f"the rows of {name} overlap")
        stride = width
    return rk_matrix(t.data_ptr(), stride, _TYPES.get(t.dtype) if t.dtype in _TYPES else _type_of(t))


_F32, _I32 = ("float32",), ("int32",)


def _plain(t, name, shape, dtypes):
    """The address of a contiguous tensor of that shape and of one of these types, or None."""
    if t is None:
        return None
    known = _TYPES or _types()
    if t.shape != shape or not t.is_contiguous() or (t.dtype != known[dtypes[0]] and t.dtype != known[dtypes[-1]]):
        _refuse(f"{name} is no contiguous {' or '.join(dtypes)} tensor of shape {tuple(shape)}")
    return t.data_ptr()


def _same_device(first, *others):
    device = first.get_device()
    if device < 0:
        _refuse("the tensors are not on a GPU")
    for t in others:
        if t is not None and t.get_device() != device:
            _refuse("the tensors are not on one GPU")


def _ref(s):
    return None if s is None else C.byref(s)


_OPERATORS = {
    "rk_norm_forward": "cbqu" + "m" * 4 + "p", "rk_norm_backward": "cbqu" + "mmp" + "m" * 4 + "g",
    "rk_route_forward": "crqm" + "p" * 8, "rk_route_backward": "crqm" + "p" * 6 + "m",
    "rk_distill_loss": "cdqumt" + "ppp", "rk_distill_backward": "cdqumt" + "ppm", "rk_distill_loss_backward": "cdqumt" + "ppppm",
    "rk_recur_forward": "csqu" + "m" * 5, "rk_recur_backward": "csqu" + "m" * 9 + "p",
    "rk_dropout_forward": "coqu" + "mmm", "rk_dropout_backward": "coqu" + "mm",
    "rk_head_loss": "chquu" + "mmpp" + "ppp", "rk_head_backward": "chquu" + "mmpp" + "ppmm", "rk_head_loss_backward": "chquu" + "mmpp" + "ppppmm",
}


_functions = {}


def _operator(name):
    """The library's function, its argument types known (which spares wrapping every number of every call): an object of the binding's
    own, so that whoever calls the library's attribute of that name finds it as it was."""
    f = _functions.get(name)
    if f is None:
        kinds = {"c": C.c_void_p, "q": C.c_uint64, "u": C.c_uint32, "p": C.c_void_p, "b": C.POINTER(rk_norm_block), "g": C.POINTER(rk_norm_grads),
                 "m": C.POINTER(rk_matrix), "r": C.POINTER(rk_router), "d": C.POINTER(rk_distill), "t": C.POINTER(rk_teacher),
                 "s": C.POINTER(rk_recur), "o": C.POINTER(rk_dropout), "h": C.POINTER(rk_head)}
        f = load_library()[name]
        f.restype, f.argtypes = C.c_int32, [kinds[k] for k in _OPERATORS[name]]
        _functions[name] = f
    return f


class NormBlock:
    """The norms around a block with its gate and residual scale (rk_norm_block).  post and pre: "none", "rms" or "layer";
    vectors are [width] tensors of one type, gate is [1, width] for all rows (gate_rows 0) or [gates, width], one for every
    gate_rows rows."""

    def __init__(self, post="rms", pre="rms", post_weight=None, post_bias=None, pre_weight=None, pre_bias=None, gate=None,
                 gate_rows=0, res_scale=1.0, post_eps=1e-6, pre_eps=1e-6):
        if post not in RK_NORM_KINDS or pre not in RK_NORM_KINDS:
            _refuse(f"norms are one of {tuple(RK_NORM_KINDS)}")
        self.vectors = {"post_weight": post_weight, "post_bias": post_bias, "pre_weight": pre_weight, "pre_bias": pre_bias}
        self.gate = gate
        self.given = [t for t in (*self.vectors.values(), gate) if t is not None]
        self.width = int(self.given[0].shape[-1]) if self.given else None
        if len({(t.dtype, t.device) for t in self.given}) > 1:
            _refuse("weights, biases and gate are of one type, on one GPU")
        for name, t in self.vectors.items():
            if t is not None and (tuple(t.shape) != (self.width,) or not t.is_contiguous()):
                _refuse(f"{name} is no contiguous vector of {self.width} elements")
        c_gate = _matrix(gate, "gate")
        if gate is not None and (gate.shape[1] != self.width or (gate_rows == 0 and gate.shape[0] != 1)):
            _refuse("gate is [1, width], or [gates, width] with gate_rows")
        self.gate_capacity = gate.shape[0] * int(gate_rows) if gate is not None and gate_rows else None
        self.c = rk_norm_block(RK_NORM_KINDS[post], RK_NORM_KINDS[pre], post_eps, pre_eps, res_scale,
                               _type_of(self.given[0]) if self.given else RK_F32,
                               *[None if t is None else t.data_ptr() for t in self.vectors.values()],
                               None if gate is None else gate.data_ptr(), int(gate_rows),
                               c_gate.stride if c_gate is not None else 0)

    def _rows(self, t, name):
        """The shape of the rows that a call is about."""
        size = t.shape
        if len(size) != 2 or (self.width is not None and size[1] != self.width):
            _refuse(f"{name} has no rows of {self.width} elements")
        if self.gate_capacity is not None and self.gate_capacity < size[0]:
            _refuse(f"{self.gate.shape[0]} gates of {self.c.gate_rows} rows for {size[0]} rows")
        return size


class NormGrads:
    """Room for the gradients of a block's vectors, float32; `tensors` by name (all that the block has, or those named).  Of gates that
    no row of a call uses, the gradients are zero."""

    def __init__(self, block: NormBlock, names=None):
        import torch
        self.block = block
        have = dict(block.vectors, gate=block.gate)
        self.tensors = {n: torch.empty(t.shape, dtype=torch.float32, device=t.device) for n, t in have.items()
                        if t is not None and (names is None or n in names)}
        ptr = {n: t.data_ptr() for n, t in self.tensors.items()}
        self.c = rk_norm_grads(*[ptr.get(n) for n in ("post_weight", "post_bias", "pre_weight", "pre_bias", "gate")],
                               block.width or 0, block.gate.shape[0] if block.gate is not None and block.c.gate_rows else 0)


def rk_norm_forward(ctx, block: NormBlock, x, y, x_out, u, stats):
    """y, x_out and u may be None as the header says; stats is [rows, 4] float32."""
    size = block._rows(x, "x")
    _same_device(x, y, x_out, u, stats, *block.given[:1])
    _check(ctx, _operator("rk_norm_forward")(
        ctx, C.byref(block.c), size[0], size[1], C.byref(_matrix(x, "x")), _ref(_matrix(y, "y", size)), _ref(_matrix(x_out, "x_out", size)),
        _ref(_matrix(u, "u", size)), _plain(stats, "stats", (size[0], 4), _F32)))


def rk_norm_backward(ctx, block: NormBlock, x_out, y, stats, dx_out, du, dx, dy, grads: NormGrads = None):
    size = block._rows(x_out, "x_out")
    _same_device(x_out, y, stats, dx_out, du, dx, dy, *block.given[:1])
    if grads is not None and grads.block is not block:
        _refuse("the gradients are another block's")
    _check(ctx, _operator("rk_norm_backward")(
        ctx, C.byref(block.c), size[0], size[1], C.byref(_matrix(x_out, "x_out")), _ref(_matrix(y, "y", size)),
        _plain(stats, "stats", (size[0], 4), _F32), _ref(_matrix(dx_out, "dx_out", size)), _ref(_matrix(du, "du", size)),
        C.byref(_matrix(dx, "dx", size)), _ref(_matrix(dy, "dy", size)), None if grads is None else C.byref(grads.c)))


def make_router(n_experts, top_k, renormalise=True, group_tokens=0) -> rk_router:
    return rk_router(int(n_experts), int(top_k), int(bool(renormalise)), int(group_tokens))


def _router_sizes(router, logits):
    size = logits.shape
    if len(size) != 2 or size[1] != router.n_experts:
        _refuse(f"logits are not [tokens, {router.n_experts}]")
    n, per = size[0], router.group_tokens
    return n, router.top_k, size[1], (n + per - 1) // per if per else 1


def rk_route_forward(ctx, router: rk_router, logits, mask, expert, weight, lse, counts, prob_sum, tokens, loss):
    """mask uint8 [tokens] or None; expert int32 and weight float32 [tokens, top_k]; lse [tokens]; counts int32 and prob_sum
    [groups, experts]; tokens int32 [groups]; loss [2]: balance, z."""
    n, k, e, groups = _router_sizes(router, logits)
    _same_device(logits, mask, expert, weight, lse, counts, prob_sum, tokens, loss)
    _check(ctx, _operator("rk_route_forward")(
        ctx, C.byref(router), n, C.byref(_matrix(logits, "logits")), _plain(mask, "mask", (n,), ("uint8", "bool")),
        _plain(expert, "expert", (n, k), _I32), _plain(weight, "weight", (n, k), _F32), _plain(lse, "lse", (n,), _F32),
        _plain(counts, "counts", (groups, e), _I32), _plain(prob_sum, "prob_sum", (groups, e), _F32),
        _plain(tokens, "tokens", (groups,), _I32), _plain(loss, "loss", (2,), _F32)))


def rk_route_backward(ctx, router: rk_router, logits, expert, lse, counts, tokens, d_loss, d_weight, d_logits):
    n, k, e, groups = _router_sizes(router, logits)
    _same_device(logits, expert, lse, counts, tokens, d_loss, d_weight, d_logits)
    _check(ctx, _operator("rk_route_backward")(
        ctx, C.byref(router), n, C.byref(_matrix(logits, "logits")), _plain(expert, "expert", (n, k), _I32),
        _plain(lse, "lse", (n,), _F32), _plain(counts, "counts", (groups, e), _I32), _plain(tokens, "tokens", (groups,), _I32),
        _plain(d_loss, "d_loss", (2,), _F32), _plain(d_weight, "d_weight", (n, k), _F32),
        _ref(_matrix(d_logits, "d_logits", (n, e)))))


def make_distill(temperature=1.0, kd_weight=1.0, ce_weight=0.0) -> rk_distill:
    return rk_distill(float(temperature), float(kd_weight), float(ce_weight))


def _distill_call(ctx, name, distill, student, teacher_logits, teacher_index, label, row_weight, *rest):
    size = student.shape
    if len(size) != 2:
        _refuse("student is not [rows, vocab]")
    rows = size[0]
    if (teacher_logits is None) != (teacher_index is None):
        _refuse("the teacher's logits and their indices go together")
    logits, k = None, 0
    if teacher_logits is not None:
        k = teacher_logits.shape[-1]
        logits = _matrix(teacher_logits, "teacher_logits", (rows, k))
    teacher = rk_teacher(None if logits is None else C.addressof(logits), _plain(teacher_index, "teacher_index", (rows, k), _I32), k,
                         _plain(label, "label", (rows,), _I32), _plain(row_weight, "row_weight", (rows,), _F32))
    _check(ctx, _operator(name)(ctx, C.byref(distill), rows, size[1], C.byref(_matrix(student, "student")), C.byref(teacher), *rest))


def rk_distill_loss(ctx, distill: rk_distill, student, teacher_logits, teacher_index, label, row_weight, loss, lse, total):
    """teacher_logits [rows, k] with teacher_index int32 (None if kd_weight is 0); label int32 [rows] (None if ce_weight is 0);
    row_weight float32 [rows] or None; loss [rows], lse [rows, 2], total [1], all float32."""
    _same_device(student, teacher_logits, teacher_index, label, row_weight, loss, lse, total)
    rows = student.shape[0]
    _distill_call(ctx, "rk_distill_loss", distill, student, teacher_logits, teacher_index, label, row_weight,
                  _plain(loss, "loss", (rows,), _F32), _plain(lse, "lse", (rows, 2), _F32), _plain(total, "total", (1,), _F32))


def rk_distill_backward(ctx, distill: rk_distill, student, teacher_logits, teacher_index, label, row_weight, lse, d_total, d_student):
    _same_device(student, teacher_logits, teacher_index, label, row_weight, lse, d_total, d_student)
    _distill_call(ctx, "rk_distill_backward", distill, student, teacher_logits, teacher_index, label, row_weight,
                  _plain(lse, "lse", (student.shape[0], 2), _F32), _plain(d_total, "d_total", (1,), _F32),
                  _ref(_matrix(d_student, "d_student", student.shape)))


def rk_distill_loss_backward(ctx, distill: rk_distill, student, teacher_logits, teacher_index, label, row_weight, d_total, loss, lse,
                             total, d_student):
    _same_device(student, teacher_logits, teacher_index, label, row_weight, d_total, loss, lse, total, d_student)
    rows = student.shape[0]
    _distill_call(ctx, "rk_distill_loss_backward", distill, student, teacher_logits, teacher_index, label, row_weight,
                  _plain(d_total, "d_total", (1,), _F32), _plain(loss, "loss", (rows,), _F32),
                  _plain(lse, "lse", (rows, 2), _F32), _plain(total, "total", (1,), _F32),
                  _ref(_matrix(d_student, "d_student", student.shape)))


class Recur:
    """A gated linear recurrence (rk_recur).  bias [width] or None; offsets int32 [sequences + 1] on the GPU, or None: every seq_rows rows
    are a sequence (0: all of them are one)."""

    def __init__(self, coupled=True, bias=None, offsets=None, seq_rows=0):
        if bias is not None and (bias.dim() != 1 or not bias.is_contiguous()):
            _refuse("bias is no contiguous vector")
        if offsets is not None and (offsets.dim() != 1 or len(offsets) < 1 or seq_rows):
            _refuse("offsets are a vector of the sequences' number and one, or there are seq_rows")
        if not 0 <= int(seq_rows) < 1 << 64:
            _refuse(f"sequences of {seq_rows} rows")
        self.bias, self.offsets = bias, offsets
        self.n_seqs = None if offsets is None else len(offsets) - 1
        at = None if offsets is None else _plain(offsets, "offsets", offsets.shape, _I32)
        self.c = rk_recur(int(bool(coupled)), RK_F32 if bias is None else _type_of(bias), None if bias is None else bias.data_ptr(), at,
                          self.n_seqs or 0, int(seq_rows))

    def _sizes(self, z):
        """The shapes of the rows and of the states that a call is about."""
        size = z.shape
        if len(size) != 2 or (self.bias is not None and len(self.bias) != size[1]):
            _refuse("z has no rows of the bias's width")
        per = self.c.seq_rows
        seqs = self.n_seqs if self.offsets is not None else (size[0] + per - 1) // per if per else 1
        return size, size[:0] + (seqs, size[1])


def rk_recur_forward(ctx, recur: Recur, x, z, state_in, h, state_out):
    """x, z, h [rows, width]; state_in and state_out float32 [sequences, width] or None."""
    size, states = recur._sizes(z)
    _same_device(z, x, state_in, h, state_out, recur.bias, recur.offsets)
    _check(ctx, _operator("rk_recur_forward")(
        ctx, C.byref(recur.c), size[0], size[1], _ref(_matrix(x, "x", size)), C.byref(_matrix(z, "z")), _ref(_matrix(state_in, "state_in", states)),
        _ref(_matrix(h, "h", size)), _ref(_matrix(state_out, "state_out", states))))


def rk_recur_backward(ctx, recur: Recur, x, z, h, state_in, dh, d_state_out, dx, dz, d_state_in, d_bias):
    """d_bias float32 [width] or None; x may be None if the recurrence is not coupled."""
    size, states = recur._sizes(z)
    _same_device(z, x, h, state_in, dh, d_state_out, dx, dz, d_state_in, d_bias, recur.bias, recur.offsets)
    _check(ctx, _operator("rk_recur_backward")(
        ctx, C.byref(recur.c), size[0], size[1], _ref(_matrix(x, "x", size)), C.byref(_matrix(z, "z")), _ref(_matrix(h, "h", size)),
        _ref(_matrix(state_in, "state_in", states)), _ref(_matrix(dh, "dh", size)), _ref(_matrix(d_state_out, "d_state_out", states)),
        _ref(_matrix(dx, "dx", size)), _ref(_matrix(dz, "dz", size)), _ref(_matrix(d_state_in, "d_state_in", states)),
        _plain(d_bias, "d_bias", size[1:], _F32)))


class Dropout:
    """Dropout of a share p (rk_dropout) under rng: int64 [2] on the GPU, the seed and the offset, which the kernels read when they run."""

    def __init__(self, p, rng):
        self.rng = rng
        self.c = rk_dropout(float(p), _plain(rng, "rng", (2,), ("int64",)))


def rk_dropout_forward(ctx, dropout: Dropout, x, residual, out):
    """out [rows, width] has the residual's type (None: that of x): x's or float32."""
    size = x.shape
    _same_device(x, residual, out, dropout.rng)
    _check(ctx, _operator("rk_dropout_forward")(
        ctx, C.byref(dropout.c), size[0], size[-1], C.byref(_matrix(x, "x")), _ref(_matrix(residual, "residual", size)), _ref(_matrix(out, "out", size))))


def rk_dropout_backward(ctx, dropout: Dropout, d_out, dx):
    size = d_out.shape
    _same_device(d_out, dx, dropout.rng)
    _check(ctx, _operator("rk_dropout_backward")(
        ctx, C.byref(dropout.c), size[0], size[-1], C.byref(_matrix(d_out, "d_out")), _ref(_matrix(dx, "dx", size))))


def make_head(logit_scale=1.0, z_weight=0.0) -> rk_head:
    return rk_head(float(logit_scale), float(z_weight))


def _head_call(ctx, name, head, x, weight, label, row_weight, *rest):
    size = x.shape
    if len(size) != 2 or weight.dim() != 2 or weight.shape[1] != size[1]:
        _refuse("x and weight are not [rows, width] and [vocab, width]")
    _check(ctx, _operator(name)(
        ctx, C.byref(head), size[0], size[1], weight.shape[0], C.byref(_matrix(x, "x")), C.byref(_matrix(weight, "weight")),
        _plain(label, "label", size[:1], _I32), _plain(row_weight, "row_weight", size[:1], _F32), *rest))


def rk_head_loss(ctx, head: rk_head, x, weight, label, row_weight, loss, lse, total):
    """x [rows, width], weight [vocab, width]; label int32 [rows], row_weight float32 [rows] or None; loss [rows], lse [rows], total [1], all
    float32."""
    _same_device(x, weight, label, row_weight, loss, lse, total)
    rows = x.shape[:1]
    _head_call(ctx, "rk_head_loss", head, x, weight, label, row_weight, _plain(loss, "loss", rows, _F32), _plain(lse, "lse", rows, _F32),
               _plain(total, "total", (1,), _F32))


def rk_head_backward(ctx, head: rk_head, x, weight, label, row_weight, lse, d_total, dx, d_weight):
    """dx or d_weight may be None."""
    _same_device(x, weight, label, row_weight, lse, d_total, dx, d_weight)
    _head_call(ctx, "rk_head_backward", head, x, weight, label, row_weight, _plain(lse, "lse", x.shape[:1], _F32),
               _plain(d_total, "d_total", (1,), _F32), _ref(_matrix(dx, "dx", x.shape)), _ref(_matrix(d_weight, "d_weight", weight.shape)))


def rk_head_loss_backward(ctx, head: rk_head, x, weight, label, row_weight, d_total, loss, lse, total, dx, d_weight):
    _same_device(x, weight, label, row_weight, d_total, loss, lse, total, dx, d_weight)
    rows = x.shape[:1]
    _head_call(ctx, "rk_head_loss_backward", head, x, weight, label, row_weight, _plain(d_total, "d_total", (1,), _F32),
               _plain(loss, "loss", rows, _F32), _plain(lse, "lse", rows, _F32), _plain(total, "total", (1,), _F32),
               _ref(_matrix(dx, "dx", x.shape)), _ref(_matrix(d_weight, "d_weight", weight.shape)))
