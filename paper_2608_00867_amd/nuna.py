"""Thin ctypes binding over ``libnuna.so`` (C ABI in ``include/nuna.h``).

Argument marshalling only: every collective runs in the library's gfx950
kernels.  Torch tensors supply device memory and the stream; nothing here
computes on the host, and there is no fallback: if the library is missing,
loading it raises.

Two layers:

* ``raw`` functions take integer device pointers and return the status code
  (used to exercise the C ABI directly, including its argument checks);
* tensor functions take lists of CUDA tensors (one per simulated rank),
  enqueue on the current torch stream and raise ``NunaError`` on failure.
"""
import ctypes
import functools
import os

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libnuna.so")

OK, ERR_INVALID_ARG, ERR_UNSUPPORTED, ERR_MISALIGNED, ERR_OVERLAP, ERR_HIP, ERR_NO_MEMORY = range(7)
STATUS_NAMES = {0: "NUNA_OK", 1: "NUNA_ERR_INVALID_ARG", 2: "NUNA_ERR_UNSUPPORTED", 3: "NUNA_ERR_MISALIGNED",
                4: "NUNA_ERR_OVERLAP", 5: "NUNA_ERR_HIP", 6: "NUNA_ERR_NO_MEMORY"}
F32, BF16 = 0, 1
SCALE_F32, SCALE_E8M0 = 0, 1
SCORE_SOFTMAX, SCORE_SIGMOID = 0, 1
F8_BLOCK = 128
MAX_EXPERTS = 1024
FEW_TOKENS = 64
LINEAR, XCD = 0, 1
ALGO_AUTO, ALGO_ONE_SHOT, ALGO_TWO_SHOT, ALGO_ONE_SHOT_SPLIT, ALGO_TWO_SHOT_TWO_KERNELS = 0, 1, 2, 3, 4

PLACEMENTS = {"linear": LINEAR, "xcd": XCD, LINEAR: LINEAR, XCD: XCD}
ALGOS = {"auto": ALGO_AUTO, "one_shot": ALGO_ONE_SHOT, "two_shot": ALGO_TWO_SHOT, "one_shot_split": ALGO_ONE_SHOT_SPLIT,
         "two_shot_two_kernels": ALGO_TWO_SHOT_TWO_KERNELS,
         ALGO_AUTO: ALGO_AUTO, ALGO_ONE_SHOT: ALGO_ONE_SHOT, ALGO_TWO_SHOT: ALGO_TWO_SHOT,
         ALGO_ONE_SHOT_SPLIT: ALGO_ONE_SHOT_SPLIT, ALGO_TWO_SHOT_TWO_KERNELS: ALGO_TWO_SHOT_TWO_KERNELS}

_vp = ctypes.c_void_p
_vpp = ctypes.POINTER(ctypes.c_void_p)
_i64p = ctypes.POINTER(ctypes.c_int64)
_i32p = ctypes.POINTER(ctypes.c_int32)

NAP_MAX_DOMAINS = 16
NAP_MAX_STACKS = 16


class DeviceInfo(ctypes.Structure):
    """Mirror of nuna_device_info_t."""
    _fields_ = [("device", ctypes.c_int32), ("cu_count", ctypes.c_int32), ("xcd_count", ctypes.c_int32),
                ("map_verified", ctypes.c_int32)]


class LaunchInfo(ctypes.Structure):
    """Mirror of nuna_launch_info_t."""
    _fields_ = [("kernels", ctypes.c_char * 96), ("launches", ctypes.c_int32), ("map", ctypes.c_int32),
                ("group_size", ctypes.c_int64), ("grid", ctypes.c_int64), ("threads", ctypes.c_int32),
                ("vectors_per_thread", ctypes.c_int32)]


MAP_NAMES = {0: "linear", 1: "xcd_groups", 2: "xcd_pages", 3: "xcd_lists", 4: "xcd_shards"}


class NapTopology(ctypes.Structure):
    """Mirror of nuna_nap_topology_t."""
    _fields_ = [("num_domains", ctypes.c_int32), ("cus_per_domain", ctypes.c_int32),
                ("num_stacks", ctypes.c_int32), ("reserved", ctypes.c_int32),
                ("cu_budget", ctypes.c_int64), ("stack_budget", ctypes.c_int64),
                ("stack_pref", (ctypes.c_int32 * NAP_MAX_STACKS) * NAP_MAX_DOMAINS)]

# Every function the header declares, with its ctypes signature.
SIGNATURES = {
    "nuna_init": ([], ctypes.c_int),
    "nuna_get_device_info": ([ctypes.POINTER(DeviceInfo)], ctypes.c_int),
    "nuna_last_launch": ([ctypes.POINTER(LaunchInfo)], ctypes.c_int),
    "nuna_check_dispatch_map": ([_i32p, ctypes.c_int64, ctypes.c_int32], ctypes.c_int),
    "nuna_last_error_string": ([], ctypes.c_char_p),
    "nuna_version": ([], ctypes.c_int),
    "nuna_set_max_workgroups": ([ctypes.c_int], ctypes.c_int),
    "nuna_set_tunable": ([ctypes.c_char_p, ctypes.c_int64], ctypes.c_int),
    "nuna_get_tunable": ([ctypes.c_char_p, _i64p], ctypes.c_int),
    "nuna_allreduce": ([_vpp, _vpp, ctypes.c_int, ctypes.c_size_t, ctypes.c_int, ctypes.c_int, ctypes.c_int, _vp],
                       ctypes.c_int),
    "nuna_reduce_scatter": ([_vpp, _vpp, ctypes.c_int, ctypes.c_size_t, ctypes.c_int, ctypes.c_int, _vp],
                            ctypes.c_int),
    "nuna_all_gather": ([_vpp, _vpp, ctypes.c_int, ctypes.c_size_t, ctypes.c_int, ctypes.c_int, _vp], ctypes.c_int),
    "nuna_a2a_layout_create": ([ctypes.c_int, ctypes.c_int, ctypes.c_int, ctypes.c_int, _vp,
                                ctypes.POINTER(_vp)], ctypes.c_int),
    "nuna_a2a_layout_upload": ([_vp], ctypes.c_int),
    "nuna_a2a_layout_recv_rows": ([_vp, _i64p], ctypes.c_int),
    "nuna_a2a_layout_recv_map": ([_vp, ctypes.c_int, _i32p, _i32p], ctypes.c_int),
    "nuna_a2a_layout_destroy": ([_vp], None),
    "nuna_all_to_all": ([_vpp, _vpp, _vp, ctypes.c_size_t, ctypes.c_size_t, ctypes.c_int, ctypes.c_int, _vp],
                        ctypes.c_int),
    "nuna_all_to_all_routed": ([_vpp, _vpp, _vp, ctypes.c_int, ctypes.c_int, ctypes.c_int, ctypes.c_int,
                                ctypes.c_size_t, ctypes.c_size_t, ctypes.c_int, ctypes.c_int, _vp, _vp], ctypes.c_int),
    "nuna_all_to_all_combine": ([_vpp, _vpp, _vp, _vp, ctypes.c_size_t, ctypes.c_size_t, ctypes.c_int,
                                 ctypes.c_int, _vp], ctypes.c_int),
    "nuna_moe_sort_workspace": ([ctypes.c_int64, ctypes.c_int, ctypes.c_int, ctypes.POINTER(ctypes.c_size_t)],
                                ctypes.c_int),
    "nuna_moe_sort": ([_vp, ctypes.c_int64, ctypes.c_int, ctypes.c_int, ctypes.c_int, _vp, _vp, _vp, _vp,
                       ctypes.c_size_t, _vp], ctypes.c_int),
    "nuna_moe_gather": ([_vp, ctypes.c_int64, _vp, ctypes.c_int64, ctypes.c_int, ctypes.c_size_t, _vp, ctypes.c_size_t,
                         ctypes.c_int, _vp], ctypes.c_int),
    "nuna_moe_gather_f8": ([_vp, ctypes.c_int64, _vp, ctypes.c_int64, ctypes.c_int, ctypes.c_size_t, _vp, _vp,
                            ctypes.c_size_t, ctypes.c_int, ctypes.c_int, _vp], ctypes.c_int),
    "nuna_moe_scatter": ([_vp, _vp, _vp, ctypes.c_int64, ctypes.c_int, ctypes.c_size_t, ctypes.c_size_t, _vp,
                          ctypes.c_int, _vp], ctypes.c_int),
    "nuna_moe_scatter_grad": ([_vp, _vp, _vp, _vp, ctypes.c_int64, ctypes.c_int, ctypes.c_size_t, ctypes.c_size_t, _vp,
                               _vp, ctypes.c_int, _vp], ctypes.c_int),
    "nuna_f8_quantize": ([_vp, ctypes.c_int64, ctypes.c_size_t, ctypes.c_size_t, ctypes.c_int, _vp, _vp, ctypes.c_int,
                          _vp], ctypes.c_int),
    "nuna_f8_quantize_blocks": ([_vp, ctypes.c_int, ctypes.c_size_t, ctypes.c_size_t, ctypes.c_int, _vp, _vp,
                                 ctypes.c_int, _vp], ctypes.c_int),
    "nuna_f8_quantize_cols": ([_vp, ctypes.c_int64, ctypes.c_size_t, _vp, ctypes.c_int, _vp, ctypes.c_int,
                               ctypes.c_size_t, ctypes.c_size_t, ctypes.c_int, _vp, _vp, ctypes.c_int, _vp],
                              ctypes.c_int),
    "nuna_f8_matmul": ([_vp, _vp, _vp, _vp, _vp, ctypes.c_int, ctypes.c_size_t, ctypes.c_size_t, ctypes.c_size_t, _vp,
                        ctypes.c_int, ctypes.c_int, _vp], ctypes.c_int),
    "nuna_f8_wgrad": ([_vp, _vp, _vp, _vp, _vp, ctypes.c_int, ctypes.c_size_t, ctypes.c_size_t, ctypes.c_size_t, _vp,
                       ctypes.c_int, ctypes.c_int, _vp], ctypes.c_int),
    "nuna_rms_norm": ([_vp, ctypes.c_int64, _vp, ctypes.c_int64, _vp, ctypes.c_int, ctypes.c_float, ctypes.c_size_t,
                       ctypes.c_size_t, _vp, ctypes.c_int64, _vp, _vp, _vp, ctypes.c_int, _vp, ctypes.c_int, _vp],
                      ctypes.c_int),
    "nuna_rms_norm_grad_workspace": ([ctypes.c_size_t, ctypes.c_size_t, ctypes.POINTER(ctypes.c_size_t)], ctypes.c_int),
    "nuna_rms_norm_grad": ([_vp, _vp, ctypes.c_int64, _vp, ctypes.c_int, _vp, _vp, ctypes.c_size_t, ctypes.c_size_t, _vp,
                            _vp, _vp, ctypes.c_size_t, ctypes.c_int, _vp], ctypes.c_int),
    "nuna_route_topk": ([_vp, ctypes.c_int64, _vp, ctypes.c_int64, ctypes.c_int, ctypes.c_int, ctypes.c_int, ctypes.c_int,
                         ctypes.c_float, _vp, _vp, ctypes.c_int, _vp], ctypes.c_int),
    "nuna_route_topk_grad": ([_vp, _vp, ctypes.c_int64, _vp, ctypes.c_int64, ctypes.c_int, ctypes.c_int, ctypes.c_int,
                              ctypes.c_int, ctypes.c_float, _vp, ctypes.c_int, _vp], ctypes.c_int),
    "nuna_swiglu": ([_vp, _vp, ctypes.c_int, ctypes.c_size_t, ctypes.c_size_t, _vp, _vp, _vp, ctypes.c_int, ctypes.c_int,
                     _vp], ctypes.c_int),
    "nuna_swiglu_grad": ([_vp, _vp, _vp, ctypes.c_int, ctypes.c_size_t, ctypes.c_size_t, _vp, _vp, _vp, ctypes.c_int,
                          ctypes.c_int, _vp], ctypes.c_int),
    "nuna_expert_layer_few_workspace": ([ctypes.c_int, ctypes.c_int, ctypes.c_size_t, ctypes.c_size_t,
                                         ctypes.POINTER(ctypes.c_size_t)], ctypes.c_int),
    "nuna_expert_layer_few": ([_vp, ctypes.c_int64, _vp, _vp, ctypes.c_int, ctypes.c_int, _vp, _vp, _vp, _vp, ctypes.c_int,
                               ctypes.c_int, ctypes.c_size_t, ctypes.c_size_t, _vp, _vp, ctypes.c_size_t, ctypes.c_int,
                               ctypes.c_int, _vp], ctypes.c_int),
    "nuna_placement_items": ([ctypes.c_int, ctypes.c_int64, ctypes.c_int64, ctypes.c_int64, ctypes.c_int64, _i64p,
                              ctypes.c_int64, _i64p], ctypes.c_int),
    "nuna_placement_grid": ([ctypes.c_int, ctypes.c_int64, ctypes.c_int64, _i64p], ctypes.c_int),
    "nuna_placement_direct": ([ctypes.c_int, ctypes.c_int64, ctypes.c_int64, _i64p, ctypes.c_int64, _i64p],
                              ctypes.c_int),
    "nuna_probe_xcc": ([ctypes.c_int, _vp, _vp, _vp], ctypes.c_int),
    "nuna_copy": ([_vp, _vp, ctypes.c_size_t, _vp], ctypes.c_int),
    "nuna_ref_stream": ([ctypes.c_int, _vpp, _vpp, ctypes.c_int, ctypes.c_size_t, _vp], ctypes.c_int),
    "nuna_nap_topology_mi355x": ([ctypes.POINTER(NapTopology)], ctypes.c_int),
    "nuna_nap_plan": ([ctypes.POINTER(NapTopology), ctypes.c_int, ctypes.c_int64, _i64p, _i64p, _i64p, _i64p,
                       _i64p, _i32p, _i32p, _i32p, _i64p], ctypes.c_int),
    "nuna_probe_load_latency_cus": ([_vp, ctypes.c_size_t, ctypes.c_size_t, ctypes.c_int, _vp, _vp, _vp, _vp],
                                    ctypes.c_int),
    "nuna_probe_load_latency": ([_vp, ctypes.c_size_t, ctypes.c_size_t, ctypes.c_size_t, ctypes.c_int, _vp, _vp],
                                ctypes.c_int),
}

_lib = None


class NunaError(RuntimeError):
    def __init__(self, status, msg):
        super().__init__(f"{STATUS_NAMES.get(status, status)}: {msg}")
        self.status = status


def lib():
    """Load libnuna.so once.  Raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is not built; run `python -c 'import __graft_entry__ as g; g.build()'`")
        L = ctypes.CDLL(LIB_PATH)
        for name, (args, res) in SIGNATURES.items():
            fn = getattr(L, name)
            fn.argtypes = args
            fn.restype = res
        _lib = L
    return _lib


def last_error():
    return lib().nuna_last_error_string().decode()


def _check(st):
    if st != OK:
        raise NunaError(st, last_error())


def _ptr_array(ptrs):
    return (ctypes.c_void_p * max(len(ptrs), 1))(*[int(p) if p is not None else None for p in ptrs])


# ------------------------------------------------------------------ raw ABI (integer pointers)

def allreduce_raw(in_ptrs, out_ptrs, P, count, dtype, algo=ALGO_AUTO, place=XCD, stream=0):
    a = _ptr_array(in_ptrs) if in_ptrs is not None else None
    b = _ptr_array(out_ptrs) if out_ptrs is not None else None
    return lib().nuna_allreduce(a, b, P, count, dtype, algo, place, stream)


def reduce_scatter_raw(in_ptrs, out_ptrs, P, recvcount, dtype, place=XCD, stream=0):
    a = _ptr_array(in_ptrs) if in_ptrs is not None else None
    b = _ptr_array(out_ptrs) if out_ptrs is not None else None
    return lib().nuna_reduce_scatter(a, b, P, recvcount, dtype, place, stream)


def all_gather_raw(in_ptrs, out_ptrs, P, sendcount, dtype, place=XCD, stream=0):
    a = _ptr_array(in_ptrs) if in_ptrs is not None else None
    b = _ptr_array(out_ptrs) if out_ptrs is not None else None
    return lib().nuna_all_gather(a, b, P, sendcount, dtype, place, stream)


def all_to_all_raw(send_ptrs, recv_ptrs, layout_handle, row_elems, recv_capacity_rows, dtype, place=XCD, stream=0):
    a = _ptr_array(send_ptrs) if send_ptrs is not None else None
    b = _ptr_array(recv_ptrs) if recv_ptrs is not None else None
    return lib().nuna_all_to_all(a, b, layout_handle, row_elems, recv_capacity_rows, dtype, place, stream)


def all_to_all_combine_raw(y_ptrs, out_ptrs, layout_handle, row_elems, y_capacity_rows, dtype, place=XCD, stream=0,
                           weights_ptr=None):
    a = _ptr_array(y_ptrs) if y_ptrs is not None else None
    b = _ptr_array(out_ptrs) if out_ptrs is not None else None
    return lib().nuna_all_to_all_combine(a, b, layout_handle, weights_ptr, row_elems, y_capacity_rows, dtype, place,
                                         stream)


def placement_items(place, b, G, groups, group_size):
    """Work items workgroup b of G runs, in order (host mirror of the kernels' map)."""
    import numpy as np
    cnt = ctypes.c_int64()
    lib().nuna_placement_items(PLACEMENTS[place], b, G, groups, group_size, None, 0, ctypes.byref(cnt))
    n = cnt.value
    buf = np.zeros(max(n, 1), dtype=np.int64)
    _check(lib().nuna_placement_items(PLACEMENTS[place], b, G, groups, group_size, buf.ctypes.data_as(_i64p), n,
                                      ctypes.byref(cnt)))
    return buf[:n].tolist()


def placement_grid(place, groups, group_size):
    """Workgroups a launch of this placement uses (before the cap)."""
    g = ctypes.c_int64()
    _check(lib().nuna_placement_grid(PLACEMENTS[place], groups, group_size, ctypes.byref(g)))
    return g.value


def placement_direct(place, items, chunk_bytes):
    """Item each workgroup of a one-item-per-workgroup launch runs (-1: padding), host mirror."""
    import numpy as np
    g = ctypes.c_int64()
    lib().nuna_placement_direct(PLACEMENTS[place], items, chunk_bytes, None, 0, ctypes.byref(g))
    buf = np.zeros(max(g.value, 1), dtype=np.int64)
    _check(lib().nuna_placement_direct(PLACEMENTS[place], items, chunk_bytes, buf.ctypes.data_as(_i64p), g.value,
                                       ctypes.byref(g)))
    return buf[:g.value]


def nap_topology_mi355x(cu_budget=None, stack_budget=None):
    """The library's MI355X topology for the placement planner, budgets optionally replaced."""
    t = NapTopology()
    _check(lib().nuna_nap_topology_mi355x(ctypes.byref(t)))
    if cu_budget is not None:
        t.cu_budget = int(cu_budget)
    if stack_budget is not None:
        t.stack_budget = int(stack_budget)
    return t


def nap_plan(tb_chunks, tb_bytes, nar_max, topo=None, entry_pages=None):
    """Algorithm 1 in the library: tb_chunks is a list of chunk-id lists (one per threadblock),
    tb_bytes the charge of each.  Returns numpy arrays tb_group, tb_domain, tb_cu, entry_stack
    (aligned with the flattened chunk lists) and the group count."""
    import numpy as np
    topo = nap_topology_mi355x() if topo is None else topo
    n = len(tb_chunks)
    off = np.zeros(n + 1, dtype=np.int64)
    off[1:] = np.cumsum([len(c) for c in tb_chunks])
    ids = np.array([c for cs in tb_chunks for c in cs], dtype=np.int64)
    cs = np.ascontiguousarray(tb_bytes, dtype=np.int64)
    pages = None if entry_pages is None else np.ascontiguousarray(entry_pages, dtype=np.int64)
    g = np.zeros(n, dtype=np.int64)
    d = np.zeros(n, dtype=np.int32)
    cu = np.zeros(n, dtype=np.int32)
    st = np.zeros(max(1, ids.size), dtype=np.int32)
    ng = ctypes.c_int64()
    ptr = lambda a, t: a.ctypes.data_as(t) if a is not None and a.size else None  # noqa: E731
    _check(lib().nuna_nap_plan(ctypes.byref(topo), int(nar_max), n, ptr(off, _i64p), ptr(ids, _i64p),
                               ptr(cs, _i64p), ptr(pages, _i64p), ptr(g, _i64p), ptr(d, _i32p), ptr(cu, _i32p),
                               ptr(st, _i32p), ctypes.byref(ng)))
    return {"tb_group": g, "tb_domain": d, "tb_cu": cu, "entry_stack": st[:ids.size], "num_groups": ng.value}


def set_tunable(name, value):
    """Set a launch-shape tunable (NUNA_* name) for later calls; never changes results."""
    _check(lib().nuna_set_tunable(name.encode(), int(value)))


def get_tunable(name):
    v = ctypes.c_int64()
    _check(lib().nuna_get_tunable(name.encode(), ctypes.byref(v)))
    return v.value


class tunables:
    """Context manager: set tunables on entry, restore the previous values on exit."""

    def __init__(self, **values):
        self.values = values
        self.saved = {}

    def __enter__(self):
        for k, v in self.values.items():
            self.saved[k] = get_tunable(k)
            set_tunable(k, v)
        return self

    def __exit__(self, *exc):
        for k, v in self.saved.items():
            set_tunable(k, v)
        return False


def init():
    """Probe the current device (architecture, dispatch map); XCD placement needs it."""
    _check(lib().nuna_init())


def device_info():
    """What nuna_init found on the current device: dict of device, cu_count, xcd_count, map_verified."""
    info = DeviceInfo()
    _check(lib().nuna_get_device_info(ctypes.byref(info)))
    return {k: int(getattr(info, k)) for k, _ in DeviceInfo._fields_}


def last_launch():
    """Kernels and map of the calling thread's last collective call (dict)."""
    info = LaunchInfo()
    _check(lib().nuna_last_launch(ctypes.byref(info)))
    d = {k: getattr(info, k) for k, _ in LaunchInfo._fields_}
    d["kernels"] = info.kernels.decode()
    d["map"] = MAP_NAMES.get(int(info.map), int(info.map))
    return d


def check_dispatch_map_raw(xcc, cu_count):
    """Status of the library's host-side dispatch-map check on an int32 array of per-workgroup XCC ids."""
    import numpy as np
    a = np.ascontiguousarray(xcc, dtype=np.int32)
    return lib().nuna_check_dispatch_map(a.ctypes.data_as(_i32p) if a.size else None, int(a.size), int(cu_count))


def set_max_workgroups(n):
    """Cap workgroups per launch (0 = default); launch shape only, never results."""
    _check(lib().nuna_set_max_workgroups(int(n)))


# ------------------------------------------------------------------ tensor API

_torch_module = None


def _torch():
    global _torch_module
    if _torch_module is None:
        import torch
        _torch_module = torch
    return _torch_module


def _dtype_code(t):
    torch = _torch()
    if t.dtype == torch.float32:
        return F32
    if t.dtype == torch.bfloat16:
        return BF16
    raise TypeError(f"unsupported dtype {t.dtype}")


def _stream(stream):
    torch = _torch()
    s = torch.cuda.current_stream() if stream is None else stream
    return s.cuda_stream


def _check_ranks(ts, name):
    if not ts:
        raise ValueError(f"{name}: need at least one rank buffer")
    d, n = ts[0].dtype, ts[0].numel()
    for t in ts:
        if not t.is_cuda or not t.is_contiguous() or t.dtype != d or t.numel() != n:
            raise ValueError(f"{name}: rank buffers must be contiguous CUDA tensors of one dtype and size")
    return d, n


def _check_outs(ins, outs, n_out):
    """One output per input rank, each of the input dtype and n_out elements: checked before any
    pointer reaches the library, which sizes every output from the input dtype."""
    if len(outs) != len(ins):
        raise ValueError(f"need one output per rank: {len(outs)} outputs for {len(ins)} inputs")
    for o in outs:
        if o.dtype != ins[0].dtype:
            raise ValueError(f"output dtype {o.dtype} differs from input dtype {ins[0].dtype}")
        if o.numel() != n_out:
            raise ValueError(f"each output holds {n_out} elements, got {o.numel()}")


def allreduce(ins, outs=None, algo="auto", placement="xcd", stream=None):
    """out[d] = sum over ranks r (ascending, fp32 accumulation) of ins[r], for every d."""
    _, n = _check_ranks(ins, "ins")
    if outs is None:
        outs = [_torch().empty_like(ins[0]) for _ in ins]
    _check_outs(ins, outs, n)
    _check_ranks(outs, "outs")
    _check(allreduce_raw([t.data_ptr() for t in ins], [t.data_ptr() for t in outs], len(ins), n,
                         _dtype_code(ins[0]), ALGOS[algo], PLACEMENTS[placement], _stream(stream)))
    return outs


class Prepared:
    """A collective call whose buffers were checked and whose arguments were marshalled once.
    Calling it launches the collective again, on `stream` (a torch stream, a raw stream handle, or
    None for torch's current stream), with no per-call Python checks.  The tensors it was built
    from must stay alive and keep their storage; they are held by this object."""

    def __init__(self, fn, args, keep):
        self._fn = fn
        self._args = args
        self._keep = keep

    def __call__(self, stream=None):
        if stream is None:
            h = _torch().cuda.current_stream().cuda_stream
        elif isinstance(stream, int):
            h = stream
        else:
            h = stream.cuda_stream
        _check(self._fn(*self._args, h))


def prepare_allreduce(ins, outs, algo="auto", placement="xcd"):
    """allreduce(ins, outs, algo, placement) as a Prepared call."""
    _, n = _check_ranks(ins, "ins")
    _check_outs(ins, outs, n)
    _check_ranks(outs, "outs")
    a = _ptr_array([t.data_ptr() for t in ins])
    b = _ptr_array([t.data_ptr() for t in outs])
    args = (a, b, len(ins), n, _dtype_code(ins[0]), ALGOS[algo], PLACEMENTS[placement])
    return Prepared(lib().nuna_allreduce, args, (list(ins), list(outs)))


def reduce_scatter(ins, outs=None, placement="xcd", stream=None):
    """outs[r][j] = sum over q ascending of ins[q][r*m + j], m = numel / P."""
    _, n = _check_ranks(ins, "ins")
    P = len(ins)
    if n % P:
        raise ValueError("reduce-scatter input size must be a multiple of P")
    m = n // P
    if outs is None:
        outs = [_torch().empty(m, dtype=ins[0].dtype, device=ins[0].device) for _ in ins]
    _check_outs(ins, outs, m)
    _check_ranks(outs, "outs")
    _check(reduce_scatter_raw([t.data_ptr() for t in ins], [t.data_ptr() for t in outs], P, m, _dtype_code(ins[0]),
                              PLACEMENTS[placement], _stream(stream)))
    return outs


def all_gather(ins, outs=None, placement="xcd", stream=None):
    """outs[d][r*m + j] = ins[r][j] for every d."""
    _, m = _check_ranks(ins, "ins")
    P = len(ins)
    if outs is None:
        outs = [_torch().empty(P * m, dtype=ins[0].dtype, device=ins[0].device) for _ in ins]
    _check_outs(ins, outs, P * m)
    _check_ranks(outs, "outs")
    _check(all_gather_raw([t.data_ptr() for t in ins], [t.data_ptr() for t in outs], P, m, _dtype_code(ins[0]),
                          PLACEMENTS[placement], _stream(stream)))
    return outs


class A2ALayout:
    """Routing plan of one MoE dispatch (host planning in the library)."""

    def __init__(self, topk_idx, num_experts):
        import numpy as np
        topk = np.ascontiguousarray(topk_idx, dtype=np.int32)
        if topk.ndim != 3:
            raise ValueError("topk_idx must be [P, tokens_per_rank, topk]")
        self.P, self.T, self.k = (int(x) for x in topk.shape)
        self.num_experts = int(num_experts)
        self._topk = topk
        h = ctypes.c_void_p()
        _check(lib().nuna_a2a_layout_create(self.P, self.T, self.k, self.num_experts,
                                            topk.ctypes.data if topk.size else None, ctypes.byref(h)))
        self.handle = h

    def upload(self):
        _check(lib().nuna_a2a_layout_upload(self.handle))
        return self

    def recv_rows(self):
        import numpy as np
        rows = np.zeros(self.P, dtype=np.int64)
        _check(lib().nuna_a2a_layout_recv_rows(self.handle, rows.ctypes.data_as(_i64p)))
        return rows

    def recv_map(self, d):
        import numpy as np
        n = int(self.recv_rows()[d])
        sr = np.zeros(max(n, 1), dtype=np.int32)
        st = np.zeros(max(n, 1), dtype=np.int32)
        _check(lib().nuna_a2a_layout_recv_map(self.handle, d, sr.ctypes.data_as(_i32p), st.ctypes.data_as(_i32p)))
        return sr[:n], st[:n]

    def close(self):
        if getattr(self, "handle", None) is not None and self.handle.value:
            lib().nuna_a2a_layout_destroy(self.handle)
        self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def all_to_all(send, recv, layout, placement="xcd", stream=None):
    """recv[d][j] = send[s][t] for the j-th row (s, t) routed to d by the layout."""
    P = layout.P
    if len(send) != P or len(recv) != P:
        raise ValueError("one send and one recv buffer per rank")
    for t in send:
        if not t.is_cuda or not t.is_contiguous() or t.dim() != 2 or t.shape != send[0].shape:
            raise ValueError("send buffers must be contiguous CUDA tensors [T, row]")
    row = send[0].shape[1]
    cap = recv[0].shape[0]
    for t in recv:
        if not t.is_cuda or not t.is_contiguous() or t.dim() != 2 or t.shape[1] != row or t.dtype != send[0].dtype:
            raise ValueError("recv buffers must be contiguous CUDA tensors [capacity, row] of the send dtype")
        cap = min(cap, t.shape[0])
    _check(all_to_all_raw([t.data_ptr() for t in send], [t.data_ptr() for t in recv], layout.handle, row, cap,
                          _dtype_code(send[0]), PLACEMENTS[placement], _stream(stream)))
    return recv


def all_to_all_routed_raw(send_ptrs, recv_ptrs, topk_ptr, P, T, k, E, row_elems, recv_capacity_rows, dtype,
                          rows_ptr, place=XCD, stream=0):
    a = _ptr_array(send_ptrs) if send_ptrs is not None else None
    b = _ptr_array(recv_ptrs) if recv_ptrs is not None else None
    return lib().nuna_all_to_all_routed(a, b, topk_ptr, P, T, k, E, row_elems, recv_capacity_rows, dtype, place,
                                        rows_ptr, stream)


def all_to_all_routed(send, recv, topk_idx, num_experts, rows_per_rank, placement="xcd", stream=None):
    """Dispatch with the routing on the device and no allocation: topk_idx an int32 CUDA tensor
    [P, T, k]; rows_per_rank an int64 CUDA tensor of P + 1 that receives the rows each rank gets
    (and, last, the count of out-of-range experts)."""
    torch = _torch()
    P = len(send)
    if len(recv) != P or topk_idx.dim() != 3 or topk_idx.shape[0] != P or topk_idx.dtype != torch.int32:
        raise ValueError("one send and one recv buffer per rank; topk_idx int32 [P, T, k]")
    if not topk_idx.is_cuda or not topk_idx.is_contiguous():
        raise ValueError("topk_idx must be a contiguous CUDA tensor")
    if (not rows_per_rank.is_cuda or rows_per_rank.dtype != torch.int64 or rows_per_rank.numel() != P + 1
            or not rows_per_rank.is_contiguous()):
        raise ValueError("rows_per_rank must be a contiguous int64 CUDA tensor of P + 1")
    T, k = int(topk_idx.shape[1]), int(topk_idx.shape[2])
    for t in send:
        if not t.is_cuda or not t.is_contiguous() or t.dim() != 2 or t.shape != (T, send[0].shape[1]):
            raise ValueError("send buffers must be contiguous CUDA tensors [T, row]")
    row = send[0].shape[1]
    cap = recv[0].shape[0]
    for t in recv:
        if not t.is_cuda or not t.is_contiguous() or t.dim() != 2 or t.shape[1] != row or t.dtype != send[0].dtype:
            raise ValueError("recv buffers must be contiguous CUDA tensors [capacity, row] of the send dtype")
        cap = min(cap, t.shape[0])
    _check(all_to_all_routed_raw([t.data_ptr() for t in send], [t.data_ptr() for t in recv], topk_idx.data_ptr(),
                                 P, T, k, int(num_experts), row, cap, _dtype_code(send[0]), rows_per_rank.data_ptr(),
                                 PLACEMENTS[placement], _stream(stream)))
    return recv


def all_to_all_combine(y, out, layout, placement="xcd", stream=None, weights=None):
    """out[s][t] = sum over the ranks d that token (s, t) was sent to (ascending) of its result row in y[d],
    each first scaled by weights[s, t, d] when weights (float32 CUDA tensor [P, T, P]) is given."""
    P = layout.P
    wp = None
    if weights is not None:
        if (not weights.is_cuda or weights.dtype != _torch().float32 or not weights.is_contiguous()
                or tuple(weights.shape) != (P, layout.T, P)):
            raise ValueError("weights must be a contiguous float32 CUDA tensor [P, T, P]")
        wp = weights.data_ptr()
    if len(y) != P or len(out) != P:
        raise ValueError("one result and one output buffer per rank")
    for t in out:
        if not t.is_cuda or not t.is_contiguous() or t.dim() != 2 or t.shape != out[0].shape:
            raise ValueError("output buffers must be contiguous CUDA tensors [T, row]")
    row = out[0].shape[1]
    cap = y[0].shape[0]
    for t in y:
        if not t.is_cuda or not t.is_contiguous() or t.dim() != 2 or t.shape[1] != row or t.dtype != out[0].dtype:
            raise ValueError("result buffers must be contiguous CUDA tensors [capacity, row] of the output dtype")
        cap = min(cap, t.shape[0])
    _check(all_to_all_combine_raw([t.data_ptr() for t in y], [t.data_ptr() for t in out], layout.handle, row, cap,
                                  _dtype_code(out[0]), PLACEMENTS[placement], _stream(stream), wp))
    return out


# ------------------------------------------------------------------ the expert layer
#
# All tensors of a call are on the current device, and so is the stream.

SCALES = {"f32": SCALE_F32, "e8m0": SCALE_E8M0}


def f8_width(cols):
    """Columns of an 8-bit matrix as it is kept: whole blocks of 128."""
    return -(-cols // F8_BLOCK) * F8_BLOCK


def f8_pitch(cols):
    """Scales in one of its rows: a block each, to a multiple of four."""
    return -(-(f8_width(cols) // F8_BLOCK) // 4) * 4


def f8_cols_width(rows, groups):
    """Columns of `rows` rows laid out along the rows of `groups` groups (f8_quantize_cols)."""
    return F8_BLOCK * (rows // F8_BLOCK + groups)


def _scale_kind(t, name="scale"):
    torch = _torch()
    if t.dtype == torch.float32:
        return SCALE_F32
    if t.dtype == torch.float8_e8m0fnu:
        return SCALE_E8M0
    raise TypeError(f"{name}: unsupported scale dtype {t.dtype}")


def _scale_dtype(scale):
    torch = _torch()
    if scale not in SCALES:
        raise ValueError(f"scale {scale!r} is not one of {sorted(SCALES)}")
    return torch.float32 if scale == "f32" else torch.float8_e8m0fnu


def _current_device():
    return _torch()._C._cuda_getDevice()


def _device_of(t, name):
    """The device of a call's first tensor, which has to be the current one: kernels are launched there."""
    dev = t.get_device()
    if dev < 0:
        raise ValueError(f"{name} must be a CUDA tensor, got {list(t.shape)} of {t.dtype} on the CPU")
    if dev != _current_device():
        raise ValueError(f"{name} is on device {dev}, the current one is {_current_device()}")
    return dev


def _handle(stream, dev):
    """The stream to enqueue on: that given (a torch stream or a raw handle), or torch's current one of device `dev`.
    The raw handle is asked for directly: making the Stream object took 2.7 us, of calls of 4 to 5 us."""
    if stream is None:
        return _torch()._C._cuda_getCurrentRawStream(dev)
    if isinstance(stream, int):
        return stream
    if stream.device_index != dev:
        raise ValueError(f"a stream of device {stream.device_index} for tensors on device {dev}")
    return stream.cuda_stream


def _check_tensor(t, name, shape, dtype, dev):
    """A contiguous tensor of this shape (a tuple) and dtype on device `dev`."""
    if not (t.dtype is dtype and t.shape == shape and t.get_device() == dev and t.is_contiguous()):
        raise ValueError(f"{name} must be a contiguous CUDA tensor {list(shape)} of {dtype} on device {dev}, "
                         f"got {list(t.shape)} of {t.dtype} on {t.device}")


def _check_matrix(t, name, dev):
    """A tensor [rows, cols] on device `dev` whose rows are contiguous; returns its row stride."""
    if t.get_device() != dev or t.dim() != 2:
        raise ValueError(f"{name} must be a CUDA tensor [rows, cols] with contiguous rows, on device {dev}")
    rows, cols = t.shape
    if t.is_contiguous() and cols:
        return cols
    if cols < 1 or (cols > 1 and t.stride(1) != 1):
        raise ValueError(f"{name} must be a CUDA tensor [rows, cols] with contiguous rows")
    stride = t.stride(0) if rows > 1 else cols
    if stride < cols:
        raise ValueError(f"{name}: its rows overlap")
    return stride


def _check_table(t, name, dev):
    if not (t.get_device() == dev and t.dtype is _torch().int32 and t.dim() == 2 and t.is_contiguous() and t.shape[1]):
        raise ValueError(f"{name} must be a contiguous int32 CUDA tensor [tokens, topk], on device {dev}")
    return t.shape


def _check_offsets(t, dev):
    if t.get_device() != dev or not t.is_contiguous() or t.dim() != 1 or t.dtype != _torch().int32 or t.numel() < 2:
        raise ValueError(f"offsets must be a contiguous int32 CUDA tensor [groups + 1], on device {dev}")
    return t.numel() - 1


def _new(stream, shape, dtype, device):
    """An uninitialised tensor that belongs to the stream it is used on."""
    torch = _torch()
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    if isinstance(stream, int):
        raise ValueError("a raw stream handle needs every output and workspace to be given")
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=device)


def _f8_outputs(out, scale_out, shape, scale_shape, scale, stream, device, dev):
    """The 8-bit output and its scales: those given, checked, or new ones of the scale type `scale`."""
    torch = _torch()
    if out is None:
        out = _new(stream, shape, torch.float8_e4m3fn, device)
    if scale_out is None:
        scale_out = _new(stream, scale_shape, _scale_dtype(scale), device)
    _check_tensor(out, "out", shape, torch.float8_e4m3fn, dev)
    _check_tensor(scale_out, "scale_out", scale_shape, _scale_dtype(scale), dev)
    return out, scale_out


@functools.lru_cache(maxsize=256)
def moe_sort_workspace(tokens, topk, num_experts):
    """Bytes of workspace that moe_sort needs."""
    n = ctypes.c_size_t()
    _check(lib().nuna_moe_sort_workspace(int(tokens), int(topk), int(num_experts), ctypes.byref(n)))
    return n.value


def moe_sort(topk_idx, num_experts, first_expert=0, offsets=None, slot_of=None, row_of=None, workspace=None,
             stream=None):
    """Sort the slots of topk_idx (int32 CUDA tensor [T, k]) by expert, stable, for the num_experts experts from
    first_expert on; other entries sort nowhere.  Returns (offsets [num_experts + 1], slot_of [T * k], row_of [T, k]),
    int32: expert e holds the rows offsets[e] .. offsets[e + 1], slot_of[row] is a row's slot t * k + j (-1 past the
    last), row_of[t, j] a slot's row (-1: none).  Where none of them is given they are parts of one allocation.
    workspace: a uint8 CUDA tensor of moe_sort_workspace bytes."""
    torch = _torch()
    index = _device_of(topk_idx, "topk_idx")
    T, k = _check_table(topk_idx, "topk_idx", index)
    num_experts = int(num_experts)
    need = moe_sort_workspace(T, k, num_experts)
    dev, n = topk_idx.device, T * k
    if offsets is None and slot_of is None and row_of is None:
        # A workspace that is not given is a fourth part (2 MiB at most): an allocation of its own took 1 us of 13.
        own = need // 4 if workspace is None else 0
        sizes = (n, n, num_experts + 1, own) if own else (n, n, num_experts + 1)
        size = 2 * n + num_experts + 1 + own
        whole = topk_idx.new_empty(size) if stream is None else _new(stream, (size,), torch.int32, dev)
        slot_of, row_of, offsets, *part = whole.split_with_sizes(sizes)
        row_of = row_of.view(T, k)
        if own:
            workspace = part[0].view(torch.uint8)
    else:
        offsets = _new(stream, (num_experts + 1,), torch.int32, dev) if offsets is None else offsets
        slot_of = _new(stream, (n,), torch.int32, dev) if slot_of is None else slot_of
        row_of = _new(stream, (T, k), torch.int32, dev) if row_of is None else row_of
        _check_tensor(offsets, "offsets", (num_experts + 1,), torch.int32, index)
        _check_tensor(slot_of, "slot_of", (n,), torch.int32, index)
        _check_tensor(row_of, "row_of", (T, k), torch.int32, index)
    if workspace is None:
        workspace = _new(stream, (need,), torch.uint8, dev) if need else None
    elif workspace.get_device() != index or not workspace.is_contiguous() or workspace.dtype != torch.uint8:
        raise ValueError(f"workspace must be a contiguous uint8 CUDA tensor on device {index}")
    _check(lib().nuna_moe_sort(topk_idx.data_ptr(), T, k, int(first_expert), num_experts, offsets.data_ptr(),
                               slot_of.data_ptr(), row_of.data_ptr(), workspace.data_ptr() if need else None,
                               workspace.numel() if need else 0, _handle(stream, index)))
    return offsets, slot_of, row_of


def moe_gather(x, row_of, out, scale_out=None, stream=None):
    """out[row_of[t, j]] = x[t] for every slot with a row of out; other rows are left untouched.  x [T, H] with
    contiguous rows.  out [rows, H] of x's dtype, or float8_e4m3fn [rows, f8_width(H)] with scale_out [rows,
    f8_pitch(H)] (float32 or float8_e8m0fnu): each row quantised as f8_quantize does.  Returns out, or (out,
    scale_out).  The gradient of the first form is moe_scatter without weights."""
    torch = _torch()
    dev = _device_of(x, "x")
    T, k = _check_table(row_of, "row_of", dev)
    stride = _check_matrix(x, "x", dev)
    H = x.shape[1]
    if x.shape[0] != T:
        raise ValueError(f"x has {x.shape[0]} rows, row_of {T}")
    if out.dim() != 2:
        raise ValueError("out must be [rows, columns]")
    cap = out.shape[0]
    if scale_out is None:
        _check_tensor(out, "out", (cap, H), x.dtype, dev)
        _check(lib().nuna_moe_gather(x.data_ptr(), stride, row_of.data_ptr(), T, k, H, out.data_ptr(), cap,
                                     _dtype_code(x), _handle(stream, dev)))
        return out
    _check_tensor(out, "out", (cap, f8_width(H)), torch.float8_e4m3fn, dev)
    kind = _scale_kind(scale_out, "scale_out")
    _check_tensor(scale_out, "scale_out", (cap, f8_pitch(H)), scale_out.dtype, dev)
    _check(lib().nuna_moe_gather_f8(x.data_ptr(), stride, row_of.data_ptr(), T, k, H, out.data_ptr(),
                                    scale_out.data_ptr(), cap, _dtype_code(x), kind, _handle(stream, dev)))
    return out, scale_out


def _check_weights(weights, T, k, dev):
    _check_tensor(weights, "weights", (T, k), _torch().float32, dev)
    return weights.data_ptr()


def moe_scatter(y, row_of, weights=None, out=None, stream=None):
    """out[t] = sum over j, ascending, of weights[t, j] * y[row_of[t, j]] (float32 weights [T, k], or None: 1) over
    the slots with a row of y; fp32 sums, rounded once.  A token without a row gets zeros."""
    dev = _device_of(y, "y")
    T, k = _check_table(row_of, "row_of", dev)
    if y.dim() != 2:
        raise ValueError("y must be [rows, columns]")
    cap, H = y.shape
    _check_tensor(y, "y", (cap, H), y.dtype, dev)
    wp = None if weights is None else _check_weights(weights, T, k, dev)
    if out is None:
        out = _new(stream, (T, H), y.dtype, y.device)
    _check_tensor(out, "out", (T, H), y.dtype, dev)
    _check(lib().nuna_moe_scatter(y.data_ptr(), row_of.data_ptr(), wp, T, k, H, cap, out.data_ptr(), _dtype_code(y),
                                  _handle(stream, dev)))
    return out


def moe_scatter_grad(dout, y, row_of, weights, dy=None, dweights=None, stream=None):
    """Gradient of moe_scatter: (dy, dweights) with dy[row_of[t, j]] = weights[t, j] * dout[t] and dweights[t, j] =
    <dout[t], y[row_of[t, j]]> (fp32; 0 for a slot without a row).  Rows of dy that no slot names are left untouched,
    and are zeros where dy is not given."""
    torch = _torch()
    dev = _device_of(y, "y")
    T, k = _check_table(row_of, "row_of", dev)
    if y.dim() != 2:
        raise ValueError("y must be [rows, columns]")
    cap, H = y.shape
    _check_tensor(y, "y", (cap, H), y.dtype, dev)
    _check_tensor(dout, "dout", (T, H), y.dtype, dev)
    wp = _check_weights(weights, T, k, dev)
    if dy is None:
        dy = _new(stream, (cap, H), y.dtype, y.device)
        with torch.cuda.stream(stream):
            dy.zero_()
    if dweights is None:
        dweights = _new(stream, (T, k), torch.float32, y.device)
    _check_tensor(dy, "dy", (cap, H), y.dtype, dev)
    _check_tensor(dweights, "dweights", (T, k), torch.float32, dev)
    _check(lib().nuna_moe_scatter_grad(dout.data_ptr(), y.data_ptr(), row_of.data_ptr(), wp, T, k, H, cap,
                                       dy.data_ptr(), dweights.data_ptr(), _dtype_code(y), _handle(stream, dev)))
    return dy, dweights


def f8_quantize(x, scale="f32", out=None, scale_out=None, stream=None):
    """x [rows, cols] (contiguous rows) to e4m3 with a scale ("f32" or "e8m0") for every 128 columns of a row.  Returns
    (out float8_e4m3fn [rows, f8_width(cols)], zeros past the last column; scale_out [rows, f8_pitch(cols)])."""
    dev = _device_of(x, "x")
    stride = _check_matrix(x, "x", dev)
    rows, cols = x.shape
    out, scale_out = _f8_outputs(out, scale_out, (rows, f8_width(cols)), (rows, f8_pitch(cols)), scale, stream,
                                 x.device, dev)
    _check(lib().nuna_f8_quantize(x.data_ptr(), stride, rows, cols, _dtype_code(x), out.data_ptr(),
                                  scale_out.data_ptr(), SCALES[scale], _handle(stream, dev)))
    return out, scale_out


def f8_quantize_blocks(x, scale="f32", out=None, scale_out=None, stream=None):
    """Weights x [.., rows, cols] to e4m3 with a scale for every block of 128 x 128.  Returns (out [.., rows,
    f8_width(cols)], scale_out [.., ceil(rows / 128), f8_pitch(cols)])."""
    dev = _device_of(x, "x")
    if not x.is_contiguous() or x.dim() < 2 or x.shape[-1] < 1:
        raise ValueError("x must be a contiguous CUDA tensor [.., rows, cols]")
    lead, (rows, cols) = tuple(x.shape[:-2]), x.shape[-2:]
    batch = 1
    for n in lead:
        batch *= n
    out, scale_out = _f8_outputs(out, scale_out, (*lead, rows, f8_width(cols)),
                                 (*lead, -(-rows // F8_BLOCK), f8_pitch(cols)), scale, stream, x.device, dev)
    _check(lib().nuna_f8_quantize_blocks(x.data_ptr(), batch, rows, cols, _dtype_code(x), out.data_ptr(),
                                         scale_out.data_ptr(), SCALES[scale], _handle(stream, dev)))
    return out, scale_out


def f8_quantize_cols(x, offsets, scale="f32", out=None, scale_out=None, slot_of=None, topk=1, stream=None):
    """The rows of x grouped by offsets (int32 [groups + 1]), transposed and quantised along the rows of each group: a
    scale for every 128 rows of a group.  With slot_of (int32 [rows], of moe_sort) row r is row slot_of[r] // topk of
    x, so that x need not be gathered first.  Returns (out [cols, f8_cols_width(rows, groups)], scale_out), the
    operands of f8_wgrad."""
    torch = _torch()
    dev = _device_of(x, "x")
    stride = _check_matrix(x, "x", dev)
    groups = _check_offsets(offsets, dev)
    x_rows, cols = x.shape
    rows = x_rows
    if slot_of is not None:
        rows = slot_of.numel()
        _check_tensor(slot_of, "slot_of", (rows,), torch.int32, dev)
    width = f8_cols_width(rows, groups)
    out, scale_out = _f8_outputs(out, scale_out, (cols, width), (cols, f8_pitch(width)), scale, stream, x.device,
                                 dev)
    _check(lib().nuna_f8_quantize_cols(x.data_ptr(), stride, x_rows, None if slot_of is None else slot_of.data_ptr(),
                                       int(topk), offsets.data_ptr(), groups, rows, cols, _dtype_code(x),
                                       out.data_ptr(), scale_out.data_ptr(), SCALES[scale], _handle(stream, dev)))
    return out, scale_out


def f8_matmul(a, a_scale, b, b_scale, out=None, offsets=None, out_dtype=None, stream=None):
    """out[r] = b[g] @ a[r] in 8 bits, g the group of row r.  a [rows, k] with its scales (f8_quantize), b [groups, n,
    k] with its block scales (f8_quantize_blocks); offsets int32 [groups + 1] (moe_sort); without offsets b is [n, k]
    and every row is multiplied by it.  out [rows, n] of out_dtype (bfloat16 unless given); rows in no group are left
    untouched, and are zeros where out is not given.  fp32 results come from exact products and fp32 sums; for bfloat16
    the 8-bit matrix instructions lose up to 7 * 2^-13 of the largest product of every 8 (include/nuna.h)."""
    torch = _torch()
    f8 = torch.float8_e4m3fn
    dev = _device_of(a, "a")
    groups = 1 if offsets is None else _check_offsets(offsets, dev)
    lead = () if offsets is None else (groups,)
    if a.dim() != 2 or b.dim() != 2 + len(lead):
        raise ValueError("a must be [rows, k] and b [n, k], or [groups, n, k] with offsets")
    (rows, k), n = a.shape, b.shape[-2]
    kind = _scale_kind(a_scale, "a_scale")
    _check_tensor(a, "a", (rows, k), f8, dev)
    _check_tensor(b, "b", (*lead, n, k), f8, dev)
    _check_tensor(a_scale, "a_scale", (rows, f8_pitch(k)), a_scale.dtype, dev)
    _check_tensor(b_scale, "b_scale", (*lead, -(-n // F8_BLOCK), f8_pitch(k)), a_scale.dtype, dev)
    if out is None:
        out = _new(stream, (rows, n), out_dtype or torch.bfloat16, a.device)
        if offsets is not None:
            with torch.cuda.stream(stream):
                out.zero_()
    _check_tensor(out, "out", (rows, n), out_dtype or out.dtype, dev)
    _check(lib().nuna_f8_matmul(a.data_ptr(), a_scale.data_ptr(), b.data_ptr(), b_scale.data_ptr(),
                                None if offsets is None else offsets.data_ptr(), groups, rows, n, k, out.data_ptr(),
                                kind, _dtype_code(out), _handle(stream, dev)))
    return out


def f8_wgrad(a, a_scale, b, b_scale, offsets, out=None, out_dtype=None, stream=None):
    """Gradient of grouped weights: out[g] = sum over the rows r of group g of a[:, r] b[:, r]^T.  a [n, width] and
    b [k, width] with their scales, both of f8_quantize_cols with these offsets.  out [groups, n, k] of out_dtype
    (float32 unless given; it chooses the sums' precision as in f8_matmul), zeros for a group without rows."""
    torch = _torch()
    f8 = torch.float8_e4m3fn
    dev = _device_of(a, "a")
    groups = _check_offsets(offsets, dev)
    if a.dim() != 2 or b.dim() != 2:
        raise ValueError("a must be [n, width] and b [k, width]")
    (n, width), k = a.shape, b.shape[0]
    rows = width - F8_BLOCK * groups + F8_BLOCK - 1  # the most that this width is the layout of
    if width % F8_BLOCK or rows < 0:
        raise ValueError(f"a of {width} columns is no layout of {groups} groups")
    kind = _scale_kind(a_scale, "a_scale")
    _check_tensor(a, "a", (n, width), f8, dev)
    _check_tensor(b, "b", (k, width), f8, dev)
    _check_tensor(a_scale, "a_scale", (n, f8_pitch(width)), a_scale.dtype, dev)
    _check_tensor(b_scale, "b_scale", (k, f8_pitch(width)), a_scale.dtype, dev)
    if out is None:
        out = _new(stream, (groups, n, k), out_dtype or torch.float32, a.device)
    _check_tensor(out, "out", (groups, n, k), out_dtype or out.dtype, dev)
    _check(lib().nuna_f8_wgrad(a.data_ptr(), a_scale.data_ptr(), b.data_ptr(), b_scale.data_ptr(), offsets.data_ptr(),
                               groups, rows, n, k, out.data_ptr(), kind, _dtype_code(out), _handle(stream, dev)))
    return out


# ------------------------------------------------------------------ around the expert layer
#
# As there, all tensors of a call are on the current device, and so is the stream.

SCORES = {"softmax": SCORE_SOFTMAX, "sigmoid": SCORE_SIGMOID}


def _f8_wanted(scale, q_out, scale_out):
    """Whether a call that can also leave its result in 8 bits shall: where a scale type or an output is given.  Returns
    the scale type, or None."""
    if scale is None and scale_out is not None:
        scale = "f32" if _scale_kind(scale_out, "scale_out") == SCALE_F32 else "e8m0"
    if scale is None and q_out is not None:
        raise ValueError("q_out needs a scale type, or scale_out")
    return scale


def _check_workspace(workspace, dev):
    if workspace.get_device() != dev or not workspace.is_contiguous() or workspace.dtype != _torch().uint8:
        raise ValueError(f"workspace must be a contiguous uint8 CUDA tensor on device {dev}")


def _norm_weight(weight, cols, dtype, dev):
    if weight.dtype is not dtype:
        dtype = _torch().float32
    _check_tensor(weight, "weight", (cols,), dtype, dev)
    return _dtype_code(weight)


def rms_norm(x, weight, eps=1e-6, residual=None, residual_out=None, scale=None, out=None, q_out=None, scale_out=None,
             rstd=None, stream=None):
    """Root-mean-square norm of the rows of x [T, H] (contiguous rows): x / sqrt(mean(x^2) + eps) * weight.  weight [H]
    of x's dtype or float32.  With a residual [T, H] it is added to x first; the sum, rounded to x's dtype, is what is
    normed, and is left in residual_out (the residual itself unless given).  Returns out [T, H]; with a scale type ("f32"
    or "e8m0") or scale_out, the result in 8 bits (q_out, scale_out) as f8_quantize writes it, and out is written only
    where it is given.  rstd: a float32 tensor [T] that receives 1 / sqrt(mean + eps), for the gradient."""
    torch = _torch()
    dev = _device_of(x, "x")
    stride = _check_matrix(x, "x", dev)
    T, H = x.shape
    wd = _norm_weight(weight, H, x.dtype, dev)
    rp = sp = None
    rs = ss = 0
    if residual is not None:
        rs = _check_matrix(residual, "residual", dev)
        residual_out = residual if residual_out is None else residual_out
        ss = rs if residual_out is residual else _check_matrix(residual_out, "residual_out", dev)
        for t, name in ((residual, "residual"), (residual_out, "residual_out")):
            if t.shape != x.shape or t.dtype is not x.dtype:
                raise ValueError(f"{name} must be {list(x.shape)} of {x.dtype}, got {list(t.shape)} of {t.dtype}")
        rp, sp = residual.data_ptr(), residual_out.data_ptr()
    elif residual_out is not None:
        raise ValueError("residual_out without a residual")
    scale = _f8_wanted(scale, q_out, scale_out)
    if scale is not None:
        q_out, scale_out = _f8_outputs(q_out, scale_out, (T, f8_width(H)), (T, f8_pitch(H)), scale, stream, x.device, dev)
    elif out is None:
        out = _new(stream, (T, H), x.dtype, x.device)
    if out is not None:
        _check_tensor(out, "out", (T, H), x.dtype, dev)
    if rstd is not None:
        _check_tensor(rstd, "rstd", (T,), torch.float32, dev)
    _check(lib().nuna_rms_norm(x.data_ptr(), stride, rp, rs, weight.data_ptr(), wd, eps, T, H, sp, ss,
                               None if out is None else out.data_ptr(), None if scale is None else q_out.data_ptr(),
                               None if scale is None else scale_out.data_ptr(), SCALES[scale or "f32"],
                               None if rstd is None else rstd.data_ptr(), _dtype_code(x), _handle(stream, dev)))
    return out if scale is None else (q_out, scale_out)


@functools.lru_cache(maxsize=256)
def rms_norm_grad_workspace(rows, cols):
    """Bytes of workspace that rms_norm_grad needs."""
    n = ctypes.c_size_t()
    _check(lib().nuna_rms_norm_grad_workspace(int(rows), int(cols), ctypes.byref(n)))
    return n.value


def rms_norm_grad(dout, z, weight, rstd, dresidual=None, dx=None, dweight=None, workspace=None, stream=None):
    """Gradient of rms_norm: (dx, dweight).  z [T, H] (contiguous rows) is what was normed (x, or the sum that residual_out
    holds), rstd float32 [T] what rms_norm left there.  dx [T, H] is the gradient of x and of the residual alike;
    dresidual (or None), what reaches the sum by another way, is added to it and may be dx itself.  dweight float32 [H].
    workspace: a uint8 CUDA tensor of rms_norm_grad_workspace bytes."""
    torch = _torch()
    dev = _device_of(z, "z")
    stride = _check_matrix(z, "z", dev)
    T, H = z.shape
    wd = _norm_weight(weight, H, z.dtype, dev)
    _check_tensor(dout, "dout", (T, H), z.dtype, dev)
    _check_tensor(rstd, "rstd", (T,), torch.float32, dev)
    if dresidual is not None:
        _check_tensor(dresidual, "dresidual", (T, H), z.dtype, dev)
    need = rms_norm_grad_workspace(T, H)
    if dx is None:
        dx = _new(stream, (T, H), z.dtype, z.device)
    if dweight is None:
        dweight = _new(stream, (H,), torch.float32, z.device)
    if workspace is None:
        workspace = _new(stream, (need,), torch.uint8, z.device)
    _check_tensor(dx, "dx", (T, H), z.dtype, dev)
    _check_tensor(dweight, "dweight", (H,), torch.float32, dev)
    _check_workspace(workspace, dev)
    _check(lib().nuna_rms_norm_grad(dout.data_ptr(), z.data_ptr(), stride, weight.data_ptr(), wd, rstd.data_ptr(),
                                    None if dresidual is None else dresidual.data_ptr(), T, H, dx.data_ptr(),
                                    dweight.data_ptr(), workspace.data_ptr(), workspace.numel(), _dtype_code(z),
                                    _handle(stream, dev)))
    return dx, dweight


def _score(score):
    if score not in SCORES:
        raise ValueError(f"score {score!r} is not one of {sorted(SCORES)}")
    return SCORES[score]


def route_topk(logits, topk, score="softmax", bias=None, normalize=True, factor=1.0, topk_idx=None, weights=None,
               stream=None):
    """The router's choice: of each token's scores, "softmax" or "sigmoid" of its logits [T, E] (contiguous rows), the topk
    largest.  Returns (topk_idx int32 [T, topk], weights float32 [T, topk]), in descending order, the lowest expert first
    among equals: what moe_sort, all_to_all_routed and moe_scatter take.  bias (float32 [E], sigmoid only) is added to the
    scores for the choice alone.  weights: the chosen scores, divided by their sum where normalize is set, times factor.
    An expert whose logit is -inf is never chosen; where none is left the entry is -1 with weight 0."""
    torch = _torch()
    dev = _device_of(logits, "logits")
    stride = _check_matrix(logits, "logits", dev)
    T, E = logits.shape
    topk = int(topk)
    if bias is not None:
        _check_tensor(bias, "bias", (E,), torch.float32, dev)
    if topk_idx is None:
        topk_idx = _new(stream, (T, topk), torch.int32, logits.device)
    if weights is None:
        weights = _new(stream, (T, topk), torch.float32, logits.device)
    _check_tensor(topk_idx, "topk_idx", (T, topk), torch.int32, dev)
    _check_tensor(weights, "weights", (T, topk), torch.float32, dev)
    _check(lib().nuna_route_topk(logits.data_ptr(), stride, None if bias is None else bias.data_ptr(), T, E, topk,
                                 _score(score), int(bool(normalize)), factor, topk_idx.data_ptr(), weights.data_ptr(),
                                 _dtype_code(logits), _handle(stream, dev)))
    return topk_idx, weights


def route_topk_grad(dweights, logits, topk_idx, score="softmax", normalize=True, factor=1.0, dlogits=None, stream=None):
    """Gradient of route_topk's weights by the logits, [T, E] of their dtype, from dweights float32 [T, topk] and the
    topk_idx of the forward call (the choice itself and its bias have no gradient)."""
    dev = _device_of(logits, "logits")
    stride = _check_matrix(logits, "logits", dev)
    T, E = logits.shape
    rows, k = _check_table(topk_idx, "topk_idx", dev)
    if rows != T:
        raise ValueError(f"logits has {T} rows, topk_idx {rows}")
    _check_tensor(dweights, "dweights", (T, k), _torch().float32, dev)
    if dlogits is None:
        dlogits = _new(stream, (T, E), logits.dtype, logits.device)
    _check_tensor(dlogits, "dlogits", (T, E), logits.dtype, dev)
    _check(lib().nuna_route_topk_grad(dweights.data_ptr(), logits.data_ptr(), stride, topk_idx.data_ptr(), T, E, k,
                                      _score(score), int(bool(normalize)), factor, dlogits.data_ptr(),
                                      _dtype_code(logits), _handle(stream, dev)))
    return dlogits


def _swiglu_outputs(gu, cols, offsets, scale, out, q_out, scale_out, stream, dev):
    """(groups, scale type or None, out, q_out, scale_out) of swiglu or its gradient: those given, checked, or new ones,
    zeros where rows of no group are left alone."""
    rows = gu.shape[0]
    groups = 0 if offsets is None else _check_offsets(offsets, dev)
    scale = _f8_wanted(scale, q_out, scale_out)
    fresh = []
    if scale is not None:
        fresh += [name for name, t in (("q", q_out), ("scale", scale_out)) if t is None]
        q_out, scale_out = _f8_outputs(q_out, scale_out, (rows, f8_width(cols)), (rows, f8_pitch(cols)), scale, stream,
                                       gu.device, dev)
    elif out is None:
        fresh.append("out")
        out = _new(stream, (rows, cols), gu.dtype, gu.device)
    if out is not None:
        _check_tensor(out, "out", (rows, cols), gu.dtype, dev)
    if offsets is not None and fresh:
        torch = _torch()
        with torch.cuda.stream(stream):
            for name in fresh:
                {"q": q_out, "scale": scale_out, "out": out}[name].view(torch.uint8).zero_()
    return groups, scale, out, q_out, scale_out


def swiglu(gu, offsets=None, scale=None, out=None, q_out=None, scale_out=None, stream=None):
    """gate * sigmoid(gate) * up of the halves of gu [rows, 2 * inner]: what stands between an expert's two products.
    Returns out [rows, inner] of gu's dtype; with a scale type ("f32" or "e8m0") or scale_out, the result in 8 bits (q_out,
    scale_out) as f8_quantize writes it, and out is written only where it is given.  offsets int32 [groups + 1]
    (moe_sort): rows in no group are left untouched, and are zeros in outputs that are not given."""
    dev = _device_of(gu, "gu")
    if gu.dim() != 2 or gu.shape[1] < 2 or gu.shape[1] % 2:
        raise ValueError("gu must be [rows, 2 * inner]")
    rows, inner = gu.shape[0], gu.shape[1] // 2
    _check_tensor(gu, "gu", (rows, 2 * inner), gu.dtype, dev)
    groups, scale, out, q_out, scale_out = _swiglu_outputs(gu, inner, offsets, scale, out, q_out, scale_out, stream, dev)
    _check(lib().nuna_swiglu(gu.data_ptr(), None if offsets is None else offsets.data_ptr(), groups, rows, inner,
                             None if out is None else out.data_ptr(), None if scale is None else q_out.data_ptr(),
                             None if scale is None else scale_out.data_ptr(), SCALES[scale or "f32"], _dtype_code(gu),
                             _handle(stream, dev)))
    return out if scale is None else (q_out, scale_out)


def swiglu_grad(dout, gu, offsets=None, scale=None, out=None, q_out=None, scale_out=None, stream=None):
    """Gradient of swiglu by gu, [rows, 2 * inner], from dout [rows, inner]; its outputs and offsets as there."""
    dev = _device_of(gu, "gu")
    if gu.dim() != 2 or gu.shape[1] < 2 or gu.shape[1] % 2:
        raise ValueError("gu must be [rows, 2 * inner]")
    rows, inner = gu.shape[0], gu.shape[1] // 2
    _check_tensor(gu, "gu", (rows, 2 * inner), gu.dtype, dev)
    _check_tensor(dout, "dout", (rows, inner), gu.dtype, dev)
    groups, scale, out, q_out, scale_out = _swiglu_outputs(gu, 2 * inner, offsets, scale, out, q_out, scale_out, stream, dev)
    _check(lib().nuna_swiglu_grad(dout.data_ptr(), gu.data_ptr(), None if offsets is None else offsets.data_ptr(), groups,
                                  rows, inner, None if out is None else out.data_ptr(),
                                  None if scale is None else q_out.data_ptr(),
                                  None if scale is None else scale_out.data_ptr(), SCALES[scale or "f32"],
                                  _dtype_code(gu), _handle(stream, dev)))
    return out if scale is None else (q_out, scale_out)


@functools.lru_cache(maxsize=256)
def expert_layer_few_workspace(tokens, topk, hidden, inner):
    """Bytes of workspace that expert_layer_few needs."""
    n = ctypes.c_size_t()
    _check(lib().nuna_expert_layer_few_workspace(int(tokens), int(topk), int(hidden), int(inner), ctypes.byref(n)))
    return n.value


def expert_layer_few(x, topk_idx, weights, w1, w1_scale, w2, w2_scale, first_expert=0, out=None, workspace=None,
                     stream=None):
    """A whole expert layer for up to FEW_TOKENS tokens, in two kernels: out[t] = sum over j of weights[t, j] * w2[e] @
    swiglu(w1[e] @ x[t]) for e = topk_idx[t, j] - first_expert in [0, experts); a token with none gets zeros.  x [T, H]
    (contiguous rows), topk_idx int32 and weights float32 [T, k], w1 [experts, 2 * inner, f8_width(H)] and w2 [experts, H,
    f8_width(inner)] with their scales (f8_quantize_blocks).  The tokens are not quantised.  workspace: a uint8 CUDA tensor
    of expert_layer_few_workspace bytes, which calls that may run at the same time do not share."""
    torch = _torch()
    f8 = torch.float8_e4m3fn
    dev = _device_of(x, "x")
    stride = _check_matrix(x, "x", dev)
    T, H = x.shape
    rows, k = _check_table(topk_idx, "topk_idx", dev)
    if rows != T:
        raise ValueError(f"x has {T} rows, topk_idx {rows}")
    wp = _check_weights(weights, T, k, dev)
    if w1.dim() != 3 or w1.shape[1] < 2 or w1.shape[1] % 2:
        raise ValueError("w1 must be [experts, 2 * inner, f8_width(hidden)]")
    E, inner = w1.shape[0], w1.shape[1] // 2
    kind = _scale_kind(w1_scale, "w1_scale")
    _check_tensor(w1, "w1", (E, 2 * inner, f8_width(H)), f8, dev)
    _check_tensor(w2, "w2", (E, H, f8_width(inner)), f8, dev)
    _check_tensor(w1_scale, "w1_scale", (E, -(-2 * inner // F8_BLOCK), f8_pitch(H)), w1_scale.dtype, dev)
    _check_tensor(w2_scale, "w2_scale", (E, -(-H // F8_BLOCK), f8_pitch(inner)), w1_scale.dtype, dev)
    need = expert_layer_few_workspace(T, k, H, inner)
    if out is None:
        out = _new(stream, (T, H), x.dtype, x.device)
    if workspace is None:
        workspace = _new(stream, (need,), torch.uint8, x.device)
    _check_tensor(out, "out", (T, H), x.dtype, dev)
    _check_workspace(workspace, dev)
    _check(lib().nuna_expert_layer_few(x.data_ptr(), stride, topk_idx.data_ptr(), wp, T, k, w1.data_ptr(),
                                       w1_scale.data_ptr(), w2.data_ptr(), w2_scale.data_ptr(), int(first_expert), E, H,
                                       inner, out.data_ptr(), workspace.data_ptr(), workspace.numel(), kind,
                                       _dtype_code(x), _handle(stream, dev)))
    return out


def probe_xcc(G, stream=None):
    """Run the dispatch probe: per workgroup, the XCC id and raw HW_ID it ran on."""
    torch = _torch()
    xcc = torch.full((G,), -1, dtype=torch.int32, device="cuda")
    hw = torch.full((G,), -1, dtype=torch.int32, device="cuda")
    _check(lib().nuna_probe_xcc(G, xcc.data_ptr(), hw.data_ptr(), _stream(stream)))
    return xcc, hw


def _check_flat(ts, name):
    """Each tensor is a contiguous CUDA tensor, so that its data pointer and numel() * element_size() bytes
    span exactly its own storage (an expanded or strided view would span more or other memory)."""
    for t in ts:
        if not t.is_cuda or not t.is_contiguous():
            raise ValueError(f"{name}: buffers must be contiguous CUDA tensors")


def copy(dst, src, stream=None):
    _check_flat((dst, src), "copy")
    nbytes = src.numel() * src.element_size()
    if dst.numel() * dst.element_size() < nbytes:
        raise ValueError("dst too small")
    _check(lib().nuna_copy(dst.data_ptr(), src.data_ptr(), nbytes, _stream(stream)))
    return dst


REF_KINDS = {"read": 0, "write": 1, "copy": 2}


def ref_read_checksum_bytes(n, nbytes):
    """Bytes a reference read of n buffers of nbytes writes to dst[0]: one 16-byte checksum per item of
    max(1, 8 // n) blocks of 4 KiB."""
    item = (1 if n >= 8 else 8 // n) * 4096
    return (nbytes + item - 1) // item * 16


def ref_stream_raw(kind, src_ptrs, dst_ptrs, n, nbytes, stream=0):
    """nuna_ref_stream on raw device addresses (lists of ints or None) and a raw stream handle;
    returns the status code."""
    src = _ptr_array(src_ptrs) if src_ptrs is not None else None
    dst = _ptr_array(dst_ptrs) if dst_ptrs is not None else None
    return lib().nuna_ref_stream(REF_KINDS[kind], src, dst, n, nbytes, stream)


def ref_stream(kind, srcs, dsts, stream=None):
    """Reference stream over CUDA tensors: "read" (srcs; dsts[0] receives ref_read_checksum_bytes of
    checksums), "write" (dsts), or "copy" (dsts[r] = srcs[r]).  Every buffer holds the same number of
    bytes."""
    if kind not in REF_KINDS:
        raise ValueError(f"reference stream kind {kind!r} is not one of {sorted(REF_KINDS)}")
    bufs = dsts if kind == "write" else srcs
    if not bufs or not dsts:
        raise ValueError("reference stream needs its buffers and at least one destination")
    _check_flat(list(bufs) + list(dsts), "ref_stream")
    nbytes = bufs[0].numel() * bufs[0].element_size()
    if any(b.numel() * b.element_size() != nbytes for b in bufs):
        raise ValueError("reference stream buffers differ in size")
    if kind == "read" and dsts[0].numel() * dsts[0].element_size() < ref_read_checksum_bytes(len(srcs), nbytes):
        raise ValueError("checksum buffer too small")
    if kind == "copy" and (len(dsts) != len(srcs) or any(d.numel() * d.element_size() < nbytes for d in dsts)):
        raise ValueError("copy destinations must match the sources")
    n = len(bufs)
    _check(ref_stream_raw(kind, None if kind == "write" else [s.data_ptr() for s in srcs],
                          [d.data_ptr() for d in dsts], n, nbytes, _stream(stream)))
    return dsts


def probe_load_latency(buf, stride, line_offset, xcd, stream=None):
    """Cold-load latency (shader cycles) of each stride-sized block of `buf` (a CUDA tensor) seen from
    XCD `xcd`.  The caller evicts the caches first.  Returns an int64 CPU tensor."""
    torch = _torch()
    _check_flat((buf,), "probe")
    nbytes = buf.numel() * buf.element_size()
    cyc = torch.zeros(nbytes // stride, dtype=torch.int32, device=buf.device)
    _check(lib().nuna_probe_load_latency(buf.data_ptr(), nbytes, stride, line_offset, xcd, cyc.data_ptr(),
                                         _stream(stream)))
    torch.cuda.current_stream().synchronize() if stream is None else stream.synchronize()
    return cyc.cpu().to(torch.int64)


def memory_affinity(buf, stride=8192, line_offset=256, xcds=(0, 4), evict_bytes=1 << 30):
    """Near XCD group of each block of `buf`: probe it cold from one XCD of each group and return
    (latencies [len(xcds), nblocks] int64, near index per block).  Eviction between passes streams
    `evict_bytes` through a scratch tensor (plumbing on the host side of the call)."""
    torch = _torch()
    ev = torch.empty(evict_bytes // 4, dtype=torch.int32, device=buf.device)
    lats = []
    for j, x in enumerate(xcds):
        ev.fill_(j)
        torch.cuda.synchronize()
        lats.append(probe_load_latency(buf, stride, line_offset, x))
    del ev
    lat = torch.stack(lats)
    return lat, lat.argmin(dim=0)


def probe_load_latency_cus(buf, xcd, stride=8192, stream=None):
    """Cold-load latency (shader cycles) of every stride-sized block of `buf` from each compute unit of
    XCD `xcd` it reaches.  Returns (latencies int64 [cus, nblocks] on the CPU, HW_ID CU keys [cus],
    compute units seen).  The caller evicts the caches first."""
    torch = _torch()
    _check_flat((buf,), "probe")
    nbytes = buf.numel() * buf.element_size()
    nb = nbytes // stride
    work = torch.zeros(257, dtype=torch.int32, device=buf.device)
    cyc = torch.zeros((32, nb), dtype=torch.int32, device=buf.device)
    cu = torch.full((32,), -1, dtype=torch.int32, device=buf.device)
    _check(lib().nuna_probe_load_latency_cus(buf.data_ptr(), nbytes, stride, xcd, work.data_ptr(), cyc.data_ptr(),
                                             cu.data_ptr(), _stream(stream)))
    torch.cuda.current_stream().synchronize() if stream is None else stream.synchronize()
    seen = int(work[256].item())
    n = min(seen, 32)
    return cyc[:n].cpu().to(torch.int64), cu[:n].cpu().to(torch.int64), seen


def cu_latency_map(buf, stride=8192, xcds=range(8), evict_bytes=1 << 30):
    """Per-XCD, per-compute-unit cold-load latencies over every block of `buf`: dict xcd ->
    (latencies [cus, nblocks], CU keys, compute units seen).  Caches are evicted before each XCD's
    pass by streaming `evict_bytes` through a scratch tensor (plumbing on the host side)."""
    torch = _torch()
    ev = torch.empty(evict_bytes // 4, dtype=torch.int32, device=buf.device)
    out = {}
    for j, x in enumerate(xcds):
        ev.fill_(j)
        torch.cuda.synchronize()
        out[x] = probe_load_latency_cus(buf, x, stride)
    del ev
    return out
