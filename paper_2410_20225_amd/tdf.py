"""ctypes binding of include/tdf.h.  Same names as the C entry points, without the prefix.

Tensors are torch tensors on the GPU; the binding passes their data pointers and the current
HIP stream.  No computation happens here.
"""
import ctypes as C
import os

# torch ships its own copy of the HIP runtime; it must be loaded before libtdf.so so that the
# library binds to the same runtime (one context, shared streams) instead of loading a second one
import torch  # noqa: F401

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "libtdf.so")
if not os.path.exists(_LIB_PATH):
    raise ImportError("libtdf.so is not built: run `python -m paper_2410_20225_amd.build` "
                      "(there is no fallback path)")
lib = C.CDLL(_LIB_PATH)

OK, ERR_BAD_PROGRAM, ERR_BAD_ARG, ERR_WORKSPACE, ERR_TABLE_FULL, ERR_STEP_LIMIT, ERR_DEVICE = 0, -1, -2, -3, -4, -5, -6
ERR_UNSUPPORTED = -7
F32, BF16 = 0, 1
(OP_IN, OP_OUT, OP_CONST, OP_ADD, OP_SUB, OP_MUL, OP_EQ, OP_LT, OP_ID, OP_SWITCH, OP_MERGE, OP_CALLFN,
 OP_TREE_ISLEAF, OP_TREE_LEFT, OP_TREE_RIGHT, OP_TREE_TOKEN, OP_EMBED, OP_RNN_CELL, OP_LSTM_CELL,
 OP_CE_HEAD, OP_LOOP, OP_NEXT, OP_CE_NODE) = range(23)
SNODE_MERGE_ENTRY, SNODE_CALL, SNODE_RETURN, SNODE_ENTER, SNODE_NEXT, SNODE_EXIT = 100, 101, 102, 103, 104, 105
MAX_INPUTS = 4
STATS_MAX_COUNTS = 256
TAGS_STEP_MACHINE, TAGS_LANES, TAGS_WALK = range(3)   # Stats.tag_phase
PHASES = ("tags", "leaves", "levels", "cells_fwd", "head", "cells_bwd", "weight_grad", "embed_grad", "tail_fwd", "tail_bwd")


class Ref(C.Structure):
    _fields_ = [("node", C.c_int32), ("port", C.c_int32)]


class NodeDesc(C.Structure):
    _fields_ = [("op", C.c_int32), ("n_in", C.c_int32), ("inp", Ref * MAX_INPUTS), ("imm", C.c_int64)]


class FunctionDesc(C.Structure):
    _fields_ = [("name", C.c_char_p), ("n_params", C.c_int32), ("n_nodes", C.c_int32),
                ("nodes", C.POINTER(NodeDesc))]


class ProgramDesc(C.Structure):
    _fields_ = [("n_functions", C.c_int32), ("functions", C.POINTER(FunctionDesc)), ("result_fn", C.c_int32)]


class SNode(C.Structure):
    _fields_ = [("kind", C.c_int32), ("fn", C.c_int32), ("label", C.c_int32), ("param", C.c_int32),
                ("is_grad", C.c_int32), ("imm", C.c_int64)]


class SEdge(C.Structure):
    _fields_ = [("src", C.c_int32), ("src_port", C.c_int32), ("dst", C.c_int32), ("dst_slot", C.c_int32),
                ("is_control", C.c_int32)]


class GraphInfo(C.Structure):
    _fields_ = [("n_nodes", C.c_int32), ("n_edges", C.c_int32), ("n_labels", C.c_int32),
                ("nodes", C.POINTER(SNode)), ("edges", C.POINTER(SEdge))]


class Inputs(C.Structure):
    _fields_ = [("n_instances", C.c_int32), ("n_args", C.c_int32), ("args", C.c_void_p),
                ("n_tree_nodes", C.c_int32), ("left", C.c_void_p), ("right", C.c_void_p), ("token", C.c_void_p),
                ("node_label", C.c_void_p),
                ("dtype", C.c_int32), ("hidden", C.c_int32), ("vocab", C.c_int32),
                ("E", C.c_void_p), ("W", C.c_void_p), ("b", C.c_void_p),
                ("n_classes", C.c_int32), ("U", C.c_void_p), ("u0", C.c_void_p),
                ("max_tags", C.c_int64), ("step_limit", C.c_int32), ("stats_level", C.c_int32)]


class Outputs(C.Structure):
    _fields_ = [("out_i64", C.c_void_p), ("out_f32", C.c_void_p), ("out_h", C.c_void_p), ("out_c", C.c_void_p),
                ("out_node_loss", C.c_void_p)]


class Seed(C.Structure):
    _fields_ = [("dy", C.c_void_p), ("dnode", C.c_void_p)]


class Grads(C.Structure):
    _fields_ = [("dW", C.c_void_p), ("db", C.c_void_p), ("dE", C.c_void_p)]


class Stats(C.Structure):
    _fields_ = [("n_tags", C.c_int64), ("n_steps", C.c_int64), ("n_tokens", C.c_int64),
                ("n_leaf_rows", C.c_int64), ("n_cell_rows", C.c_int64), ("n_waves", C.c_int64),
                ("n_wide_waves", C.c_int64), ("n_wide_cells", C.c_int64), ("deep_cells", C.c_int64),
                ("n_grad_firings", C.c_int64), ("n_grad_not_once", C.c_int64),
                ("max_tag_depth", C.c_int64), ("table_capacity", C.c_int64),
                ("max_probe", C.c_int64), ("peak_frames", C.c_int64), ("frames_reclaimed", C.c_int64), ("phase_ms", C.c_double * len(PHASES)), ("phase_launches", C.c_int64 * len(PHASES)),
                ("fwd_cells_span_ms", C.c_double), ("wide_step_frames", C.c_int64 * 8), ("wide_step_created", C.c_int64 * 8),
                ("wide_step_us", C.c_double * 8),
                ("device_status", C.c_int32), ("n_counts", C.c_int32),
                ("n_machines", C.c_int32), ("die_local", C.c_int32), ("generated", C.c_int32),
                ("repeats", C.c_int32), ("tail_used", C.c_int32), ("deep_split", C.c_int32),
                ("fire_count", C.c_int64 * STATS_MAX_COUNTS), ("tag_phase", C.c_int32), ("reserved", C.c_int32)]


class Norm(C.Structure):
    _fields_ = [("n_rows", C.c_int64), ("n_cols", C.c_int64), ("dtype", C.c_int32), ("eps", C.c_float), ("x", C.c_void_p), ("ld_x", C.c_int64),
                ("weight", C.c_void_p), ("bias", C.c_void_p)]


class NormGrads(C.Structure):
    _fields_ = [("dy", C.c_void_p), ("ld_dy", C.c_int64), ("mean", C.c_void_p), ("rstd", C.c_void_p), ("dx", C.c_void_p), ("ld_dx", C.c_int64),
                ("dweight", C.c_void_p), ("dbias", C.c_void_p)]


class Scan(C.Structure):
    _fields_ = [("n_rows", C.c_int64), ("n_cols", C.c_int64), ("n_seqs", C.c_int64), ("dtype", C.c_int32), ("f", C.c_void_p), ("ld_f", C.c_int64),
                ("x", C.c_void_p), ("ld_x", C.c_int64), ("offsets", C.c_void_p), ("h0", C.c_void_p)]


class ScanGrads(C.Structure):
    _fields_ = [("h", C.c_void_p), ("ld_h", C.c_int64), ("dh", C.c_void_p), ("ld_dh", C.c_int64), ("dh_last", C.c_void_p),
                ("df", C.c_void_p), ("ld_df", C.c_int64), ("dx", C.c_void_p), ("ld_dx", C.c_int64), ("dh0", C.c_void_p)]


class ScanStep(C.Structure):
    _fields_ = [("n_rows", C.c_int64), ("n_cols", C.c_int64), ("n_states", C.c_int64), ("dtype", C.c_int32), ("f", C.c_void_p), ("ld_f", C.c_int64),
                ("x", C.c_void_p), ("ld_x", C.c_int64), ("slot", C.c_void_p), ("state", C.c_void_p), ("h", C.c_void_p), ("ld_h", C.c_int64)]


class AdamwTensor(C.Structure):
    _fields_ = [("n", C.c_int64), ("param_dtype", C.c_int32), ("grad_dtype", C.c_int32), ("state_bits", C.c_int32), ("weight_decay", C.c_float),
                ("param", C.c_void_p), ("grad", C.c_void_p), ("copy", C.c_void_p), ("m", C.c_void_p), ("v", C.c_void_p),
                ("m_scale", C.c_void_p), ("v_scale", C.c_void_p)]


class AdamwStep(C.Structure):
    _fields_ = [("lr", C.c_double), ("beta1", C.c_double), ("beta2", C.c_double), ("eps", C.c_double), ("step", C.c_int64),
                ("grad_scale", C.c_void_p), ("seed", C.c_uint32), ("reserved", C.c_uint32)]


def _declare(l):
    """Argument and result types of every entry point of a loaded library."""
    l.tdf_graph_build.argtypes = [C.POINTER(ProgramDesc), C.c_int, C.POINTER(C.c_void_p)]
    l.tdf_graph_build.restype = C.c_int
    l.tdf_graph_destroy.argtypes = [C.c_void_p]
    l.tdf_graph_destroy.restype = None
    l.tdf_graph_info.argtypes = [C.c_void_p, C.POINTER(GraphInfo)]
    l.tdf_graph_info.restype = C.c_int
    l.tdf_graph_precompile.argtypes = [C.c_void_p, C.c_char_p, C.POINTER(C.c_size_t)]
    l.tdf_graph_precompile.restype = C.c_int
    l.tdf_workspace_size.argtypes = [C.c_void_p, C.POINTER(Inputs), C.c_int, C.POINTER(C.c_size_t)]
    l.tdf_workspace_size.restype = C.c_int
    l.tdf_eval.argtypes = [C.c_void_p, C.POINTER(Inputs), C.POINTER(Outputs), C.c_void_p, C.c_size_t,
                             C.c_void_p, C.POINTER(Stats)]
    l.tdf_eval.restype = C.c_int
    l.tdf_eval_grad.argtypes = [C.c_void_p, C.POINTER(Inputs), C.POINTER(Seed), C.POINTER(Outputs),
                                  C.POINTER(Grads), C.c_void_p, C.c_size_t, C.c_void_p, C.POINTER(Stats)]
    l.tdf_eval_grad.restype = C.c_int
    l.tdf_graph_prepare.argtypes = [C.c_void_p]
    l.tdf_graph_prepare.restype = C.c_int
    l.tdf_eval_static.argtypes = [C.c_void_p, C.POINTER(Inputs), C.POINTER(Outputs), C.c_void_p, C.POINTER(Stats)]
    l.tdf_eval_static.restype = C.c_int
    l.tdf_last_error.argtypes = []
    l.tdf_last_error.restype = C.c_char_p
    P = C.POINTER
    for name, args in (("layer_norm", [P(Norm), C.c_void_p, C.c_int64, C.c_void_p, C.c_void_p, C.c_void_p]),
                       ("layer_norm_grad_workspace_size", [C.c_int64, C.c_int64, P(C.c_size_t)]),
                       ("layer_norm_grad", [P(Norm), P(NormGrads), C.c_void_p, C.c_size_t, C.c_void_p]),
                       ("gated_scan_workspace_size", [C.c_int64, C.c_int64, P(C.c_size_t)]),
                       ("gated_scan", [P(Scan), C.c_void_p, C.c_int64, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]),
                       ("gated_scan_grad", [P(Scan), P(ScanGrads), C.c_void_p, C.c_size_t, C.c_void_p]),
                       ("gated_scan_step", [P(ScanStep), C.c_void_p]),
                       ("adamw_build", [P(AdamwTensor), C.c_int64, P(C.c_void_p)]),
                       ("adamw_workspace_size", [C.c_void_p, P(C.c_size_t)]),
                       ("adamw_prepare", [C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]),
                       ("adamw", [C.c_void_p, P(AdamwStep), C.c_void_p])):
        f = getattr(l, "tdf_" + name)
        f.argtypes, f.restype = args, C.c_int
    l.tdf_adamw_destroy.argtypes, l.tdf_adamw_destroy.restype = [C.c_void_p], None
    return l


def load_library(path):
    """Another build of the library (the tests load the one with the test hooks compiled in); a graph
    built while it is current (use_library) keeps calling it."""
    return _declare(C.CDLL(path))


class use_library:
    """with use_library(l): graph_build and last_error go to `l` instead of the default library."""

    def __init__(self, l):
        self.l = l

    def __enter__(self):
        global lib
        self.prev, lib = lib, self.l
        return self.l

    def __exit__(self, *exc):
        global lib
        lib = self.prev


_declare(lib)
STATIC_WORKSPACE_BYTES = 64 << 20


class TdfError(RuntimeError):
    def __init__(self, status, where):
        self.status = status
        msg = lib.tdf_last_error()
        super().__init__("%s failed with status %d: %s" % (where, status, msg.decode() if msg else ""))


def last_error():
    msg = lib.tdf_last_error()
    return msg.decode() if msg else ""


def _ptr(t):
    return None if t is None else C.c_void_p(t.data_ptr())


class Graph:
    """Owns a tdf_graph*; destroyed with the object."""

    def __init__(self, handle, library):
        self.handle = handle
        self.lib = library      # the library that built the graph serves every later call on it

    def __del__(self):
        if getattr(self, "handle", None) and getattr(self, "lib", None) is not None and C is not None:
            self.lib.tdf_graph_destroy(self.handle)
            self.handle = None


def graph_build(functions, result_fn, want_grad=False):
    """functions: list of (name, n_params, [(op, [(node, port), ...], imm), ...])."""
    keep = []
    fdescs = (FunctionDesc * len(functions))()
    for i, (name, n_params, nodes) in enumerate(functions):
        arr = (NodeDesc * max(len(nodes), 1))()
        for j, (op, ins, imm) in enumerate(nodes):
            arr[j].op, arr[j].n_in, arr[j].imm = op, len(ins), imm
            for k, (n, p) in enumerate(ins[:MAX_INPUTS]):
                arr[j].inp[k].node, arr[j].inp[k].port = n, p
        keep.append(arr)
        fdescs[i].name, fdescs[i].n_params, fdescs[i].n_nodes = name.encode(), n_params, len(nodes)
        fdescs[i].nodes = C.cast(arr, C.POINTER(NodeDesc))
    prog = ProgramDesc(len(functions), C.cast(fdescs, C.POINTER(FunctionDesc)), result_fn)
    handle = C.c_void_p()
    st = lib.tdf_graph_build(C.byref(prog), int(bool(want_grad)), C.byref(handle))
    if st != OK:
        raise TdfError(st, "tdf_graph_build")
    return Graph(handle, lib)


def graph_info(graph):
    info = GraphInfo()
    st = graph.lib.tdf_graph_info(graph.handle, C.byref(info))
    if st != OK:
        raise TdfError(st, "tdf_graph_info")
    nodes = [dict(kind=n.kind, fn=n.fn, label=n.label, param=n.param, is_grad=n.is_grad, imm=n.imm)
             for n in (info.nodes[i] for i in range(info.n_nodes))]
    edges = [dict(src=e.src, src_port=e.src_port, dst=e.dst, dst_slot=e.dst_slot, is_control=e.is_control)
             for e in (info.edges[i] for i in range(info.n_edges))]
    return dict(nodes=nodes, edges=edges, n_labels=info.n_labels)


def graph_precompile(graph, arch="gfx950"):
    """Compiles the specialised step kernels of `graph` for `arch`; returns the code size in bytes."""
    n = C.c_size_t()
    st = graph.lib.tdf_graph_precompile(graph.handle, arch.encode(), C.byref(n))
    if st != OK:
        raise TdfError(st, "tdf_graph_precompile")
    return n.value


def make_inputs(n_instances, args=None, n_args=0, left=None, right=None, token=None, dtype=F32, hidden=0,
                vocab=0, E=None, W=None, b=None, U=None, u0=None, n_classes=0, max_tags=0, step_limit=0, stats_level=1,
                node_label=None):
    n_tree = 0 if left is None else int(left.numel())
    return Inputs(n_instances, n_args, _ptr(args), n_tree, _ptr(left), _ptr(right), _ptr(token), _ptr(node_label), dtype, hidden,
                  vocab, _ptr(E), _ptr(W), _ptr(b), n_classes, _ptr(U), _ptr(u0), max_tags, step_limit, stats_level)


def workspace_size(graph, inputs, with_grad=False):
    n = C.c_size_t()
    st = graph.lib.tdf_workspace_size(graph.handle, C.byref(inputs), int(bool(with_grad)), C.byref(n))
    if st != OK:
        raise TdfError(st, "tdf_workspace_size")
    return n.value


def _stream():
    return C.c_void_p(torch.cuda.current_stream().cuda_stream)


def eval(graph, inputs, workspace, out_i64=None, out_f32=None, out_h=None, out_c=None, out_node_loss=None, check=True):
    """Returns (status, Stats)."""
    outs = Outputs(_ptr(out_i64), _ptr(out_f32), _ptr(out_h), _ptr(out_c), _ptr(out_node_loss))
    stats = Stats()
    st = graph.lib.tdf_eval(graph.handle, C.byref(inputs), C.byref(outs), _ptr(workspace),
                      workspace.numel() * workspace.element_size(), _stream(), C.byref(stats))
    if check and st != OK:
        raise TdfError(st, "tdf_eval")
    return st, stats


def graph_prepare(graph):
    st = graph.lib.tdf_graph_prepare(graph.handle)
    if st != OK:
        raise TdfError(st, "tdf_graph_prepare")


def eval_static(graph, inputs, out_i64=None, out_f32=None, out_h=None, out_c=None, out_node_loss=None, check=True):
    """tdf_eval in the library's static workspace (no allocation).  Returns (status, Stats)."""
    outs = Outputs(_ptr(out_i64), _ptr(out_f32), _ptr(out_h), _ptr(out_c), _ptr(out_node_loss))
    stats = Stats()
    st = graph.lib.tdf_eval_static(graph.handle, C.byref(inputs), C.byref(outs), _stream(), C.byref(stats))
    if check and st != OK:
        raise TdfError(st, "tdf_eval_static")
    return st, stats


def eval_grad(graph, inputs, dy, workspace, dW, db, dE, out_f32=None, out_h=None, out_c=None, out_node_loss=None,
              dnode=None, check=True):
    outs = Outputs(None, _ptr(out_f32), _ptr(out_h), _ptr(out_c), _ptr(out_node_loss))
    seed = Seed(_ptr(dy), _ptr(dnode))
    grads = Grads(_ptr(dW), _ptr(db), _ptr(dE))
    stats = Stats()
    st = graph.lib.tdf_eval_grad(graph.handle, C.byref(inputs), C.byref(seed), C.byref(outs), C.byref(grads),
                           _ptr(workspace), workspace.numel() * workspace.element_size(), _stream(),
                           C.byref(stats))
    if check and st != OK:
        raise TdfError(st, "tdf_eval_grad")
    return st, stats


# ---- operators beside the evaluations ---------------------------------------------------------
# These enqueue on the current stream and return.  Tensors are checked here for what the library cannot see (device, type,
# shape), everything else there.
_DTYPES = {torch.float32: F32, torch.bfloat16: BF16}


def _first(t, name):
    """(pointer, distance between rows, shape, type, GPU) of a call's first matrix, which the others are compared with."""
    if t.dim() != 2 or not t.is_cuda or t.dtype not in _DTYPES:
        raise ValueError("%s: a matrix of float32 or bfloat16 on the GPU is wanted, not %s %s on %s" % (name, tuple(t.shape), t.dtype, t.device))
    shape, dtype, device = t.shape, t.dtype, t.get_device()
    return (*_matrix(t, name, shape, dtype, device), shape, dtype, device)


def _matrix(t, name, shape, dtype, device):
    """(pointer, distance between rows) of a matrix whose rows are contiguous.  (On the CPU get_device() is -1.)"""
    if t.dtype is dtype and t.get_device() == device and t.shape == shape:
        rows, cols = shape
        along, inner = t.stride()
        if (inner == 1 or cols <= 1) and (along >= cols or rows <= 1):
            return t.data_ptr(), along if along > cols else cols
        raise ValueError("%s: rows are contiguous and do not overlap, strides %s do not fit" % (name, (along, inner)))
    raise ValueError("%s: a matrix like the first (%s %s) on GPU %d is wanted, not %s %s on %s" % (name, tuple(shape), dtype, device, tuple(t.shape), t.dtype, t.device))


def _vector(t, name, shape, device, dtype=torch.float32):
    """Pointer of a contiguous tensor on the matrix's GPU, None for None."""
    if t is None:
        return None
    if t.dtype is dtype and t.get_device() == device and t.shape == shape and t.is_contiguous():
        return t.data_ptr()
    raise ValueError("%s: a contiguous %s %s on GPU %d is wanted, not %s %s on %s" % (name, dtype, tuple(shape), device, tuple(t.shape), t.dtype, t.device))


def _bytes(t, device):
    if t is None:
        return None, 0
    if t.get_device() != device or not t.is_contiguous():
        raise ValueError("workspace: a contiguous tensor on GPU %d is wanted" % device)
    return t.data_ptr(), t.nbytes


def _stream_of(device):
    """The current stream of the tensors' GPU, which has to be the current one."""
    if device != torch._C._cuda_getDevice():
        raise ValueError("the tensors are on GPU %d, the current device is %d" % (device, torch.cuda.current_device()))
    return torch._C._cuda_getCurrentRawStream(device)


def _done(status, where):
    if status != OK:
        raise TdfError(status, where)


def _size(fn, where, *args):
    n = C.c_size_t()
    _done(fn(*args, C.byref(n)), where)
    return n.value


def layer_norm(x, y, weight=None, bias=None, eps=1e-5, mean=None, rstd=None):
    """y = (x - mean) * rstd * weight + bias over the rows of x; y may be x.  mean and rstd, where given, receive the statistics."""
    px, ld_x, (rows, cols), dtype, gpu = _first(x, "x")
    py, ld_y = _matrix(y, "y", (rows, cols), dtype, gpu)
    in_ = Norm(rows, cols, _DTYPES[dtype], eps, px, ld_x, _vector(weight, "weight", (cols,), gpu), _vector(bias, "bias", (cols,), gpu))
    _done(lib.tdf_layer_norm(in_, py, ld_y, _vector(mean, "mean", (rows,), gpu), _vector(rstd, "rstd", (rows,), gpu), _stream_of(gpu)), "tdf_layer_norm")


def layer_norm_grad_workspace_size(n_rows, n_cols):
    return _size(lib.tdf_layer_norm_grad_workspace_size, "tdf_layer_norm_grad_workspace_size", n_rows, n_cols)


def layer_norm_grad(x, dy, mean, rstd, dx, dweight, dbias, workspace, weight=None):
    """Gradients of layer_norm; each of dx, dweight and dbias may be None.  dx may be dy."""
    px, ld_x, shape, dtype, gpu = _first(x, "x")
    pdy, ld_dy = _matrix(dy, "dy", shape, dtype, gpu)
    pdx, ld_dx = (None, 0) if dx is None else _matrix(dx, "dx", shape, dtype, gpu)
    rows, cols = shape
    in_ = Norm(rows, cols, _DTYPES[dtype], 0.0, px, ld_x, _vector(weight, "weight", (cols,), gpu), None)
    grads = NormGrads(pdy, ld_dy, _vector(mean, "mean", (rows,), gpu), _vector(rstd, "rstd", (rows,), gpu), pdx, ld_dx,
                      _vector(dweight, "dweight", (cols,), gpu), _vector(dbias, "dbias", (cols,), gpu))
    _done(lib.tdf_layer_norm_grad(in_, grads, *_bytes(workspace, gpu), _stream_of(gpu)), "tdf_layer_norm_grad")


def gated_scan_workspace_size(n_rows, n_cols):
    return _size(lib.tdf_gated_scan_workspace_size, "tdf_gated_scan_workspace_size", n_rows, n_cols)


def _scan(f, x, offsets, h0):
    pf, ld_f, shape, dtype, gpu = _first(f, "f")
    px, ld_x = _matrix(x, "x", shape, dtype, gpu)
    rows, cols = shape
    if offsets is not None and (offsets.dim() != 1 or offsets.numel() < 2):
        raise ValueError("offsets: a vector of the sequences' first rows and the last one's end is wanted")
    seqs = 1 if offsets is None else offsets.numel() - 1
    return Scan(rows, cols, seqs, _DTYPES[dtype], pf, ld_f, px, ld_x, _vector(offsets, "offsets", (seqs + 1,), gpu, torch.int64),
                _vector(h0, "h0", (seqs, cols), gpu)), (shape, dtype, gpu), (seqs, cols)


def gated_scan(f, x, h, workspace, offsets=None, h0=None, h_last=None):
    """h_t = sigmoid(f_t) h_(t-1) + (1 - sigmoid(f_t)) x_t over the rows offsets[s] .. offsets[s + 1] - 1 of every sequence s (offsets None:
    one sequence of all rows), from the state h0[s]; h_last[s] receives the state after the last row.  A state that is carried from
    call to call has two buffers: h_last that overlaps h0 is refused, as is dh0 that overlaps dh_last or h0 in gated_scan_grad."""
    in_, like, state = _scan(f, x, offsets, h0)
    gpu = like[2]
    ph, ld_h = _matrix(h, "h", *like)
    _done(lib.tdf_gated_scan(in_, ph, ld_h, _vector(h_last, "h_last", state, gpu), *_bytes(workspace, gpu), _stream_of(gpu)), "tdf_gated_scan")


def gated_scan_grad(f, x, h, dh, df, dx, workspace, offsets=None, h0=None, dh_last=None, dh0=None):
    """Gradients of gated_scan with respect to f, x and h0 from those of h (dh, None: zeros) and h_last (dh_last)."""
    in_, like, state = _scan(f, x, offsets, h0)
    gpu = like[2]
    grads = ScanGrads(*_matrix(h, "h", *like), *((None, 0) if dh is None else _matrix(dh, "dh", *like)), _vector(dh_last, "dh_last", state, gpu),
                      *_matrix(df, "df", *like), *_matrix(dx, "dx", *like), _vector(dh0, "dh0", state, gpu))
    _done(lib.tdf_gated_scan_grad(in_, grads, *_bytes(workspace, gpu), _stream_of(gpu)), "tdf_gated_scan_grad")


def gated_scan_step(f, x, state, h=None, slot=None):
    """One row of many sequences: state[slot[r]] (slot None: state[r]) becomes its next state, which row r of h receives too."""
    pf, ld_f, shape, dtype, gpu = _first(f, "f")
    px, ld_x = _matrix(x, "x", shape, dtype, gpu)
    ph, ld_h = (None, 0) if h is None else _matrix(h, "h", shape, dtype, gpu)
    rows, cols = shape
    states = state.shape[0]
    in_ = ScanStep(rows, cols, states, _DTYPES[dtype], pf, ld_f, px, ld_x, _vector(slot, "slot", (rows,), gpu, torch.int32),
                   _vector(state, "state", (states, cols), gpu), ph, ld_h)
    _done(lib.tdf_gated_scan_step(in_, _stream_of(gpu)), "tdf_gated_scan_step")


def adamw_tensor(param, grad, m, v, m_scale=None, v_scale=None, copy=None, weight_decay=0.0):
    """One tensor of adamw_build.  m and v: float32 like param, or int8 and uint8 with m_scale and v_scale, a float32 for every
    128 elements.  copy: a bfloat16 tensor that receives the float32 param rounded."""
    return dict(param=param, grad=grad, m=m, v=v, m_scale=m_scale, v_scale=v_scale, copy=copy, weight_decay=weight_decay)


class AdamwPlan:
    """Owns a tdf_adamw_plan* and keeps its tensors; destroyed with the object."""

    def __init__(self, handle, library, tensors):
        self.handle, self.lib, self.tensors, self.workspace = handle, library, tensors, None
        self.gpu = tensors[0]["param"].get_device()

    def __del__(self):
        if getattr(self, "handle", None) and getattr(self, "lib", None) is not None and C is not None:
            self.lib.tdf_adamw_destroy(self.handle)
            self.handle = None


def adamw_build(tensors):
    """tensors: a list of adamw_tensor(...).  The plan holds their addresses: build another one for other tensors."""
    arr = (AdamwTensor * max(len(tensors), 1))()
    for k, t in enumerate(tensors):
        p = t["param"]
        n, bits = p.numel(), 32 if t["m"].dtype == torch.float32 else 8
        scales = ((n + 127) // 128,)
        for name, dtypes, numel in (("param", _DTYPES, n), ("grad", _DTYPES, n), ("copy", (torch.bfloat16,), n),
                                    ("m", (torch.float32,) if bits == 32 else (torch.int8,), n), ("v", (torch.float32,) if bits == 32 else (torch.uint8,), n),
                                    ("m_scale", (torch.float32,), scales[0]), ("v_scale", (torch.float32,), scales[0])):
            x = t[name]
            if x is None and name in ("copy", "m_scale", "v_scale"):
                continue
            if x.dtype not in dtypes or x.numel() != numel or not x.is_contiguous() or not x.is_cuda or x.device != tensors[0]["param"].device:
                raise ValueError("tensor %d, %s: %d contiguous elements on the parameter's GPU are wanted, not %s %s on %s" % (
                    k, name, numel, tuple(x.shape), x.dtype, x.device))
        a = arr[k]
        a.n, a.param_dtype, a.grad_dtype, a.state_bits, a.weight_decay = n, _DTYPES[p.dtype], _DTYPES[t["grad"].dtype], bits, t["weight_decay"]
        for name in ("param", "grad", "copy", "m", "v", "m_scale", "v_scale"):
            setattr(a, name, None if t[name] is None or t[name].numel() == 0 else t[name].data_ptr())
    handle = C.c_void_p()
    _done(lib.tdf_adamw_build(arr, len(tensors), C.byref(handle)), "tdf_adamw_build")
    return AdamwPlan(handle, lib, list(tensors))


def adamw_workspace_size(plan):
    return _size(plan.lib.tdf_adamw_workspace_size, "tdf_adamw_workspace_size", plan.handle)


def adamw_prepare(plan, workspace):
    """Lays the plan out in the workspace, which belongs to it from then on (set-up call)."""
    _done(plan.lib.tdf_adamw_prepare(plan.handle, *_bytes(workspace, plan.gpu), _stream_of(plan.gpu)), "tdf_adamw_prepare")
    plan.workspace = workspace


def adamw(plan, step, lr, beta1=0.9, beta2=0.999, eps=1e-8, seed=None, grad_scale=None):
    """One AdamW step over the plan's tensors, the step-th (from 1).  seed: of the random rounding of 8-bit states, another one in
    every step (with the same one an element is rounded to the same side every time, and 8-bit states drift); None: the step.
    grad_scale: a float32 on the GPU that the gradients are multiplied by.  Recorded into a graph, a replay repeats the same step,
    learning rate and seed."""
    in_ = AdamwStep(lr, beta1, beta2, eps, step, None if grad_scale is None else _vector(grad_scale.reshape(1), "grad_scale", (1,), plan.gpu),
                    step if seed is None else seed, 0)
    _done(plan.lib.tdf_adamw(plan.handle, in_, _stream_of(plan.gpu)), "tdf_adamw")
