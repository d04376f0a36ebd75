"""The kernels that a call launches, with their grids: read from a graph that captures it."""
import ctypes

import torch


class _KernelNode(ctypes.Structure):        # CUDA_KERNEL_NODE_PARAMS of the driver API
    _fields_ = [("func", ctypes.c_void_p), ("grid", ctypes.c_uint * 3), ("block", ctypes.c_uint * 3), ("shared", ctypes.c_uint), ("params", ctypes.c_void_p),
                ("extra", ctypes.c_void_p), ("kern", ctypes.c_void_p), ("ctx", ctypes.c_void_p)]


def launches(call):
    """[(name, grid)] of the kernels of ``call()``, in no order.  The call is made once before it is captured; the graph is not run."""
    cu = ctypes.CDLL("libcuda.so.1")

    def ok(status):
        assert status == 0, f"driver call returned {status}"
    call()
    graph = torch.cuda.CUDAGraph(keep_graph=True)
    with torch.cuda.graph(graph):
        call()
    raw, n = ctypes.c_void_p(graph.raw_cuda_graph()), ctypes.c_size_t(0)
    ok(cu.cuGraphGetNodes(raw, None, ctypes.byref(n)))
    nodes = (ctypes.c_void_p * n.value)()
    ok(cu.cuGraphGetNodes(raw, nodes, ctypes.byref(n)))
    out = []
    for node in nodes:
        kind, p, name = ctypes.c_int(-1), _KernelNode(), ctypes.c_char_p()
        ok(cu.cuGraphNodeGetType(ctypes.c_void_p(node), ctypes.byref(kind)))
        if kind.value != 0:         # CU_GRAPH_NODE_TYPE_KERNEL
            continue
        ok(cu.cuGraphKernelNodeGetParams_v2(ctypes.c_void_p(node), ctypes.byref(p)))
        if p.kern:
            ok(cu.cuKernelGetName(ctypes.byref(name), ctypes.c_void_p(p.kern)))
        else:
            ok(cu.cuFuncGetName(ctypes.byref(name), ctypes.c_void_p(p.func)))
        out.append((name.value.decode(), tuple(p.grid)))
    return out
