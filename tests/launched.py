"""Which kernels a call launches: captured into a graph, whose kernel nodes are looked at through the driver (nothing is run)."""

import ctypes

import torch


class _KernelNode(ctypes.Structure):
    _fields_ = [("func", ctypes.c_void_p), ("grid", ctypes.c_uint * 3), ("block", ctypes.c_uint * 3), ("shared", ctypes.c_uint),
                ("params", ctypes.c_void_p), ("extra", ctypes.c_void_p), ("kern", ctypes.c_void_p), ("ctx", ctypes.c_void_p)]


def kernels(call):
    """(name as the linker knows it, grid) of every kernel that `call` launches on the current stream, in the graph's order."""
    driver = ctypes.CDLL("libcuda.so.1")
    graph = torch.cuda.CUDAGraph(keep_graph=True)
    with torch.cuda.graph(graph):
        call()
    raw, n = ctypes.c_void_p(graph.raw_cuda_graph()), ctypes.c_size_t(0)

    def ok(status, what):
        assert status == 0, f"{what}: {status}"

    ok(driver.cuGraphGetNodes(raw, None, ctypes.byref(n)), "cuGraphGetNodes")
    nodes = (ctypes.c_void_p * n.value)()
    ok(driver.cuGraphGetNodes(raw, nodes, ctypes.byref(n)), "cuGraphGetNodes")
    found = []
    for node in nodes:
        kind = ctypes.c_int(-1)
        ok(driver.cuGraphNodeGetType(ctypes.c_void_p(node), ctypes.byref(kind)), "cuGraphNodeGetType")
        if kind.value != 0:                  # (a kernel's)
            continue
        p, name = _KernelNode(), ctypes.c_char_p()
        ok(driver.cuGraphKernelNodeGetParams_v2(ctypes.c_void_p(node), ctypes.byref(p)), "cuGraphKernelNodeGetParams")
        if p.kern:
            ok(driver.cuKernelGetName(ctypes.byref(name), ctypes.c_void_p(p.kern)), "cuKernelGetName")
        else:
            ok(driver.cuFuncGetName(ctypes.byref(name), ctypes.c_void_p(p.func)), "cuFuncGetName")
        found.append((name.value.decode(), tuple(p.grid)))
    return found
