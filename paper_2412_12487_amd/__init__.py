"""MI355X timeline composer of Echo (arXiv 2412.12487): HIP kernels behind a C ABI.

    from paper_2412_12487_amd import Graph, scenarios_to_device
    g = Graph(graph_arrays, device=0)          # echo_load_graph
    d_scen, n = scenarios_to_device(scen)      # echo_scenario records on the GPU
    out = g.compose(d_scen, n, n_refine=1)     # echo_compose_batch

and the operators of the simulated training steps (`ops`, include/echo_ops.h), which need torch:

    layer_norm, layer_norm_grad, embedding, embedding_grad, cross_entropy, cross_entropy_grad
"""
from .echo import (ECHO_ERR_ARG, ECHO_ERR_CYCLE, ECHO_ERR_DEVICE, ECHO_ERR_HIP, ECHO_ERR_MATCH,
                   ECHO_ERR_NOMEM, ECHO_ERR_RANGE, ECHO_OK, EXPORTS, LIB_PATH, SCENARIO_DTYPE, EchoError,
                   Graph, lib, pack_scenarios, scenarios_to_device)

_OPS = ("layer_norm", "layer_norm_grad", "embedding", "embedding_grad", "cross_entropy", "cross_entropy_grad")

__all__ = ["Graph", "EchoError", "lib", "pack_scenarios", "scenarios_to_device", "SCENARIO_DTYPE",
           "LIB_PATH", "EXPORTS", "ECHO_OK", "ECHO_ERR_ARG", "ECHO_ERR_RANGE", "ECHO_ERR_MATCH",
           "ECHO_ERR_CYCLE", "ECHO_ERR_NOMEM", "ECHO_ERR_HIP", "ECHO_ERR_DEVICE", *_OPS]


def __getattr__(name):
    # the operators' module imports torch, which the package otherwise only needs to load its library
    if name in _OPS or name == "ops":
        from importlib import import_module

        ops = import_module(".ops", __name__)
        globals().update({n: getattr(ops, n) for n in _OPS}, ops=ops)
        return globals()[name]
    raise AttributeError(f"module {__name__!r} has no attribute {name!r}")
