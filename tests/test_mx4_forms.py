"""Which kernel the shapes of the graph and stream tests take (CPU)."""
import ctypes as C

from tests import test_gpu_mx4_graphs as gpu
from tests import test_gpu_mx4_layer as layer
from tests.test_mx4_rules import rules  # noqa: F401  (a fixture)


def test_graph_shapes_take_the_ring(rules):  # noqa: F811
    columns = C.c_bool()
    for tiling, shape in gpu.RING.items():
        assert not rules.few(*shape) and rules.split(*shape, C.byref(columns)) == 0
        assert rules.tiling(*shape) == tiling, (shape, rules.tiling(*shape))
    for way, shape in gpu.SPLIT.items():
        assert not rules.few(*shape) and rules.split(*shape, C.byref(columns)) > 0
        assert columns.value == (way == "columns")


def test_graph_layer_takes_the_ring(rules):  # noqa: F811
    heads = (layer.HQ + 2 * layer.HK) * layer.HD
    for N, K in ((heads, layer.D), (layer.D, layer.HQ * layer.HD), (2 * layer.F, layer.D), (layer.D, layer.F)):
        assert not rules.few(gpu.LAYER_ROWS, N, K)
