"""CPU checks of UNet.capture (paper_2512_08888_amd/unet.py): a recorded step holds addresses of the optimizer's memory, so the
network keeps the optimizer for as long as it keeps the graph.  The recording itself is replaced: no device is touched."""
import contextlib
import gc
import types
import weakref

import pytest

from paper_2512_08888_amd import unet


class Optimizer:
    pass


def network(recording=contextlib.nullcontext):
    net = unet.UNet.__new__(unet.UNet)
    cuda = types.SimpleNamespace(synchronize=lambda: None, CUDAGraph=type("Graph", (), {}), graph=lambda g: recording())
    net.trace, net.torch = None, types.SimpleNamespace(cuda=cuda)
    net.step = lambda: None
    net.train_step = lambda optimizer, max_norm: None
    return net


def test_a_recorded_step_keeps_its_optimizer():
    net, first, second = network(), Optimizer(), Optimizer()
    refs = weakref.ref(first), weakref.ref(second)
    net.capture(first, max_norm=1.0)
    del first
    gc.collect()
    assert refs[0]() is not None
    net.capture(second)                  # the graph that needed the first is gone
    del second
    gc.collect()
    assert refs[0]() is None and refs[1]() is not None
    net.capture()
    gc.collect()
    assert refs[1]() is None


def test_a_recording_that_fails_leaves_the_one_before():
    net, kept, failed = network(), Optimizer(), Optimizer()
    graph = net.capture(kept, max_norm=1.0)

    @contextlib.contextmanager
    def broken():
        raise RuntimeError("not recorded")
        yield

    net.torch.cuda.graph = lambda g: broken()
    refs = weakref.ref(kept), weakref.ref(failed)
    with pytest.raises(RuntimeError, match="not recorded"):
        net.capture(failed)
    del kept, failed
    gc.collect()
    assert net._graph is graph and refs[0]() is not None and refs[1]() is None
