"""The extension module that calls the training step's entry points: what it refuses before the library sees it
(no GPU; a refused call launches nothing)."""
import ctypes

import pytest

import paper_2609_38767_gb300 as tda
from paper_2609_38767_gb300 import build as tbuild


@pytest.fixture(scope="module", autouse=True)
def libs():
    return tbuild.build()


def forward(L, ws=None, wsb=0):
    tda.tda_linear_forward(L, 256, 64, 4, 256, 64, None, None, 0, 256, 32, None, 0, ws, wsb, stream=0)


def backward(L, ws=256, wsb=1 << 20):
    tda.tda_linear_backward(L, 256, 32, 256, 32, 4, 256, 64, 256, 64, 256, 32, 256, 64, 256, 64, 256, tda.TDA_F32, 0.0, ws,
                            wsb, stream=0)


@pytest.mark.parametrize("call", [forward, backward])
def test_the_layer_is_a_linear_descriptor(call):
    """Any other object with a buffer would be read by the descriptor's layout, past its end where it is short."""
    good = tda.LinearDesc(64, 32, tda.TDA_ACT_SILU, tda.TDA_F64)
    with pytest.raises(tda.TdaError):  # reaches the library, which refuses the type
        call(good)
    for other in (b"", b"short", bytes(good), bytearray(24), tda.LayerDesc(64, 32, 8, 4, 4), memoryview(good),
                  (ctypes.c_int64 * 3)(64, 32, 0), tda.TensorRef()):
        with pytest.raises(TypeError):
            call(other)


def test_workspace_sizes_are_not_negative():
    """-1 would reach the library as the largest size there is and pass its check of the workspace."""
    L = tda.LinearDesc(64, 32, tda.TDA_ACT_SILU, tda.TDA_F64)  # refused by the library if it gets there
    refs = (tda.TensorRef * 1)(tda.TensorRef(256, 256, 4, tda.TDA_F64, 0))
    for call in (lambda b: forward(L, 256, b), lambda b: backward(L, 256, b),
                 lambda b: tda.tda_embedding_backward(tda.TDA_F64, 256, 8, 4, 8, tda.TDA_I32, 256, 3, 1.0, tda.TDA_F32, 256,
                                                      8, 0.0, 256, b, stream=0),
                 lambda b: tda.tda_grad_clip(refs, 1, 1.0, 256, 256, b, stream=0)):
        for b in (-1, -(1 << 40)):
            with pytest.raises(OverflowError):
                call(b)
        with pytest.raises(tda.TdaError):
            call(1 << 20)


def test_other_threads_run_during_a_call():
    """The calls give up Python's lock, as ctypes does. In the library's place stands libc's usleep, which takes the first
    argument as microseconds."""
    import threading
    import time

    mod = tda._train()
    usleep = ctypes.cast(ctypes.CDLL(None).usleep, ctypes.c_void_p).value
    ticks, stop = [], threading.Event()

    def beat():
        while not stop.is_set():
            ticks.append(time.monotonic())
            time.sleep(0.005)

    try:
        mod.bind(tda._current_stream, tda.LinearDesc, *[usleep] * 5)
        t = threading.Thread(target=beat)
        t.start()
        t0 = time.monotonic()
        st = mod.embedding_forward(300_000, 256, 8, 4, 8, tda.TDA_I32, 256, 3, 1.0, 256, 8, 0)
        t1 = time.monotonic()
        stop.set()
        t.join()
    finally:
        tda._calls = None
        tda._train()
    assert st == 0 and t1 - t0 >= 0.25
    assert sum(t0 + 0.02 < x < t1 - 0.02 for x in ticks) >= 5


@pytest.mark.parametrize("dtype,width", [(tda.TDA_F32, 128), (tda.TDA_BF16, 256)])
def test_bias_gradient_scratch_is_one_wave_of_partial_sums(dtype, width):
    """The factor's launch makes a row of partial sums per run of tokens, over blocks of 32 lanes x 16 bytes of columns: at
    most four CTAs for each of 152 SMs in all, unless the columns alone make more."""
    up256 = lambda x: (x + 255) // 256 * 256
    for M, do in ((8192, 8192), (4096, 2048), (3000, 1000), (100000, 128), (8192, 80000), (33, 64)):
        L = tda.LinearDesc(64, do, tda.TDA_ACT_SILU, dtype)
        total = tda.tda_linear_workspace_size(tda.TDA_LINEAR_BACKWARD, L, M)
        planes = sum(up256(6 * r * c) for r, c in ((M, 64), (do, 64), (M, do))) if dtype == tda.TDA_F32 else 0
        blocks = -(-do // width)
        runs = (total - planes) // (4 * do)
        assert runs >= 1 and (runs == 1 or runs * blocks <= 4 * 152), (M, do, runs)
        # and no fewer than that allows, down to 32 tokens a run
        most = min(256, max(1, 4 * 152 // blocks))
        run = max(32, -(-M // most))
        assert up256(4 * -(-M // run) * do) == total - planes


def test_workspace_sizes_do_not_wrap():
    """Sizes whose scratch passes 64 bits are refused, not answered with what is left of it."""
    big = (1 << 31) - 8
    for dtype in (tda.TDA_BF16, tda.TDA_F32):
        for di, do, M in ((big, big, big), (big, 8, big), (1, big, big), (big, big, 1)):
            for op in (tda.TDA_LINEAR_FORWARD, tda.TDA_LINEAR_BACKWARD, tda.TDA_LINEAR_BACKWARD | tda.TDA_LINEAR_ANY_STRIDE):
                with pytest.raises(tda.TdaError) as e:
                    tda.tda_linear_workspace_size(op, tda.LinearDesc(di, do, 0, dtype), M)
                assert e.value.status == tda.TDA_ERR_INVALID_ARG
        # the largest that fit: three planes of fp32, every matrix of 2^46 elements at most
        L = tda.LinearDesc(1 << 23, 1 << 23, 0, dtype)
        size = tda.tda_linear_workspace_size(tda.TDA_LINEAR_BACKWARD | tda.TDA_LINEAR_ANY_STRIDE, L, 1 << 23)
        assert size >= 3 * (1 << 46) * (6 if dtype == tda.TDA_F32 else 2)
    assert tda.tda_embedding_workspace_size(10, 1 << 62, 1000) == 0 and tda.tda_embedding_workspace_size(10, 1 << 23, 5) == 0
    assert tda.tda_embedding_workspace_size(1 << 40, 8, 1000) == 0 and tda.tda_embedding_workspace_size(10, 1 << 22, 5) > 0
    assert tda.tda_grad_clip_workspace_size(None, 1 << 62) == 0 and tda.tda_grad_clip_workspace_size(None, 1 << 20) > 0


def test_the_first_bad_argument_is_the_error():
    """Tensors after an argument that does not convert: its own error comes out, and none of their code runs before."""
    import torch

    t = torch.zeros(8)

    class Touched:
        def data_ptr(self):
            raise AssertionError("called after an error")

        __index__ = __float__ = data_ptr

        @property
        def cuda_stream(self):
            raise AssertionError("read after an error")

    def lookup(ld_e=8, E=t, out=t, n=3, scale=1.0, stream=0):
        tda.tda_embedding_forward(tda.TDA_F64, E, ld_e, 4, 8, tda.TDA_I32, t, n, scale, out, 8, stream=stream)

    for bad in (dict(ld_e=1.5), dict(ld_e="x"), dict(E="x"), dict(ld_e=1 << 70), dict(scale="a")):
        for later in (dict(), dict(out=Touched()), dict(stream=Touched())) + ((dict(n=Touched()),) if "scale" not in bad else ()):
            with pytest.raises((TypeError, AttributeError, OverflowError)):
                lookup(**bad, **later)
    with pytest.raises(TypeError):
        tda.tda_linear_forward(b"short", t, 64, 1, t, 64, None, None, 0, t, 32, stream=0)
    with pytest.raises(tda.TdaError):  # every argument converts: the library refuses the type
        lookup()
