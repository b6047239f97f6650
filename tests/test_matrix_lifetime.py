"""A described 4-bit or 8-bit matrix keeps its codes and scales until its kernel-native
copy is made, and no longer."""
import contextlib
import weakref

import numpy as np
import pytest

from test_abi import ss  # noqa: F401  (fixture: the built library)

torch = pytest.importorskip("torch")


def described(ss, kind, device):  # noqa: F811
    """The matrix, its tensors, and the calls that describe and pack it."""
    rng = np.random.default_rng(4)
    new = lambda a: torch.from_numpy(a).to(device)  # noqa: E731
    if kind == "mx4":
        t = new(rng.integers(0, 256, (3, 64, 128), dtype=np.uint8)), new(rng.integers(120, 130, (3, 64, 8), dtype=np.uint8))
        return t, ss.make_mx4, ss.prepack_mx4
    t = new(rng.integers(0, 127, (3, 64, 256), dtype=np.uint8)), new(rng.random((3, 1, 2), dtype=np.float32))
    return t, ss.make_fp8, ss.prepack_fp8


@pytest.mark.parametrize("kind", ["mx4", "fp8"])
def test_tensors_are_held_until_packed(ss, monkeypatch, kind):  # noqa: F811
    monkeypatch.setattr(ss, "_same_device", lambda *a: 0)
    monkeypatch.setattr(ss, "_run", lambda where, *a: None)
    t, make, prepack = described(ss, kind, "cpu")
    W = make(*t)
    refs = [weakref.ref(v) for v in t]
    del t
    assert all(r() is not None for r in refs)
    packed = prepack(W, device="cpu")
    assert W.packed == packed.data_ptr()
    assert all(r() is None for r in refs)
    # a matrix described with its copy needs nothing else
    t, make, prepack = described(ss, kind, "cpu")
    W = make(*t, packed=packed)
    refs = [weakref.ref(v) for v in t]
    del t
    assert all(r() is None for r in refs)


def test_the_allocator_hears_of_tensors_that_go(ss, monkeypatch):  # noqa: F811
    """Only of those that nothing else holds: another holder's own streams are its own
    business, and a stream noted for a long-lived tensor is waited for when that is freed."""
    noted = []

    class Source:
        is_cuda = True

        def record_stream(self, stream):
            noted.append(stream)

    class Matrix:
        unpacked = ()

    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: "current")
    monkeypatch.setattr(torch.cuda, "stream", lambda stream: contextlib.nullcontext())
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: capturing)
    W, kept, capturing = Matrix(), Source(), False
    W.unpacked = kept, Source()
    ss._let_go(W, 0, None)
    assert W.unpacked == () and noted == ["current"]
    W.unpacked, capturing = (Source(), Source()), True
    ss._let_go(W, 0, None)
    assert len(W.unpacked) == 2 and noted == ["current"]


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["mx4", "fp8"])
@pytest.mark.parametrize("other_stream", [False, True])
def test_packing_a_matrix_of_temporaries(ss, kind, other_stream):  # noqa: F811
    """make(...) of tensors that nothing else holds, then allocations of their sizes."""
    t, make, prepack = described(ss, kind, "cuda")
    want = prepack(make(*t))
    W = make(*(v.clone() for v in t))
    over = [torch.zeros_like(v) for v in t for _ in range(3)]  # noqa: F841
    stream = None
    if other_stream:  # the packing waits; what takes the tensors' memory meanwhile does not change it
        stream = torch.cuda.Stream()
        stream.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(stream):
            torch.cuda._sleep(1 << 24)
    got = prepack(W, stream=stream)
    over += [torch.zeros_like(v) for v in t for _ in range(3)]
    torch.cuda.synchronize()
    assert torch.equal(got, want)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["mx4", "fp8"])
def test_packing_in_a_graph(ss, kind):  # noqa: F811
    """Each replay reads the codes again: the matrix keeps them."""
    t, make, prepack = described(ss, kind, "cuda")
    want = prepack(make(*t))
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        room = torch.empty_like(want)  # what the packing takes in the graph
        W = make(*(v.clone() for v in t))
        del room
        st.synchronize()
        graph = ss.Graph()
        graph.begin()
        got = prepack(W)
        graph.end()
        over = [torch.zeros_like(v) for v in t for _ in range(3)]  # noqa: F841
        for _ in range(3):
            got.zero_()
            graph.launch()
            st.synchronize()
            assert torch.equal(got, want)
    assert len(W.unpacked) == 2
