"""What the Python binding of the stage operators refuses before a kernel sees
it, and what it keeps alive.  Host checks: no GPU."""

import gc
import os
import weakref

import pytest

torch = pytest.importorskip("torch")

from paper_2301_09830_amd import build as buildmod  # noqa: E402
from paper_2301_09830_amd import optcc  # noqa: E402


@pytest.fixture(scope="module", autouse=True)
def built():
    if not (os.path.exists(buildmod.LIB) and os.path.exists(buildmod.LAYERS)):
        buildmod.build()


# --- a workspace given by the caller -----------------------------------------
def layer_calls(ws):
    X, W, dY = torch.zeros(8, 16), torch.zeros(6, 16), torch.zeros(8, 6)
    yield lambda: optcc.occ_linear_fwd(X, W, ws=ws)
    yield lambda: optcc.occ_gated_fwd(X, W, ws=ws)
    yield lambda: optcc.occ_linear_bwd(dY, X, W, dX=torch.zeros(8, 16), ws=ws)
    yield lambda: optcc.occ_gated_bwd(dY, X, torch.zeros(12, 16), Z=torch.zeros(8, 12),
                                      dW=torch.zeros(12, 16), ws=ws)


@pytest.mark.parametrize("ws,what", [
    (torch.empty(4096, dtype=torch.uint8, device="meta"), "ws lies on another device"),
    (torch.empty(8192, dtype=torch.uint8)[::2], "ws must be contiguous"),
    (torch.empty(64, 64).t()[:, 1:], "ws must be contiguous")], ids=["device", "step", "turned"])
def test_workspace_is_checked(ws, what):
    for call in layer_calls(ws):
        with pytest.raises(ValueError, match=what):
            call()


def test_workspace_must_be_a_tensor():
    for call in layer_calls(4096):
        with pytest.raises(TypeError, match="ws must be a tensor"):
            call()


# --- the optimizer's tensors ---------------------------------------------------
class OnGpu(torch.Tensor):
    """A host tensor that says it lies on a GPU, for checks that never read it."""
    is_cuda = True
    device = torch.device("cuda", 0)


def gpu(*shape, dtype=torch.float32):
    return torch.zeros(*shape, dtype=dtype).as_subclass(OnGpu)


def tensors(rows=6, cols=300, bits=8, factors=False, make=gpu):
    """The arguments of make_param."""
    state = torch.uint8 if bits == 8 else torch.float32
    t = {"W": make(rows, cols), "m": make(rows, cols, dtype=state),
         "v": make(rows, cols, dtype=state), "W16": make(rows, cols, dtype=torch.bfloat16)}
    if factors:
        t["P"], t["Q"] = make(rows, 4), make(cols, 4)
    else:
        t["G"] = make(rows, cols)
    if bits == 8:
        t["m_scale"], t["v_scale"] = make(rows, 2), make(rows, 2)
    return t


@pytest.mark.parametrize("factors", [False, True])
@pytest.mark.parametrize("bits", [32, 8])
def test_parameters_lie_on_one_gpu(bits, factors):
    optcc.make_param(**tensors(bits=bits, factors=factors))
    for name in tensors(bits=bits, factors=factors):
        t = tensors(bits=bits, factors=factors)
        t[name] = torch.zeros_like(t[name].as_subclass(torch.Tensor))      # on the host
        with pytest.raises(ValueError, match="another device"):
            optcc.make_param(**t)
    with pytest.raises(ValueError, match="must lie on a GPU"):
        optcc.make_param(**tensors(bits=bits, factors=factors, make=torch.zeros))


def test_scale_and_flags_lie_on_a_gpu():
    """A list of no tensors is refused by the library, after the binding's checks."""
    none = (optcc.occ_param_t * 0)()
    with pytest.raises(ValueError, match="grad_scale must lie on a GPU"):
        optcc.occ_adamw_step(none, 1e-3, 1, grad_scale=torch.ones(1))
    with pytest.raises(ValueError, match="flags must lie on a GPU"):
        optcc.occ_adamw_step(none, 1e-3, 1, flags=torch.zeros(1, dtype=torch.int32))


@pytest.mark.parametrize("change", [
    {"Q": (4, 300)}, {"P": (4, 6)}, {"P": (6, 5)}, {"Q": (300, 5)}, {"Q": (1200,)}, {"P": (24,)},
    {"m": (300, 6)}, {"v": (300, 6)}, {"W16": (300, 6)}, {"m_scale": (2, 6)}, {"v_scale": (3, 4)}],
    ids=str)
def test_shapes_are_checked_not_counts(change):
    """As many contiguous values in another shape mean another order: P^T, Q^T,
    moments of the transposed weight."""
    t = tensors(factors=True)
    for name, shape in change.items():
        t[name] = gpu(*shape, dtype=t[name].dtype)
    with pytest.raises(ValueError):
        optcc.make_param(**t)


def test_flat_states_of_a_matrix_are_taken():
    """The order of the values is the matrix's: so are rank = rows and cols."""
    t = tensors(factors=True)
    for name in ("m", "v", "W16", "m_scale", "v_scale"):
        t[name] = t[name].view(-1)
    assert optcc.make_param(**t).rank == 4
    t["P"], t["Q"] = gpu(6, 6), gpu(300, 6)
    assert optcc.make_param(**t).rank == 6
    v = {k: x.view(-1) for k, x in tensors(rows=1).items()}      # a vector
    assert optcc.make_param(**v).cols == 300


def test_parameters_keep_their_tensors():
    """Temporaries given to make_param live as long as the list of parameters."""
    t = tensors()
    gone = [weakref.ref(x) for x in t.values()]
    p = optcc.make_param(**t)
    del t
    gc.collect()
    assert all(r() is not None for r in gone)
    array = optcc.make_params(q for q in [p])
    del p
    gc.collect()
    assert all(r() is not None for r in gone)
    del array
    gc.collect()
    assert all(r() is None for r in gone)


# --- the GPU that a call runs on -----------------------------------------------
class OnGpu1(OnGpu):
    device = torch.device("cuda", 1)


class Library:
    """Takes the place of the library and notes the stream of each call."""

    def __init__(self):
        self.calls = []

    def occ_adamw_step(self, params, count, hyper, stream):
        self.calls.append((count, stream))
        return 0


@pytest.mark.parametrize("stream", [None, "given"])
def test_adamw_runs_on_its_tensors_gpu(monkeypatch, stream):
    """The default stream of every GPU has the same null handle and means the
    current one, so the tensors' GPU has to be current."""
    at, seen, fake = [0], [], Library()

    class Device:
        def __init__(self, device):
            self.to, self.back = device.index, at[0]

        def __enter__(self):
            at[0] = self.to

        def __exit__(self, *_):
            at[0] = self.back

    class Stream:
        cuda_stream = 5

    monkeypatch.setattr(torch.cuda, "current_device", lambda: at[0])
    monkeypatch.setattr(torch.cuda, "device", Device)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda i: seen.append(i) or 0,
                        raising=False)
    real = fake.occ_adamw_step
    fake.occ_adamw_step = lambda *a: real(*a[:3], (at[0], a[3]))
    monkeypatch.setattr(optcc, "lib", lambda: fake)
    given = Stream() if stream else None
    handle = 5 if stream else 0
    for kind, index in ((OnGpu, 0), (OnGpu1, 1)):
        def make(*shape, dtype=torch.float32):
            return torch.zeros(*shape, dtype=dtype).as_subclass(kind)
        p = optcc.make_param(**tensors(make=make))
        optcc.occ_adamw_step([p], 1e-3, 1, stream=given, flags=make(1))
        assert fake.calls.pop() == (1, (index, handle)) and at == [0]
        assert given or seen.pop() == index
        other = OnGpu1 if index == 0 else OnGpu
        with pytest.raises(ValueError, match="another device"):
            optcc.occ_adamw_step([p], 1e-3, 1, grad_scale=torch.ones(1).as_subclass(other))
        with pytest.raises(ValueError, match="different GPUs"):
            optcc.make_params([p, optcc.make_param(**tensors(make=lambda *s, dtype=torch.float32:
                              torch.zeros(*s, dtype=dtype).as_subclass(other)))])


@pytest.mark.gpu
@pytest.mark.skipif(torch.cuda.device_count() < 2, reason="needs two GPUs")
def test_layers_run_on_their_tensors_gpu():
    """Tensors of the second GPU while the first one is current."""
    X, W = torch.randn(100, 64, device="cuda:1"), torch.randn(32, 64, device="cuda:1")
    assert torch.cuda.current_device() == 0
    Y = optcc.occ_linear_fwd(X, W)
    dX = torch.empty_like(X)
    optcc.occ_linear_bwd(Y, W=W, dX=dX)
    torch.cuda.synchronize(1)
    assert torch.cuda.current_device() == 0
    for got, want in ((Y, X.double() @ W.double().t()), (dX, Y.double() @ W.double())):
        assert torch.allclose(got.double(), want, rtol=1e-4, atol=1e-3)
