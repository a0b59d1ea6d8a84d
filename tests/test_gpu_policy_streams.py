"""The operators around the layer step on a given stream: what they allocate is that stream's.

Each test keeps the caller's stream busy and lets go of a block of memory that the call on the other stream would be handed if it took
its memory from the caller's stream (or the other way round), then looks at what the busy stream read."""
import pytest
import torch

from paper_2512_23353_amd import isopo

pytestmark = pytest.mark.gpu

N, K, OUT, VOCAB = 2048, 64, 4096, 4096


class _Calls:
    """name -> a call whose largest outputs have N * OUT fp32 elements."""

    def __init__(self, device):
        gen = torch.Generator(device=device).manual_seed(1)
        mk = lambda *s: torch.randn(s, generator=gen, device=device)  # noqa: E731
        X, W, Wb, dY, Z = mk(N, K), mk(OUT, K), mk(K, OUT), mk(N, K), mk(N, K)
        logits, w = mk(N, VOCAB), mk(N)
        y = torch.randint(0, VOCAB, (N,), generator=gen, device=device, dtype=torch.int32)
        lse = isopo.token_logprob(logits, y)["lse"]
        opt = isopo.AdamW([torch.randn(N * OUT, generator=gen, device=device)], state_bits=8)
        self.by_name = {
            "linear": lambda s: isopo.linear(X, W, act="silu", keep_z=True, stream=s),
            "linear_backward": lambda s: isopo.linear_backward(dY, Wb, Z, "silu", need_db=True, stream=s)[1],
            "token_logprob": lambda s: isopo.token_logprob(logits, y, weight=w, stream=s)["dlogits"],
            "token_logprob_backward": lambda s: isopo.token_logprob_backward(logits, y, lse, w, stream=s),
            "adamw_state": lambda s: isopo.adamw_state(opt.m[0], opt.m_scales[0], opt.v[0], opt.v_scales[0], stream=s)[0],
        }


NAMES = ("linear", "linear_backward", "token_logprob", "token_logprob_backward", "adamw_state")


def _keep_busy(a):
    for _ in range(12):                               # some 10 ms of the current stream
        a = torch.mm(a, a) * 1e-3
    return a


def _stream_that_owns(t):
    at = t.untyped_storage().data_ptr()
    (owner,) = [seg["stream"] for seg in torch.cuda.memory_snapshot() if seg["address"] <= at < seg["address"] + seg["total_size"]]
    return owner


@pytest.mark.parametrize("handle", (False, True))
@pytest.mark.parametrize("name", NAMES)
def test_a_given_stream_owns_what_is_allocated(gpu_device, name, handle):
    call, side, a = _Calls(gpu_device).by_name[name], torch.cuda.Stream(), torch.randn(4096, 4096, device=gpu_device)
    want = call(None)
    torch.cuda.synchronize()
    s = side.cuda_stream if handle else side
    # memory of the caller's stream that is still to be read when the call is made
    read = torch.arange(N * OUT, dtype=torch.float32, device=gpu_device)
    torch.cuda.synchronize()
    _keep_busy(a)
    seen = read * 1.0
    del read
    got = call(s)
    torch.cuda.synchronize()
    assert torch.equal(seen, torch.arange(N * OUT, dtype=torch.float32, device=gpu_device))
    for g, w in zip(got if isinstance(got, tuple) else (got,), want if isinstance(want, tuple) else (want,)):
        assert torch.equal(g, w) and _stream_that_owns(g) == side.cuda_stream
    # what the call returned, let go while the caller's stream is still to read it
    want = want[0] if isinstance(want, tuple) else want
    got = got[0] if isinstance(got, tuple) else got
    _keep_busy(a)
    seen = got * 1.0
    del got, g
    with torch.cuda.stream(side):
        torch.full((N * OUT,), 7.0, device=gpu_device)
    torch.cuda.synchronize()
    assert torch.equal(seen, want)


def test_the_default_stream_by_its_handle(gpu_device):
    X, W = torch.randn(8, 64, device=gpu_device), torch.randn(16, 64, device=gpu_device)
    want, side = isopo.linear(X, W), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        got = isopo.linear(X, W, stream=0)
    torch.cuda.synchronize()
    assert torch.equal(got, want) and _stream_that_owns(got) == 0


def test_the_norm_that_clips_is_the_steps_own(gpu_device):
    """Returned and dropped at once, as a caller does who does not look at it: the caller's stream does not get its memory."""
    side = torch.cuda.Stream()
    a, b = (isopo.AdamW([torch.ones(1 << 22, device=gpu_device)]) for _ in range(2))
    g = [torch.randn(1 << 22, device=gpu_device)]
    torch.cuda.synchronize()
    for _ in range(5):
        a.step(g, 1e-2, max_norm=1.0)
    torch.cuda.synchronize()
    for k in range(5):
        b.step(g, 1e-2, max_norm=1.0, stream=side)
        torch.full((), 1e9, device=gpu_device)
    torch.cuda.synchronize()
    assert torch.equal(a.params[0], b.params[0])
    norm = b.step(g, 1e-2, max_norm=1.0, stream=side)
    side.synchronize()
    assert _stream_that_owns(norm) == side.cuda_stream


def test_a_given_stream_that_is_captured(gpu_device):
    X, W = torch.randn(24, 4096, device=gpu_device), torch.randn(512, 4096, device=gpu_device)
    want = isopo.linear(X, W)
    torch.cuda.synchronize()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=side):
        got = isopo.linear(X, W, stream=side)
    for _ in range(3):
        got.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, want)
