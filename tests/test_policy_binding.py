"""The Python bindings of the operators around the layer step: what they look at before a call.  No GPU needed: nothing is launched."""
import pytest
import torch

from paper_2512_23353_amd import isopo, policy
from paper_2512_23353_amd.policy import IsopoUpdate, PolicyLinear, PolicyTrainer, _rows


def test_a_stream_for_host_tensors_is_refused():
    with pytest.raises(ValueError):
        isopo.linear(torch.zeros(4, 16), torch.zeros(8, 16), stream=1)


@pytest.mark.parametrize("bits", (8, 32))
def test_adamw_refuses_host_tensors(bits):
    with pytest.raises(ValueError):
        isopo.AdamW([torch.zeros(300), torch.zeros(5)], state_bits=bits)


class _Library:
    """Takes note of the parameters' addresses that a step names, and launches nothing."""

    def __init__(self, library):
        self.library, self.params = library, []

    def __getattr__(self, name):
        if name in ("isopo_adamw", "isopo_adamw_clipped"):
            return lambda tensors, grads, n, *rest: self.params.append([t.param for t in tensors[:n]]) or 0
        return getattr(self.library, name)


@pytest.fixture
def library(monkeypatch):
    """Host tensors pass for a GPU's, and the library is not called."""
    lib = _Library(isopo.load())
    monkeypatch.setattr(isopo, "_lib", lib)
    monkeypatch.setattr(isopo, "_stream_of", lambda t: 0)
    monkeypatch.setattr(torch.Tensor, "get_device", lambda t: 0)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    return lib


def _where(*params):
    return [p.data_ptr() for p in params]


def test_adamw_follows_its_parameters(library):
    a, b = torch.nn.Parameter(torch.ones(64)), torch.nn.Parameter(torch.ones(8, 4))
    opt = isopo.AdamW([a, b])
    g = [torch.ones(64), torch.ones(8, 4)]
    opt.step(g, 1e-3)
    assert library.params[-1] == _where(a, b)
    before = a.data_ptr()
    a.data = torch.full((64,), 2.0)
    opt.step(g, 1e-3, max_norm=1.0)
    assert a.data_ptr() != before and library.params[-1] == _where(a, b)
    c = torch.nn.Parameter(torch.zeros(8, 4))
    opt.params[1] = c
    opt.step(g, 1e-3)
    assert library.params[-1] == _where(a, c) and opt.steps_done == 3
    for bad in (torch.zeros(65), torch.zeros(64, dtype=torch.bfloat16), torch.zeros(128)[::2]):
        a.data = bad
        with pytest.raises(ValueError):
            opt.step(g, 1e-3)
    assert len(library.params) == 3 and opt.steps_done == 3


def test_adamw_holds_what_the_library_is_told_of(library):
    """A parameter's storage is not handed out again before the next step has looked; states are the optimiser's."""
    p = torch.nn.Parameter(torch.ones(1 << 20))
    opt = isopo.AdamW([p], state_bits=8)
    old = p.data_ptr()
    p.data = torch.empty(0)
    assert all(torch.empty(1 << 20).data_ptr() != old for _ in range(4))
    state = opt.m[0]
    at = state.data_ptr()
    state.data = torch.empty(0)
    del state
    assert opt.m[0].data_ptr() == at == opt._tensors[0].m
    with pytest.raises(TypeError):
        opt.m[0] = torch.zeros(1 << 20, dtype=torch.uint8)
    with pytest.raises(AttributeError):
        opt.v = []
    opt.m_scales[0].fill_(2.0)
    assert bool((opt.m_scales[0] == 2.0).all()) and opt.masters is None
    given = torch.zeros(100)
    opt = isopo.AdamW([torch.zeros(100)], m=[given], v=[torch.zeros(100)])
    assert opt.m[0].data_ptr() == given.data_ptr()


def test_adamw_refuses_memory_that_is_written_twice(library):
    p, buf = torch.zeros(512), torch.zeros(1024)
    for bad in (lambda: isopo.AdamW([p, p]), lambda: isopo.AdamW([buf[:600], buf[512:]]), lambda: isopo.AdamW([p], m=[buf[:512]], v=[buf[256:768]]),
                lambda: isopo.AdamW([p], m=[p]), lambda: isopo.AdamW([buf[:512], buf[512:]], masters=[buf[512:], torch.zeros(512)])):
        with pytest.raises(ValueError):
            bad()
    opt = isopo.AdamW([buf[:512], buf[512:], torch.zeros(0), torch.zeros(0)], masters=[buf[:512], torch.zeros(512), torch.zeros(0), torch.zeros(0)])
    opt.params[1] = buf[256:768]
    with pytest.raises(ValueError):
        opt.step([torch.zeros(512), torch.zeros(512), torch.zeros(0), torch.zeros(0)], 1e-3)
    assert not library.params


def test_a_captured_step_says_that_it_repeats(library, monkeypatch, recwarn):
    opt = isopo.AdamW([torch.zeros(64)], step=4)
    opt.step([torch.zeros(64)], 1e-3)
    assert not recwarn.list
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: True)
    with pytest.warns(UserWarning, match="repeats step 6"):
        opt.step([torch.zeros(64)], 1e-3)
    layer = PolicyLinear(16, 8, dtype=torch.float32)
    layer.weight_grad = torch.zeros(8, 16)
    trainer = PolicyTrainer([layer])
    with pytest.raises(RuntimeError, match="captured"):
        trainer.step()
    assert len(library.params) == 2 and trainer.optimiser.steps_done == 0 and layer.weight_grad is not None
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    trainer.step()
    assert trainer.optimiser.steps_done == 1


@pytest.mark.parametrize("dtype", (torch.float32, torch.bfloat16))
def test_rows_are_taken_as_they_are_or_copied(dtype):
    base = torch.arange(4096).to(dtype)
    vec = 16 // base.element_size()
    assert base.data_ptr() % 16 == 0
    for t in (base[:256].view(4, 64), base.view(32, 128)[:, :64], base.view(32, 128)[:, vec:vec + 64], base.view(32, 128)[3:4, :64], base[:0].view(0, 64),
              base[:1].view(1, 1).expand(1, 64).contiguous(), base[:7].view(7, 1)[:1]):
        assert _rows(t) is t
    for t in (base[1:257].view(4, 64), base[:64].view(1, 64).expand(4, 64), base.view(64, 64).t(), base[:4090].view(10, 409)[:, :64], base.view(32, 128)[:, 1:65],
              base[:1].view(1, 1).expand(4, 64), base.as_strided((2, 8), (4, 1))):
        got = _rows(t)
        assert got is not t and got.is_contiguous() and got.data_ptr() % 16 == 0 and torch.equal(got, t)


def test_no_z_is_kept_where_nothing_is_recorded(monkeypatch):
    kept = []

    def linear(x, weight, bias, act, residual, keep_z):
        kept.append(keep_z)
        y = x @ weight.t()
        return (y, y.clone()) if keep_z else y

    monkeypatch.setattr(isopo, "linear", linear)
    layer, x = PolicyLinear(16, 8, act="silu", dtype=torch.float32), torch.zeros(4, 16)
    with torch.no_grad():
        layer(x)
    with torch.inference_mode():
        layer(torch.zeros(4, 16))
    layer(x)
    layer.weight.requires_grad_(False)
    layer(x)
    layer(x.clone().requires_grad_())
    PolicyLinear(16, 8, dtype=torch.float32)(x)
    assert kept == [False, False, True, False, True, False]


def test_a_backward_pass_is_of_sequences_that_were_named_for_it(monkeypatch):
    """Offsets and advantages of the microbatch before are not taken for the next one's, whatever its number of tokens."""
    steps = []

    def layer_step(x, delta, offsets, advantages, cfg):
        steps.append(advantages)
        return delta.t() @ x

    monkeypatch.setattr(policy, "_hip_layer_step", layer_step)
    monkeypatch.setattr(isopo, "weighted_grad", lambda layer, c: layer.Delta.t() @ layer.X)
    monkeypatch.setattr(isopo, "linear", lambda x, weight, *a, **kw: x.detach() @ weight.detach().t())
    monkeypatch.setattr(isopo, "linear_backward", lambda dy, weight, *a, **kw: (dy, dy @ weight.detach(), None))
    a, b = PolicyLinear(8, 8, dtype=torch.float32), PolicyLinear(8, 8, dtype=torch.float32)
    update, x = IsopoUpdate([a, b]), torch.ones(4, 8)
    one, two = torch.ones(1), torch.full((1,), 2.0)
    with pytest.raises(RuntimeError, match="begin"):
        b(a(x)).sum().backward()
    loss = b(a(x)).sum()
    update.begin([0, 4], one)                         # after the forward pass
    loss.backward(retain_graph=True)
    loss.backward()                                   # the same microbatch again
    assert len(steps) == 4
    loss = b(a(x)).sum()                              # another one
    with pytest.raises(RuntimeError, match="begin"):
        loss.backward(retain_graph=True)
    assert len(steps) == 4
    update.begin([0, 4], two)
    loss.backward()
    assert len(steps) == 6 and steps[-1] is two
    update.begin([0, 4], one)                         # before the forward pass; a layer used twice
    b(a(a(x))).sum().backward()
    assert len(steps) == 9 and steps[-1] is one
    first, second = b(a(x)).sum(), b(a(x)).sum()      # two forward, then two backward
    update.begin([0, 4], one)
    first.backward()
    update.begin([0, 4], two)
    second.backward()
    assert [s is two for s in steps[-4:]] == [False, False, True, True]
    update.remove()
    b(a(x)).sum().backward()
    a.update = lambda layer, x, delta: steps.append(layer) or delta.t() @ x
    b(a(x)).sum().backward()
    assert steps[-1] is a


def test_the_trainer_follows_its_layers(library):
    """bf16 weights with fp32 masters; the library is not called, so parameters change from outside alone."""
    torch.manual_seed(0)
    a, b = PolicyLinear(16, 8), PolicyLinear(8, 16, bias=True)
    trainer = PolicyTrainer([a, b])
    low = [m * (1 + 2.0 ** -12) for m in trainer.optimiser.masters]
    for m, value in zip(trainer.optimiser.masters, low):
        m.copy_(value)                                # low bits that the parameters do not have

    def step():
        for layer, name in trainer._slots:
            setattr(layer, name + "_grad", torch.zeros(getattr(layer, name).shape))
        trainer.step()
        assert library.params[-1] == _where(a.weight, b.weight, b.bias)
        return trainer.optimiser.masters

    assert all(torch.equal(m, v) for m, v in zip(step(), low))
    loaded = {k: v.clone() for k, v in a.state_dict().items()}
    loaded["weight"][0] = 3.0
    a.load_state_dict(loaded)                         # a checkpoint, one row of which is new
    masters = step()
    assert bool((masters[0][0] == 3.0).all()) and torch.equal(masters[0][1:], low[0][1:]) and torch.equal(masters[1], low[1])
    a.weight.data = a.weight.data.clone()             # other storage, the same values
    assert torch.equal(step()[0], masters[0])
    b.weight = torch.nn.Parameter(torch.full((16, 8), 5.0, dtype=torch.bfloat16))
    masters = step()
    assert bool((masters[1] == 5.0).all()) and torch.equal(masters[0][1:], low[0][1:])
    b.bias.data.fill_(2.0)                            # leaves no trace
    trainer.read_parameters()
    assert bool((step()[2] == 2.0).all()) and torch.equal(step()[0][1:], low[0][1:])
    a.to(torch.float32)
    with pytest.raises(ValueError):
        step()
    with pytest.raises(ValueError):
        PolicyTrainer([b, b])


def test_a_backward_pass_through_weights_that_a_step_changed_is_refused(library, monkeypatch):
    monkeypatch.setattr(isopo, "linear", lambda x, weight, *a, **kw: x.detach() @ weight.detach().t())
    monkeypatch.setattr(isopo, "linear_backward", lambda dy, weight, *a, **kw: (dy, dy @ weight.detach(), None))
    monkeypatch.setattr(isopo, "weighted_grad", lambda layer, c: layer.Delta.t() @ layer.X)
    a, b = PolicyLinear(8, 8, dtype=torch.float32), PolicyLinear(8, 8, dtype=torch.float32)
    trainer = PolicyTrainer([a, b])
    for _ in range(2):
        loss = b(a(torch.ones(4, 8))).sum()
        loss.backward(retain_graph=True)
        trainer.step()
        with pytest.raises(RuntimeError, match="inplace"):
            loss.backward()
        a.weight_grad = b.weight_grad = None
