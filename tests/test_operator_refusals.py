"""What the temporal head's operators refuse before anything reaches a GPU."""
import pytest
import torch

import paper_1806_04965_b200 as sr
from paper_1806_04965_b200 import SrError


@pytest.mark.parametrize("name, value", [("rows", 5000), ("rows", 1 << 40), ("rows", 1 << 70), ("cols", 96), ("cols", 0), ("rows", -1), ("format", "mx8"), ("format", "mx6"),
                                         ("data", torch.zeros(4, 16, dtype=torch.uint8)), ("data", torch.zeros(4, 64, dtype=torch.uint8)[:, ::2]),
                                         ("data", torch.zeros(4, 32, dtype=torch.int8)), ("scales", torch.zeros(4, dtype=torch.uint8))])
def test_a_microscaled_matrix_that_no_longer_fits_its_buffers_is_refused(name, value):
    # its attributes can be assigned after it was made; a kernel would read behind the buffers' ends
    good, bad = sr.Microscaled.empty(4, 64, "mx4", "cpu"), sr.Microscaled.empty(4, 64, "mx4", "cpu")
    setattr(bad, name, value)
    for call in (lambda: bad.values(), lambda: sr.product(good, bad), lambda: sr.product(bad, good), lambda: sr.product(bad, bad)):
        with pytest.raises(SrError, match="sizes|out of range|format"):
            call()


def test_an_argument_without_a_truth_value_raises_its_own_error():
    import numpy as np
    m = sr.Microscaled.empty(4, 64, "mx4", "cpu")
    with pytest.raises((SrError, ValueError)):                  # not a SystemError of a call that returned with an exception set
        sr.product(m, m, relu=np.array([1, 2]))


def test_status_of_something_that_is_no_cuda_device_is_refused():
    for call in (sr.operator_status, sr.operator_reset):
        with pytest.raises(SrError, match="CUDA device"):
            call("cpu")


def calls(x):
    """Every call with x (a float32 tensor of at least 2 x 64 elements) as one of its inputs."""
    m = sr.Microscaled.empty(4, 64, "mx4", "cpu") if not x.is_cuda else sr.quantize(torch.zeros(4, 64, device=x.device))
    v = torch.zeros(64, device=x.device)
    h = x.reshape(-1)[:128].view(1, 2, 64)
    o = torch.zeros(1, 2, 64, device=x.device)
    d, s = torch.zeros(2, device=x.device), torch.zeros(1, 2, 64, 64, device=x.device)
    row = x.reshape(-1)[:64]
    return [lambda: sr.quantize(x), lambda: sr.rms_norm(x), lambda: sr.rms_norm(x.detach(), row), lambda: sr.rms_norm(x.detach(), v, residual=x),
            lambda: sr.product(m, m, bias=row[:4]), lambda: sr.linear_attention_step(h, o, o, d, s), lambda: sr.linear_attention_step(o, h, o, d, s),
            lambda: sr.linear_attention_step(o, o, h, d, s), lambda: sr.linear_attention_step(o, o, o, row[:2], s),
            lambda: sr.linear_attention_run(h[None], o[None], o[None], d), lambda: sr.linear_attention_run(o[None], o[None], h[None], d),
            lambda: sr.linear_attention_run(o[None], o[None], o[None], row[:2])]


@pytest.mark.parametrize("device", ["cpu", pytest.param("cuda:0", marks=pytest.mark.gpu)])
def test_derivatives_are_refused_in_both_directions(device):
    import torch.autograd.forward_ad as forward_ad
    x = torch.ones(4, 64, device=device)
    for call in calls(x.clone().requires_grad_()):
        with pytest.raises(SrError, match="no backward pass"):
            call()
    with forward_ad.dual_level():
        for grad in (True, False):
            with torch.set_grad_enabled(grad):
                for call in calls(forward_ad.make_dual(x, torch.ones_like(x))):
                    with pytest.raises(SrError, match="no forward derivative"):
                        call()
    with pytest.raises(SrError, match="no forward derivative"):
        torch.func.jvp(lambda y: sr.rms_norm(y), (x,), (x,))


@pytest.mark.gpu
def test_what_has_no_derivative_recorded_is_still_taken():
    x = torch.ones(4, 64, device="cuda:0")
    for y in (x, x.clone().requires_grad_().detach()):
        for call in calls(y):
            call()
    with torch.no_grad():
        for call in calls(x.clone().requires_grad_()):
            call()
    with torch.inference_mode():
        for call in calls(torch.ones(4, 64, device="cuda:0")):
            call()


@pytest.mark.gpu
@pytest.mark.parametrize("compiled", [True, False])
def test_what_is_written_in_place_gets_a_new_version(compiled, monkeypatch):
    if not compiled:
        for name in ("quantize", "product", "rms_norm", "run", "step"):
            monkeypatch.setattr(sr.operators._compiled, name, lambda *_: None)
    D = "cuda:0"
    h, d = torch.ones(3, 1, 2, 64, device=D), torch.zeros(2, device=D)
    state, out = torch.zeros(1, 2, 64, 64, device=D), torch.zeros(3, 1, 2, 64, device=D)
    versions = [t._version for t in (state, out, h, d)]
    sr.linear_attention_step(h[0], h[0], h[0], d, state)
    sr.linear_attention_run(h, h, h, d, state=state)
    assert [t._version for t in (state, out, h, d)] == [versions[0] + 1] + versions[1:]
    sr.linear_attention_run(h, h, h, d, state=state, out=out, state_out=state)
    assert [t._version for t in (state, out, h, d)] == [versions[0] + 2, versions[1] + 1] + versions[2:]
    m, y = sr.quantize(torch.ones(4, 64, device=D)), torch.zeros(4, 8, device=D)
    sr.product(m, m, out=y[:, :4])
    assert y._version == 1 and m.data._version == 0
    with torch.inference_mode():
        frozen = torch.zeros(1, 2, 64, 64, device=D)
    sr.linear_attention_step(h[0], h[0], h[0], d, frozen)       # as before: written, there is no version
    assert (frozen != 0).any()
    w = torch.zeros(1, 2, 64, 64, device=D, requires_grad=True)
    kept = w * 1
    loss = (kept * kept).sum()
    with torch.no_grad():
        sr.linear_attention_step(h[0], h[0], h[0], d, kept)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()


def weights(channels=10, heads=4, groups=2, dk=32, dv=48, outputs=7):
    shapes = {"qkv": (heads * dk + groups * (dk + dv), channels), "o": (channels, heads * dv), "out": (outputs, channels), "bias": (outputs,), "norm_x": (channels,),
              "norm_o": (heads * dv,), "norm_h": (channels,), "log_decay": (groups,)}
    return {n: torch.full(s, -0.1) for n, s in shapes.items()}


def test_head_refuses_what_none_of_its_calls_would_take():
    sizes = dict(channels=10, heads=4, groups=2, dk=32, dv=48, batch=4, device="cpu")
    for bad in (dict(heads=3), dict(groups=0), dict(heads=0), dict(dk=257), dict(dv=0), dict(batch=-1), dict(dtype="fp16"), dict(format="mx6"), dict(eps=-1.0), dict(eps=float("nan")),
                dict(heads=258, groups=2)):
        with pytest.raises(SrError, match="TemporalHead: (sizes|dtype)"):
            sr.TemporalHead(weights(), **{**sizes, **bad})
    for name in weights():
        w = weights()
        del w[name]
        with pytest.raises(SrError, match="%s is missing" % name):
            sr.TemporalHead(w, **sizes)
        w = weights()
        w[name] = w[name][None]
        with pytest.raises(SrError, match="%s has shape" % name):
            sr.TemporalHead(w, **sizes)


@pytest.mark.gpu
def test_rollout_with_a_head_that_does_not_fit_changes_nothing():
    from tests.parity import make_graph, to_device
    from workloads import data, graphs
    spec = graphs.build("c2", batch=4, frames=5)
    G = make_graph(spec, "streaming", weights=data.make_weights(spec), biases=data.make_biases(spec))
    frames = [to_device(spec, data.make_inputs(spec)[v]) for v in G.input_nodes]
    want = G.rollout(frames)
    t, state = G.frame(), G.get_state(G.output_node)
    for kw in (dict(batch=3), dict(channels=11)):
        c = kw.get("channels", 10)
        head = sr.TemporalHead(weights(channels=c), c, 4, 2, 32, 48, batch=kw.get("batch", 4))
        head.state.fill_(2.0)
        with pytest.raises(SrError, match="the head takes"):
            G.rollout(frames, head=head)
        assert (head.state == 2).all() and G.frame() == t and torch.equal(torch.as_tensor(G.get_state(G.output_node)), torch.as_tensor(state))
    assert torch.equal(G.rollout(frames), want)


def test_what_is_no_tensor_is_refused():
    import numpy as np
    m, t, d = sr.Microscaled.empty(4, 64, "mx4", "cpu"), torch.zeros(1, 2, 8), torch.zeros(2)
    for no in ([1.0], np.zeros((4, 64), np.float32), 3, "x", None):
        for call in (lambda: sr.quantize(no), lambda: sr.rms_norm(no), lambda: sr.product(no, m), lambda: sr.product(m, no), lambda: sr.linear_attention_step(no, t, t, d, t),
                     lambda: sr.linear_attention_run(no, t, t, d), lambda: sr.Microscaled(no, m.scales, 4, 64, "mx4")):
            with pytest.raises(SrError, match="required"):
                call()
        if no is not None:
            for call in (lambda: sr.rms_norm(t[0], no), lambda: sr.product(m, m, bias=no), lambda: sr.product(m, m, out=no), lambda: sr.linear_attention_run(t, t, t, d, state=no)):
                with pytest.raises(SrError, match="required"):
                    call()


@pytest.mark.gpu
def test_anything_with_reset_and_run_may_stand_behind_a_rollout():
    from tests.parity import make_graph, to_device
    from workloads import data, graphs
    spec = graphs.build("c2", batch=4, frames=3)
    G = make_graph(spec, "streaming", weights=data.make_weights(spec), biases=data.make_biases(spec))
    frames = [to_device(spec, data.make_inputs(spec)[v]) for v in G.input_nodes]

    class Sum:
        def reset(self):
            self.total = 0.0

        def run(self, features):
            self.total = self.total + features.sum(0)
            return self.total
    assert torch.equal(G.rollout(frames, head=Sum()), G.rollout(frames).sum(0))
