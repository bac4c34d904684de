"""What an AdamW object passes to the library, all on the host (no GPU needed):
the calls are recorded in the library's place, CPU tensors stand in for GPU ones."""

import pytest
import torch

gift = pytest.importorskip("paper_2607_07494_amd.gift")


class Library:
    """``gift_adamw_step`` that keeps the tensors' fields of its last call."""

    def gift_adamw_step(self, ctx, count, tensors, options):
        o = options._obj
        self.options = (o.beta1, o.beta2, o.eps, o.seed, o.moments)
        self.tensors = [{f: getattr(tensors[i], f) for f, _ in gift._AdamWTensor._fields_} for i in range(count)]
        return gift.OK

    def __getattr__(self, name):
        return getattr(gift_library, name)


gift_library = gift.LIB


@pytest.fixture
def lib(monkeypatch):
    def contiguous(tensors, name):
        if not all(map(torch.Tensor.is_contiguous, tensors)):
            raise ValueError(f"{name} must be contiguous")

    fake = Library()
    monkeypatch.setattr(gift, "LIB", fake)
    monkeypatch.setattr(gift, "_all_on_current_device", contiguous)
    monkeypatch.setattr(gift, "_on_current_device", lambda **tensors: contiguous(tensors.values(), "a tensor"))
    return fake


@pytest.fixture
def ctx():
    c = gift.Context(stream=0)
    yield c
    c.close()


def zeros(params, moments):
    return {k: torch.zeros(n, dtype=t) for k, (n, t) in gift.AdamW.state_sizes(params, moments).items()}


def optimizer(ctx, moments, sizes=(600, 3, 1100)):
    params = [torch.zeros(n) for n in sizes]
    copies = [torch.zeros(n, dtype=torch.bfloat16) if k != 1 else None for k, n in enumerate(sizes)]
    return gift.AdamW(ctx, params, weight_decay=0.1, moments=moments, state=zeros(params, moments), copies=copies)


def gradients(opt):
    return [torch.zeros_like(p) for p in opt.params]


def check(lib, opt, grads):
    """The last call's addresses are those of the tensors that the object holds now."""
    for t, p, c, g, at in zip(lib.tensors, opt.params, opt.copies, grads, opt.starts):
        assert t["param"] == p.data_ptr() and t["grad"] == g.data_ptr() and t["numel"] == p.numel()
        assert t["copy"] == (c.data_ptr() if c is not None else None) and t["weight_decay"] == 0.1
        for k in "mv":
            assert t[k] == opt.state[k].data_ptr() + at * opt.state[k].element_size()
            if opt.moments == "e4m3":
                assert t[k + "_scales"] == opt.state[k + "_scales"].data_ptr() + at // 256 * 4


@pytest.mark.parametrize("moments", ["f32", "e4m3"])
def test_a_step_works_on_the_memory_that_the_tensors_have_now(lib, ctx, moments):
    opt = optimizer(ctx, moments)

    def step():
        grads = gradients(opt)
        opt.step(grads, lr=0.1)
        check(lib, opt, grads)

    step()
    opt.params[0].data = torch.ones(600)
    step()
    opt.copies[2].data = torch.ones(1100, dtype=torch.bfloat16)
    step()
    opt.params[1] = torch.ones(3)
    step()
    opt.copies[1] = torch.zeros(3, dtype=torch.bfloat16)
    step()
    opt.copies[0] = None
    step()
    for name in list(opt.state):
        opt.state[name] = opt.state[name].clone()
        step()
        opt.state[name].data = opt.state[name].clone()
        step()
    opt.state = zeros(opt.params, moments)
    step()
    assert opt.steps == 7 + 2 * len(opt.state)


def test_a_step_refuses_what_the_constructor_refuses(lib, ctx):
    opt = optimizer(ctx, "e4m3")
    grads = gradients(opt)
    opt.step(grads, lr=0.1)
    state, copies, data = dict(opt.state), list(opt.copies), [p.data for p in opt.params]
    lib.tensors = None

    def refused(error, match):
        for _ in range(2):          # the next step does not take it either
            with pytest.raises(error, match=match):
                opt.step(grads, lr=0.1)
        assert lib.tensors is None and opt.steps == 1
        opt.state, opt.copies = dict(state), list(copies)
        for p, d in zip(opt.params, data):
            p.data = d

    opt.params[0].data = data[0].to(torch.float64)
    refused(TypeError, "parameters must be float32")
    opt.params[0].data = data[0][:599]
    refused(ValueError, "a parameter must have shape")
    opt.params[0].data = torch.zeros(1200)[::2]
    refused(ValueError, "contiguous")
    opt.copies[0] = torch.zeros(600)
    refused(TypeError, "copies must be bfloat16")
    opt.copies[0] = torch.zeros(599, dtype=torch.bfloat16)
    refused(ValueError, "a copy must have shape")
    opt.copies = copies[:2]
    refused(ValueError, "keep their lengths")
    opt.state["m"] = torch.zeros(600, dtype=torch.uint8)
    refused(ValueError, "must have shape")
    opt.state["v_scales"] = state["v_scales"].double()
    refused(TypeError, "must have dtype")
    del opt.state["m"]
    refused(ValueError, "state must hold")
    opt.state["m"] = state["v"]
    refused(ValueError, "overlap")
    opt.params[2].data = torch.zeros(2000)[100:1200]
    opt.copies[2] = opt.params[2].data.view(torch.bfloat16)[:1100]
    refused(ValueError, "overlap")
    opt.step(grads, lr=0.1)
    check(lib, opt, grads)


def test_a_square_parameter_transposed_in_place_is_refused(lib, ctx):
    p = torch.zeros(4, 4)
    opt = gift.AdamW(ctx, [p], state=zeros([p], "f32"))
    opt.step([torch.zeros(4, 4)], lr=0.1)
    p.t_()
    with pytest.raises(ValueError, match="contiguous"):
        opt.step([torch.zeros(4, 4)], lr=0.1)


def test_lists_of_another_length_are_refused(lib, ctx):
    opt = optimizer(ctx, "f32")
    opt.params.append(torch.zeros(5))
    with pytest.raises(ValueError, match="keep their lengths"):
        opt.step(gradients(opt), lr=0.1)


def test_betas_eps_and_seed_set_between_steps_reach_the_library(lib, ctx):
    opt = optimizer(ctx, "e4m3")
    opt.step(gradients(opt), lr=0.1)
    assert lib.options == (0.9, 0.95, 1e-8, 0, 1)
    opt.betas, opt.eps, opt.seed = (0.8, 0.99), 1e-6, -1
    assert (opt.betas, opt.eps, opt.seed) == ((0.8, 0.99), 1e-6, 2 ** 64 - 1)
    opt.step(gradients(opt), lr=0.1)
    assert lib.options == (0.8, 0.99, 1e-6, 2 ** 64 - 1, 1)
    with pytest.raises(AttributeError):
        opt.moments = "f32"
