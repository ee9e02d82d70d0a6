"""The language model's block on the CPU, with torch's formulas in place of the library's calls: when it runs on the feed-forward kernels, and when its
maps are called."""
import pytest
import torch

from paper_2601_05732_amd import lm


class _Norm(torch.nn.Module):
    def forward(self, h):
        return h


class _Tagged(torch.Tensor):
    """A tensor that wants to see what is done with it."""


@pytest.fixture
def block(monkeypatch):
    block = lm.Block(16, 24, torch.float32, "cpu")
    block.norm = _Norm()
    block.calls = []

    def apply_gated_ffn(x, W_up, W_down):
        block.calls.append(1)
        a, b = (x @ W_up.t()).chunk(2, dim=-1)
        return (torch.nn.functional.silu(a) * b) @ W_down.t()

    monkeypatch.setattr(lm, "apply_gated_ffn", apply_gated_ffn)
    monkeypatch.setattr(lm, "takes", lambda C, H, dtype: C % 8 == 0 and H % 8 == 0)
    return block


def _maps(block, h):
    a, b = block.up(h).chunk(2, dim=-1)
    return block.down(torch.nn.functional.silu(a) * b)


def test_the_block_runs_on_the_kernels(block):
    h = torch.randn(5, 16)
    assert torch.allclose(block(h), _maps(block, h), atol=1e-6) and block.calls == [1]
    block.up.weight.requires_grad_(False)
    block(h)
    assert block.calls == [1, 1]


@pytest.mark.parametrize("name", ["up", "down"])
def test_a_forward_that_a_user_replaced_is_called(block, name):
    h = torch.randn(5, 16)
    m = getattr(block, name)
    plain, ours = block(h), m.forward
    m.forward = lambda x: 3 * ours(x)
    assert torch.equal(block(h), _maps(block, h)) and not torch.allclose(block(h), plain)
    assert block.calls == [1]
    # as some do, with a weight that is elsewhere until then
    weight = m.weight
    del m.weight
    m.forward = lambda x: torch.nn.functional.linear(x, weight)
    assert torch.equal(block(h), _maps(block, h)) and block.calls == [1]


def test_a_forward_that_a_user_replaced_for_all_maps_is_called(block, monkeypatch):
    h, forward = torch.randn(5, 16), torch.nn.Linear.forward
    monkeypatch.setattr(torch.nn.Linear, "forward", lambda self, x: 2 * forward(self, x))
    assert torch.equal(block(h), _maps(block, h)) and block.calls == []


@pytest.mark.parametrize("name", ["up", "down"])
def test_a_weight_of_another_class_is_used_by_its_map(block, name):
    h = torch.randn(5, 16)
    m = getattr(block, name)
    m.weight = torch.nn.Parameter(m.weight.detach().as_subclass(_Tagged))
    assert isinstance(m.weight, _Tagged)
    assert torch.equal(block(h), _maps(block, h)) and block.calls == []


def test_hooks_of_all_modules_see_the_maps(block):
    h, seen = torch.randn(5, 16), []
    for register in (torch.nn.modules.module.register_module_forward_hook, torch.nn.modules.module.register_module_forward_pre_hook,
                     torch.nn.modules.module.register_module_full_backward_hook):
        handle = register(lambda m, *args: seen.append(m))
        try:
            block(h.requires_grad_()).sum().backward()
        finally:
            handle.remove()
        assert block.up in seen and block.down in seen and block.calls == []
        seen.clear()
    block(h)
    assert block.calls == [1]


def test_a_compiled_map_is_called(block):
    h, seen = torch.randn(5, 16), []

    def compiled(x):
        seen.append(1)
        return block.down._call_impl(x)

    block.down._compiled_call_impl = compiled       # (what Module.compile leaves)
    block(h)
    assert seen == [1] and block.calls == []


def test_weights_of_other_shapes_go_through_the_maps(block):
    h = torch.randn(5, 16)
    block.up.weight = torch.nn.Parameter(torch.randn(40, 16))         # H = 20: no multiple of 8, whatever the map's attributes say
    block.down.weight = torch.nn.Parameter(torch.randn(16, 20))
    assert torch.equal(block(h), _maps(block, h)) and block.calls == []
    block.up.weight = torch.nn.Parameter(torch.randn(32, 16))
    block.down.weight = torch.nn.Parameter(torch.randn(8, 16))        # not as wide as its input
    assert block(h).shape == (5, 8) and block.calls == []
