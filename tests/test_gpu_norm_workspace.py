"""The workspace of the norms' backward pass: a pass of many tokens fills it and writes nothing behind it."""
import pytest

from test_gpu_attention import at, dev, normal  # noqa: F401

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D,rotary,tokens", [(64, 64, 5000), (128, 64, 3000), (80, 16, 4000), (72, 8, 900), (512, 512, 700)])        # (72: the kernel for any dimension)
def test_it_is_filled_and_nothing_behind_it_is_written(at, monkeypatch, D, rotary, tokens):  # noqa: F811
    fluxbin, held = at.fluxbin, []
    call = fluxbin.norm_rotary_backward_call

    def guarded(*words):
        *words, _, size, stream = words
        held.append((torch.full((size + 4096,), 255, dtype=torch.uint8, device="cuda"), size))
        call(*words, held[-1][0].data_ptr(), size, stream)

    monkeypatch.setattr(fluxbin, "norm_rotary_backward_call", guarded)
    w = [torch.ones(D, device="cuda", requires_grad=True) for _ in range(2)]
    n = at.NormedRotary(at.Rotary(D, rotary), *w)
    q, k = normal(1, (tokens, 9, D), "bf16"), normal(2, (tokens, 3, D), "bf16")
    y = n.apply(q, k, dev(range(tokens)))
    torch.autograd.grad(y, w, (torch.ones_like(q), torch.ones_like(k)))
    (buffer, size), = held
    assert (buffer[size:] == 255).all()
    assert not (buffer[:size].view(torch.int32) == -1).any()   # (a NaN of all ones: no sum is that)
