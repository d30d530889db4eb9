"""Arguments that the operators' binding refuses by itself, before the library is called."""
import pytest


class _Context:
    """Tensors on the CPU are where it is; nothing may be called."""

    def __init__(self, torch):
        self.device, self.index, self.handle, self.lib = torch.device("cpu"), -1, None, None


@pytest.mark.parametrize("per", [0, -1])
@pytest.mark.parametrize("gated", [False, True])
def test_a_gate_s_gradient_needs_rows_for_each_gate(per, gated):
    import torch
    from paper_2509_24859_amd import binding, operators as ops
    t = torch.zeros(6, 8)
    with pytest.raises(binding.HarpError) as err:
        ops.harp_norm_backward(_Context(torch), t, None, None, t, t, t, before="none", dgate=torch.zeros(1, 8),
                               gate=torch.zeros(1, 8) if gated else None, rows_per_gate=per)
    assert err.value.code in (binding.ERR_SHAPE, binding.ERR_INVALID_ARG)


def test_a_gate_s_gradient_needs_a_gate():
    import torch
    from paper_2509_24859_amd import binding, operators as ops
    t = torch.zeros(6, 8)
    with pytest.raises(binding.HarpError) as err:
        ops.harp_norm_backward(_Context(torch), t, None, None, t, t, t, before="none", dgate=torch.zeros(3, 8), rows_per_gate=2)
    assert err.value.code == binding.ERR_INVALID_ARG
