"""A context without a GPU, for calls that have to be refused before they reach one."""
import ctypes as C


class HostContext:
    """Tensors on the CPU are where it is.  The library gets memory that holds a device and 256 compute units: enough for its checks
    and sizes; a call that passes them would go on to the GPU, so only what has to be refused is called with it."""

    def __init__(self):
        import torch
        from paper_2509_24859_amd import binding
        self.lib = binding.load_library()
        self.device, self.index = torch.device("cpu"), -1
        self.memory = (C.c_int32 * 1024)()
        self.memory[1] = 256
        self.handle = C.cast(self.memory, C.c_void_p)

    def check(self, rc):
        from paper_2509_24859_amd import binding
        if rc != binding.OK:
            raise binding.HarpError(rc, self.lib.harp_last_error(self.handle).decode())


def refused(monkeypatch, call, *a, **k):
    """The call's error code, which must come before the GPU is used."""
    import pytest
    from paper_2509_24859_amd import binding, operators
    monkeypatch.setattr(operators, "_current", lambda ctx: 0)
    with pytest.raises(binding.HarpError) as err:
        call(*a, **k)
    assert err.value.code in (binding.ERR_INVALID_ARG, binding.ERR_SHAPE, binding.ERR_WORKSPACE), err.value
    return err.value.code
