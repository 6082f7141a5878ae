"""A plan whose scratch has been closed does not hand the freed handle to the library (no GPU needed)."""
import pytest
import torch

from paper_2507_16768_b200 import binding
from test_beam_binding import FakeBeam, plan
from test_binding_validation import FakeTensor


def test_a_closed_beam_is_no_handle(monkeypatch):
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 0, raising=False)
    seen, real = [], binding._lib

    class Library:
        def __getattr__(self, name):
            return getattr(real, name)

        def wg_beam_select(self, *args):
            seen.append(args[0])
            return 0 if args[0] else real.wg_beam_select(*args)

        def wg_beam_free(self, handle):
            seen.append(("freed", handle))

    monkeypatch.setattr(binding, "_lib", Library())
    p = plan()
    beam = p._beam
    p(FakeTensor((12, 1000), torch.float32))
    binding.Beam.close(beam)
    with pytest.raises(binding.WgError):         # the library itself refuses a missing handle
        p(FakeTensor((12, 1000), torch.float32))
    assert seen == [1, ("freed", 1), None] and isinstance(beam, FakeBeam)
