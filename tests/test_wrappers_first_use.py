"""The wrappers work whatever of their module was used before: nothing, the library's signatures, or an entry point."""
import pytest
import torch

from paper_2609_37538_amd import fp8 as F
from paper_2609_37538_amd import latent as L
from paper_2609_37538_amd import selection as S


@pytest.mark.parametrize("before", [
    lambda: None, F.load, S.load, L.load, lambda: F.avsg_fp8_quantize(0, 0, 1, 0, 128, 0, 0, F.AvsgFp8()), lambda: S.avsg_select_workspace_least(16, 1)])
def test_first_use(before, monkeypatch):
    """Tensors on the CPU are refused as such."""
    for module in (F, S):
        monkeypatch.setattr(module, "_lib", None)
    monkeypatch.setattr(L, "_t", None)
    before()
    x = torch.zeros(4, 128)
    for call in (lambda: F.fp8_quantize(x), lambda: F.Fp8(x.to(torch.float8_e4m3fn), torch.ones(4, 1)), lambda: L.mx4_quantize(x),
                 lambda: S.KeyCache(torch.zeros(1, 4, 132, dtype=torch.uint8), 1)):
        monkeypatch.setattr(L, "_t", None)
        with pytest.raises(ValueError):
            call()
