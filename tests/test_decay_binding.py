"""The binding of attention with a decay per head and of the state cache: what it refuses or passes on, without a GPU."""
import pytest
import torch

from tests.test_decay import binding  # noqa: F401


@pytest.mark.parametrize("codes,fmt", [(torch.float8_e4m3fn, "STATE_I8"), (torch.int8, "STATE_E4M3"), (torch.float8_e5m2, "STATE_E4M3"), (torch.bool, "STATE_I8"),
                                       (torch.float8_e5m2, "STATE_I8")])
def test_codes_of_another_format_are_refused(binding, codes, fmt):  # noqa: F811
    S, kept, scales = torch.zeros(2, 3, 8), torch.zeros(2, 3, 8, dtype=codes), torch.zeros(2, 3)
    with pytest.raises(ValueError, match="for this format"):
        binding.darkattn_state_store(S, kept, scales, format=getattr(binding, fmt))
    with pytest.raises(ValueError, match="for this format"):
        binding.darkattn_state_load(kept, scales, S, format=getattr(binding, fmt))


@pytest.mark.gpu
@pytest.mark.parametrize("fmt,own", [(0, torch.int8), (1, torch.float8_e4m3fn)], ids=["i8", "e4m3"])
def test_codes_may_be_plain_bytes(binding, fmt, own):  # noqa: F811
    S = torch.randn(2, 3, 64, device="cuda")
    backs = []
    for dtype in (own, torch.uint8):
        codes, scales, back = torch.zeros(2, 3, 64, dtype=dtype, device="cuda"), torch.zeros(2, 3, device="cuda"), torch.empty_like(S)
        binding.darkattn_state_store(S, codes, scales, format=fmt)
        binding.darkattn_state_load(codes, scales, back, format=fmt)
        backs.append((codes.view(torch.uint8), scales, back))
    assert all(torch.equal(a, b) for a, b in zip(*backs))
    with pytest.raises(binding.DarkAttnError):
        binding.darkattn_state_store(S, codes, scales, format=2)
