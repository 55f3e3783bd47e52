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


class _Recorder:
    """In the library's place: takes what the C interface would be handed."""

    def __init__(self, monkeypatch, binding, name):  # noqa: F811
        self.calls = []
        argtypes = getattr(binding.lib, name).argtypes

        def call(*args):
            self.calls.append([t(a).value if a is not None else None for t, a in zip(argtypes, args)])
            return 0

        monkeypatch.setattr(binding, "lib", type("lib", (), {name: staticmethod(call), "darkattn_decay_destroy": binding.lib.darkattn_decay_destroy})())
        monkeypatch.setattr(binding, "_arg", lambda t, *_: None if t is None else 1 << 20)
        monkeypatch.setattr(binding, "_device", lambda: 0)
        monkeypatch.setattr(binding, "_stream_of", lambda *_: None)


MOST = 2 ** 31 - 1


def test_a_pool_of_more_states_than_int32_counts(monkeypatch, binding):  # noqa: F811
    """Every slot that an int32 can name is one of the pool's."""
    plan = binding.darkattn_decay_plan(2, 1, 1, 1)
    seen = _Recorder(monkeypatch, binding, "darkattn_decay_step")
    row = torch.empty(2, 1, 1, dtype=torch.bfloat16, device="meta")
    for n, want in ((5, 5), (MOST, MOST), (MOST + 1, MOST), (2 ** 32 + 5, MOST)):
        binding.darkattn_decay_step(plan, row, row, row, torch.empty(1, device="meta"), torch.empty(n, 1, 1, 1, device="meta"), row, slots=torch.empty(2, device="meta"))
        assert seen.calls[-1][7] == want, n


@pytest.mark.parametrize("B,rows,cols,n_slots", [(1, 2 ** 32 + 8, 1, 1), (2 ** 32 + 1, 1, 1, 2), (1, 1, 2 ** 32 + 16, 1), (3, 2, 4, 2 ** 32 + 2)])
def test_sizes_of_a_cache_do_not_wrap(monkeypatch, binding, B, rows, cols, n_slots):  # noqa: F811
    for name in ("darkattn_state_store", "darkattn_state_load"):
        with monkeypatch.context() as m:
            seen = _Recorder(m, binding, name)
            S, codes = torch.empty(B, rows, cols, device="meta"), torch.empty(n_slots, rows, cols, dtype=torch.int8, device="meta")
            scales = torch.empty(n_slots, rows, device="meta")
            getattr(binding, name)(*((S, codes, scales) if "store" in name else (codes, scales, S)))
            assert seen.calls[-1][:3] == [min(x, MOST) for x in (B, rows, cols)] and min(n_slots, MOST) in seen.calls[-1]
    # and what large counts get: sizes alone refuse (addresses that nothing is read from)
    if n_slots < MOST:
        far = [1 << 45, 1 << 50, 1 << 55]
        args = [min(x, MOST) for x in (B, rows, cols)]
        assert binding.lib.darkattn_state_store(*args, far[0], None, MOST, 0, far[1], far[2], None) == binding.ERR_UNSUPPORTED
        assert binding.lib.darkattn_state_load(*args, far[1], far[2], None, MOST, 0, far[0], None) == binding.ERR_UNSUPPORTED
