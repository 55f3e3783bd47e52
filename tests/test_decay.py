"""Attention with a decay per head (chunked forward and backward, single-token step) and the 8-bit state cache, against the
recurrence in 64 bits.

Bounds. A result is a sum of products; `mag` is the same sum with every factor's magnitude. With every addition and product off by at
most 2^-23 of its result (tensor cores cut off instead of rounding), n of them in a row are off by n 2^-23 mag: n counts the width of a
score, two chunks of rows, the states handed from chunk to chunk (two operations each) and some for the powers of the decay. bf16 adds half
a step of the output (2^-8 of it), and on the tensor cores the same of each term, since a score times its decay, or the state a row reads, is
rounded to bf16 once."""
import ctypes
import math
from fractions import Fraction

import numpy as np
import pytest
import torch


@pytest.fixture(scope="module")
def binding():
    from paper_2603_04127_b200 import build
    build.build()
    from paper_2603_04127_b200 import binding as b
    return b


NEG_INF = -float("inf")


# ------------------------------------------------------------------------------------------------ the recurrence in 64 bits
def _lam(g):
    return torch.exp(g.double())[:, None, None]


def oracle_forward(q, k, v, g, scale, lengths=None, S=None):
    """O with zeros behind each end, and the states there."""
    B, H, N, d = q.shape
    Hk, dv = k.shape[1], v.shape[3]
    S = torch.zeros(B, Hk, d, dv, dtype=torch.float64) if S is None else S.double().clone()
    O = torch.zeros(B, H, N, dv, dtype=torch.float64)
    n = [N] * B if lengths is None else [min(max(int(x), 0), N) for x in lengths]
    for b in range(B):
        for t in range(n[b]):
            S[b] = torch.where(_lam(g) > 0, _lam(g) * S[b], 0.0) + k[b, :, t, :, None].double() * v[b, :, t, None].double()
            O[b, :, t] = scale * (q[b, :, t].double().reshape(Hk, H // Hk, d) @ S[b]).reshape(H, dv)
    return O, S


def oracle_backward(q, k, v, do, g, scale, lengths=None, S=None, dS=None):
    B, H, N, d = q.shape
    Hk, dv = k.shape[1], v.shape[3]
    G = H // Hk
    S = torch.zeros(B, Hk, d, dv, dtype=torch.float64) if S is None else S.double().clone()
    R = torch.zeros_like(S) if dS is None else dS.double().clone()
    dq, dk, dvv = (torch.zeros(t.shape, dtype=torch.float64) for t in (q, k, v))
    n = [N] * B if lengths is None else [min(max(int(x), 0), N) for x in lengths]
    lam = _lam(g)
    for b in range(B):
        for t in range(n[b]):
            S[b] = lam * S[b] + k[b, :, t, :, None].double() * v[b, :, t, None].double()
            dq[b, :, t] = scale * (do[b, :, t].double().reshape(Hk, G, dv) @ S[b].transpose(-1, -2)).reshape(H, d)
        for t in range(n[b] - 1, -1, -1):
            R[b] = R[b] + scale * q[b, :, t].double().reshape(Hk, G, d).transpose(-1, -2) @ do[b, :, t].double().reshape(Hk, G, dv)
            dk[b, :, t] = (R[b] @ v[b, :, t, :, None].double())[..., 0]
            dvv[b, :, t] = (k[b, :, t, None].double() @ R[b])[..., 0, :]
            R[b] = lam * R[b]
    return dq, dk, dvv, R


def check(got, want, mag, ops, dtype, tensor, what):
    got = got.double().cpu()
    assert torch.isfinite(got).all(), f"{what}: not finite"
    bound = ops * 2.0 ** -23 * mag + 1e-37
    if dtype == torch.bfloat16:
        bound = bound + 2.0 ** -8 * want.abs()
        if tensor:
            bound = bound + (2.0 ** -8 + 2.0 ** -16) * mag
    worst = ((got - want).abs() / bound).max().item()
    assert worst <= 1.0, f"{what}: {worst:.3f} of the bound, off by {(got - want).abs().max().item():.3e}"


def ops_of(d, dv, N):
    return max(d, dv) + 2 * 128 + 4 * (N // 64) + 16


# ------------------------------------------------------------------------------------------------ inputs
def make(B, H, N, d, dv=0, Hk=0, dtype="bf16", seed=1, decays=None, states=True):
    dv, Hk = dv or d, Hk or H
    gen = torch.Generator().manual_seed(seed)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    rnd = lambda *s: torch.randn(*s, generator=gen)  # noqa: E731
    t = {"q": rnd(B, H, N, d).to(dt), "k": rnd(B, Hk, N, d).to(dt), "v": rnd(B, Hk, N, dv).to(dt), "do": rnd(B, H, N, dv).to(dt)}
    t["S"], t["dS"] = (rnd(B, Hk, d, dv) * 3 if states else None for _ in range(2))
    t["g"] = -math.log(2) / torch.exp(math.log(2) + torch.rand(Hk, generator=gen) * 6) if decays is None else torch.tensor([decays[i % len(decays)] for i in range(Hk)])
    t["lengths"] = None
    return t


def dev(t):
    return {k: None if v is None else v.cuda() for k, v in t.items()}


def run_forward(binding, t, path=0, scale=0.0, plan=None, stream=None):
    B, H, N, d = t["q"].shape
    Hk, dv = t["k"].shape[1], t["v"].shape[3]
    plan = plan or binding.darkattn_decay_plan(B, H, N, d, dv=dv, H_kv=Hk, dtype=binding.BF16 if t["q"].dtype == torch.bfloat16 else binding.F32, path=path, scale=scale)
    D = dev(t)
    ws = torch.full((plan.workspace_bytes + 1024,), 0xff, dtype=torch.uint8, device="cuda")
    O = torch.full((B, H, N, dv), 7.0, dtype=t["q"].dtype, device="cuda")
    S_out = torch.full((B, Hk, d, dv), float("nan"), device="cuda")
    binding.darkattn_decay_forward(plan, D["q"], D["k"], D["v"], D["g"], O, ws[:plan.workspace_bytes], lengths=D["lengths"], S_in=D["S"], S_out=S_out)
    assert binding.darkattn_decay_last_device_status(plan, ws) == binding.OK
    assert bool((ws[plan.workspace_bytes:] == 0xff).all())
    return O, S_out


def run_backward(binding, t, path=0, scale=0.0):
    B, H, N, d = t["q"].shape
    Hk, dv = t["k"].shape[1], t["v"].shape[3]
    plan = binding.darkattn_decay_plan(B, H, N, d, dv=dv, H_kv=Hk, dtype=binding.BF16 if t["q"].dtype == torch.bfloat16 else binding.F32, path=path, scale=scale)
    D = dev(t)
    ws = torch.full((plan.workspace_bytes + 1024,), 0xff, dtype=torch.uint8, device="cuda")
    dq, dk, dvv = (torch.full_like(D[x], float("nan")) for x in ("q", "k", "v"))
    dS_in = torch.full((B, Hk, d, dv), float("nan"), device="cuda")
    binding.darkattn_decay_backward(plan, D["q"], D["k"], D["v"], D["g"], D["do"], dq, dk, dvv, ws[:plan.workspace_bytes], lengths=D["lengths"], S_in=D["S"],
                                    dS_out=D["dS"], dS_in=dS_in)
    assert binding.darkattn_decay_last_device_status(plan, ws) == binding.OK
    assert bool((ws[plan.workspace_bytes:] == 0xff).all())
    return dq, dk, dvv, dS_in


def check_forward(binding, t, path=0, scale=None, tag=""):
    B, H, N, d = t["q"].shape
    dv = t["v"].shape[3]
    s = scale or 1 / math.sqrt(d)
    O, S_out = run_forward(binding, t, path, scale or 0.0)
    clean = blank_padding(t)
    want, wS = oracle_forward(clean["q"], clean["k"], clean["v"], t["g"], s, t["lengths"], t["S"])
    mag, mS = oracle_forward(clean["q"].abs(), clean["k"].abs(), clean["v"].abs(), t["g"], s, t["lengths"], None if t["S"] is None else t["S"].abs())
    tensor = path != binding.PATH_SIMT
    n = ops_of(d, dv, N)
    live = alive(t)
    check(torch.where(live, O.cpu().double(), 0.0), want, mag, n, t["q"].dtype, tensor, tag + "O")
    assert bool((torch.where(live, 7.0, O.cpu().double()) == 7).all()), "rows behind the end were touched"
    check(S_out, wS, mS, n, torch.float32, tensor, tag + "S_out")


def check_backward(binding, t, path=0, scale=None, tag=""):
    B, H, N, d = t["q"].shape
    dv = t["v"].shape[3]
    s = scale or 1 / math.sqrt(d)
    got = run_backward(binding, t, path, scale or 0.0)
    clean = blank_padding(t)
    args = [clean[x] for x in ("q", "k", "v", "do")]
    want = oracle_backward(*args, t["g"], s, t["lengths"], t["S"], t["dS"])
    mag = oracle_backward(*(a.abs() for a in args), t["g"], s, t["lengths"], *(None if t[x] is None else t[x].abs() for x in ("S", "dS")))
    tensor = path != binding.PATH_SIMT
    n = ops_of(d, dv, N) * (H // t["k"].shape[1])
    for name, x, w, m in zip(("dQ", "dK", "dV"), got, want, mag):
        check(x, w, m, n, t["q"].dtype, tensor, tag + name)
    check(got[3], want[3], mag[3], n, torch.float32, tensor, tag + "dS_in")


def alive(t):
    N = t["q"].shape[2]
    n = torch.full((t["q"].shape[0],), N) if t["lengths"] is None else t["lengths"].long()
    return (torch.arange(N)[None] < n[:, None])[:, None, :, None]


def blank_padding(t):
    live = alive(t)
    return {x: torch.where(live, t[x].float(), 0.0).to(t[x].dtype) for x in ("q", "k", "v", "do")}


def poison_padding(t):
    """Not-a-numbers and infinities in the rows behind the ends."""
    live = alive(t)
    for i, x in enumerate(("q", "k", "v", "do")):
        t[x] = torch.where(live, t[x].float(), float("nan") if i % 2 else float("inf")).to(t[x].dtype)
    return t


# ------------------------------------------------------------------------------------------------ refusals (no GPU needed)
@pytest.mark.parametrize("kw,status", [(dict(B=0), 1), (dict(H=0), 1), (dict(N=0), 1), (dict(d=0), 1), (dict(dv=-1), 1), (dict(dtype=5), 1), (dict(path=7), 1),
                                       (dict(H_kv=3), 1), (dict(H_kv=16), 1), (dict(scale=-1.0), 1), (dict(scale=float("nan")), 1), (dict(d=513), 2),
                                       (dict(dv=520), 2), (dict(B=65536), 2), (dict(path=2, dtype=0), 2), (dict(path=2, d=200), 2), (dict(path=2, d=63), 2)])
def test_bad_descriptors(binding, kw, status):
    args = dict(B=1, H=8, N=100, d=64)
    args.update(kw)
    with pytest.raises(binding.DarkAttnError) as e:
        binding.darkattn_decay_plan(args.pop("B"), args.pop("H"), args.pop("N"), args.pop("d"), **args)
    assert e.value.status == status


def test_plan_sizes(binding):
    one = binding.darkattn_decay_plan(64, 16, 512, 64)
    assert one.workspace_bytes >= 256 and one.workspace_bytes % 256 == 0
    long = binding.darkattn_decay_plan(1, 4, 1 << 20, 128, dtype=binding.F32)
    assert 256 < long.workspace_bytes < 1 << 30 and long.path == binding.PATH_SIMT
    for p in (one, long):
        p.destroy()


def test_calls_refuse_before_launch(binding):
    p = binding.darkattn_decay_plan(2, 4, 100, 64, dtype=binding.F32)
    lib, a, odd = binding.lib, 1 << 20, (1 << 20) + 4
    far = 1 << 30
    fwd = lambda *x: lib.darkattn_decay_forward(p.handle, *x)  # noqa: E731
    ok = [a, a, a, a, None, None, a, None, a, None]
    for i in (0, 1, 2, 6):
        assert fwd(*[None if j == i else x for j, x in enumerate(ok)]) == binding.ERR_INVALID_ARG
        assert fwd(*[odd if j == i else x for j, x in enumerate(ok)]) == binding.ERR_INVALID_ARG
    assert fwd(a, a, a, None, None, None, a, None, a, None) == binding.ERR_INVALID_ARG
    assert fwd(a, a, a, a, None, None, a, None, None, None) == binding.ERR_WORKSPACE
    assert fwd(a, a, a, a, None, far, a, far + 16, a, None) == binding.ERR_INVALID_ARG          # S_out over S_in
    assert fwd(a, a, a, a + 2, None, None, a, None, a, None) == binding.ERR_INVALID_ARG
    assert lib.darkattn_decay_forward(None, *ok) == binding.ERR_INVALID_ARG
    bwd = lambda *x: lib.darkattn_decay_backward(p.handle, *x)  # noqa: E731
    ok = [a, a, a, a, None, None, a, None, a, a, a, None, a, None]
    for i in (0, 1, 2, 3, 6, 8, 9, 10):
        assert bwd(*[None if j == i else x for j, x in enumerate(ok)]) == binding.ERR_INVALID_ARG
    assert bwd(*(ok[:12] + [None, None])) == binding.ERR_WORKSPACE
    for other in (5, 7):
        x = list(ok)
        x[other], x[11] = far, far + 64
        assert bwd(*x) == binding.ERR_INVALID_ARG
    step = lambda *x: lib.darkattn_decay_step(p.handle, *x)  # noqa: E731
    assert step(a, a, a, a, None, None, 2, a, None) == binding.ERR_INVALID_ARG
    assert step(a, a, a, a, a, None, 1, a, None) == binding.ERR_INVALID_ARG                      # fewer states than rows
    assert step(a, a, a, a, a, a, 0, a, None) == binding.ERR_INVALID_ARG
    wide = binding.darkattn_decay_plan(1, 128, 1, 256, H_kv=1)
    assert lib.darkattn_decay_step(wide.handle, a, a, a, a, a, None, 1, a, None) == binding.ERR_UNSUPPORTED
    store, load = lib.darkattn_state_store, lib.darkattn_state_load
    assert store(0, 8, 8, a, None, 4, 0, a, a, None) == binding.ERR_INVALID_ARG
    assert store(5, 8, 8, a, None, 4, 0, a, a, None) == binding.ERR_INVALID_ARG
    assert store(2, 8, 8, a, None, 4, 2, a, a, None) == binding.ERR_INVALID_ARG
    assert store(2, 8, 8, odd, None, 4, 0, a, a, None) == binding.ERR_INVALID_ARG
    assert store(70000, 8, 8, a, None, 70000, 0, a, a, None) == binding.ERR_UNSUPPORTED
    assert load(2, 8, 0, a, a, None, 4, 0, a, None) == binding.ERR_INVALID_ARG
    assert load(2, 8, 8, a, None, None, 4, 0, a, None) == binding.ERR_INVALID_ARG
    for x in (p, wide):
        x.destroy()


def test_arrays_that_overlap_are_refused(binding):
    p = binding.darkattn_decay_plan(2, 4, 100, 64, H_kv=2)
    lib = binding.lib
    at = [(i + 1) << 24 for i in range(14)]                     # no two of them overlap; each is refused before anything is launched
    rows = 2 * 4 * 100 * 64 * 2
    fwd = [*at[:4], None, at[4], at[5], at[6], at[7], None]     # Q K V log_decay lengths S_in O S_out workspace
    for out in (6, 7, 8):
        for other in (0, 1, 2, 3, 5, 6, 7, 8):
            if out != other:
                x = list(fwd)
                x[out] = x[other] + 16 if other != 3 else x[other]
                assert lib.darkattn_decay_forward(p.handle, *x) == binding.ERR_INVALID_ARG, (out, other)
    x = list(fwd)
    x[6] = x[0] - rows + 16                                     # from below
    assert lib.darkattn_decay_forward(p.handle, *x) == binding.ERR_INVALID_ARG
    bwd = [*at[:4], None, *at[4:12], None]                      # Q K V log_decay lengths S_in dO dS_out dQ dK dV dS_in workspace
    for out in range(8, 13):
        for other in (0, 1, 2, 3, 5, 6, 7, 8, 9, 10, 11, 12):
            if out != other:
                x = list(bwd)
                x[out] = x[other]
                assert lib.darkattn_decay_backward(p.handle, *x) == binding.ERR_INVALID_ARG, (out, other)
    step = [*at[:5], at[5], 2, at[6], None]                     # q k v log_decay S slots n_slots o
    for out in (4, 7):
        for other in (0, 1, 2, 3, 4, 5, 7):
            if out != other:
                x = list(step)
                x[out] = x[other]
                assert lib.darkattn_decay_step(p.handle, *x) == binding.ERR_INVALID_ARG, (out, other)
    a, b, c, s = at[:4]
    for x in ((a, s, a, c), (a, s, b, a), (a, s, s, c), (a, s, b, s), (a, s, b, b)):
        assert lib.darkattn_state_store(2, 8, 8, x[0], x[1], 4, 0, x[2], x[3], None) == binding.ERR_INVALID_ARG
    for x in ((b, c, s, b), (b, c, s, c), (b, c, s, s)):
        assert lib.darkattn_state_load(2, 8, 8, x[0], x[1], x[2], 4, 0, x[3], None) == binding.ERR_INVALID_ARG
    p.destroy()


@pytest.mark.parametrize("rows,cols", [((1 << 30) + 1, 1), (2 ** 31 - 1, 8), (1, (1 << 30) + 1), (1, 2 ** 31 - 1)])
def test_cache_sizes_whose_indices_would_wrap_are_refused(binding, rows, cols):
    a, b, c = 1 << 45, 1 << 46, 1 << 47
    assert binding.lib.darkattn_state_store(1, rows, cols, a, None, 1, 0, b, c, None) == binding.ERR_UNSUPPORTED
    assert binding.lib.darkattn_state_load(1, rows, cols, b, c, None, 1, 0, a, None) == binding.ERR_UNSUPPORTED


def test_the_oracle_is_the_quadratic_form():
    t = make(2, 4, 37, 6, dv=5, Hk=2, dtype="f32")
    q, k, v = (t[x].double() for x in ("q", "k", "v"))
    i = torch.arange(37)
    D = torch.where(i[:, None] >= i, torch.exp(t["g"].double()[:, None, None] * (i[:, None] - i)), 0.0).repeat_interleave(2, 0)
    kk, vv = k.repeat_interleave(2, 1), v.repeat_interleave(2, 1)
    first = torch.exp(t["g"].double()[:, None] * (i + 1)).repeat_interleave(2, 0)[..., None]
    want = 0.3 * ((q @ kk.transpose(-1, -2) * D) @ vv + first * (q @ t["S"].double().repeat_interleave(2, 1)))
    got, _ = oracle_forward(t["q"], t["k"], t["v"], t["g"], 0.3, S=t["S"])
    assert torch.allclose(got, want, rtol=1e-12, atol=1e-12)


def test_the_gradients_are_the_oracles_differences():
    """L is linear in Q, K, V and the state each: a central difference of any step is the gradient."""
    t = make(1, 4, 21, 5, dv=4, Hk=2, dtype="f32")
    grads = dict(zip(("q", "k", "v", "S"), oracle_backward(t["q"], t["k"], t["v"], t["do"], t["g"], 0.5, S=t["S"], dS=t["dS"])))

    def loss(**kw):
        x = {**t, **kw}
        O, S = oracle_forward(x["q"].double(), x["k"].double(), x["v"].double(), t["g"], 0.5, S=x["S"])
        return (O * t["do"].double()).sum() + (S * t["dS"].double()).sum()

    for name, grad in grads.items():
        step = torch.randn(t[name].shape, generator=torch.Generator().manual_seed(5), dtype=torch.float64)
        diff = (loss(**{name: t[name].double() + step}) - loss(**{name: t[name].double() - step})) / 2
        assert abs(diff - (grad * step).sum()) < 1e-9 * (1 + abs(diff)), name


# ------------------------------------------------------------------------------------------------ chunked form on the GPU
SHAPES = [                                     # B, H, N, d, dv, H_kv
    (1, 1, 1, 8, 8, 1), (2, 2, 2, 5, 3, 2), (1, 2, 63, 16, 72, 1), (1, 3, 64, 65, 64, 3), (2, 4, 65, 64, 64, 2), (1, 2, 127, 128, 128, 2),
    (1, 2, 128, 64, 128, 1), (2, 1, 129, 128, 64, 1), (1, 6, 257, 80, 96, 3), (2, 2, 700, 40, 8, 2), (1, 1, 1500, 64, 64, 1), (1, 2, 300, 200, 130, 1),
    (1, 16, 300, 64, 64, 1), (2, 8, 150, 128, 128, 1), (1, 2, 150, 97, 33, 1), (1, 1, 90, 100, 92, 1), (3, 1, 1100, 72, 128, 1), (1, 2, 640, 512, 24, 2),
]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_forward(binding, shape, dtype):
    B, H, N, d, dv, Hk = shape
    for path in (binding.PATH_SIMT, binding.PATH_AUTO):
        check_forward(binding, make(B, H, N, d, dv, Hk, dtype, seed=N), path, tag=f"path {path}: ")


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_backward(binding, shape, dtype):
    B, H, N, d, dv, Hk = shape
    for path in (binding.PATH_SIMT, binding.PATH_AUTO):
        check_backward(binding, make(B, H, N, d, dv, Hk, dtype, seed=N + 1), path, tag=f"path {path}: ")


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d,dv", [(64, 64), (128, 128), (24, 80)])
def test_padded_batches(binding, dtype, d, dv):
    """Ends at none, one, inside and at the ends of chunks, beyond the array; what stands behind them is never used."""
    t = make(9, 2, 400, d, dv, 1, dtype, seed=3)
    t["lengths"] = torch.tensor([0, 1, 63, 64, 65, 128, 200, 257, 400], dtype=torch.int32)
    poison_padding(t)
    for path in (binding.PATH_SIMT, binding.PATH_AUTO):
        check_forward(binding, t, path)
        check_backward(binding, t, path)
    odd = dict(t, lengths=torch.tensor([-3, 1, 63, 64, 65, 128, 200, 257, 9999], dtype=torch.int32))
    assert torch.equal(run_forward(binding, odd)[0].nan_to_num(0), run_forward(binding, t)[0].nan_to_num(0))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("decays", [(0.0,), (NEG_INF, -1.0), (-30.0, -1e-5), (-0.7, -200.0)], ids=str)
def test_strong_and_absent_decays(binding, dtype, decays):
    t = make(1, 4, 333, 64, 64, 2, dtype, seed=9, decays=decays)
    for path in (binding.PATH_SIMT, binding.PATH_AUTO):
        check_forward(binding, t, path)
        check_backward(binding, t, path)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_without_states_and_with_a_scale(binding, dtype):
    t = make(2, 4, 200, 64, 64, 4, dtype, seed=11, states=False)
    for path in (binding.PATH_SIMT, binding.PATH_AUTO):
        check_forward(binding, t, path, scale=2.5)
        check_backward(binding, t, path, scale=2.5)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,shape", [("bf16", (2, 1, 3000, 64, 64, 1)), ("bf16", (2, 2, 2100, 128, 40, 1)), ("bf16", (4, 12, 140, 128, 64, 12)), ("bf16", (4, 16, 140, 64, 96, 4)),
                                         ("f32", (2, 1, 1700, 63, 65, 1)), ("f32", (2, 2, 1300, 128, 96, 2)), ("f32", (2, 2, 300, 200, 136, 1)), ("bf16", (2, 2, 300, 136, 129, 2))],
                         ids=str)
def test_padded_batches_in_segments_and_of_mixed_widths(binding, dtype, shape):
    """Ends inside, at and before the segments' ends; more than one wave of blocks and widths of two classes; rows of no whole number of 16 bytes."""
    B, H, N, d, dv, Hk = shape
    t = make(B, H, N, d, dv, Hk, dtype, seed=70 + N)
    for lengths in ([N, 0], [N * 3 // 5, 130], [N - 1, 1]):
        t["lengths"] = torch.tensor([lengths[i % 2] for i in range(B)], dtype=torch.int32)
        poisoned = poison_padding(dict(t))
        check_forward(binding, poisoned, tag=f"{lengths} ")
        check_backward(binding, poisoned, tag=f"{lengths} ")


@pytest.mark.gpu
@pytest.mark.parametrize("d,dv", [(64, 64), (128, 64), (128, 128)])
def test_long_sequences_of_many_heads(binding, d, dv):
    """Many chunks by one block, all stages in use: the same rows as the heads give by themselves, where they are cut into segments."""
    B, H, N = 2, 80, 4100
    gen = torch.Generator(device="cuda").manual_seed(5)
    rnd = lambda *s: torch.randn(*s, generator=gen, device="cuda").bfloat16()  # noqa: E731
    q, k, v = rnd(B, H, N, d), rnd(B, H, N, d), rnd(B, H, N, dv)
    g = torch.full((H,), -0.004, device="cuda")

    def forward(q, k, v, g):
        plan = binding.darkattn_decay_plan(*q.shape, dv=dv)
        ws = plan.alloc_workspace()
        O = torch.empty(*v.shape, dtype=q.dtype, device="cuda")
        binding.darkattn_decay_forward(plan, q, k, v, g, O, ws)
        assert binding.darkattn_decay_last_device_status(plan, ws) == binding.OK
        return O, plan.workspace_bytes

    whole, one = forward(q, k, v, g)
    part, some = forward(q[1:, 77:78].contiguous(), k[1:, 77:78].contiguous(), v[1:, 77:78].contiguous(), g[77:78])
    assert one == 256 < some
    # either is off by at most half a step for the rows out, for each score and for the state's copy
    mag, _ = oracle_forward(*(x[1:, 77:78].float().abs().cpu() for x in (q, k, v)), g[77:78].cpu(), 1 / math.sqrt(d))
    bound = 2 * (2.0 ** -8 * part.float().abs().cpu() + (2.0 ** -8 + 2.0 ** -16 + ops_of(d, dv, N) * 2.0 ** -23) * mag)
    assert ((whole[1:, 77:78].double() - part.double()).abs().cpu() <= bound).all()
    again, _ = forward(q, k, v, g)
    assert torch.equal(again, whole)


@pytest.mark.gpu
@pytest.mark.parametrize("d,dv", [(64, 64), (128, 128), (80, 64), (40, 128)])
def test_few_rows_are_rounded_once(binding, d, dv):
    """Up to 32 tokens: the scores as two bf16 parts, which leave 2^-16 of each; beside that the rows' own rounding alone."""
    for N in (1, 2, 3, 17, 31, 32):
        t = make(3, 4, N, d, dv, 2, "bf16", seed=40 + N, states=False)
        t["lengths"] = torch.tensor([N, 1, max(N - 1, 0)], dtype=torch.int32)
        s = 1 / math.sqrt(d)
        clean, live = blank_padding(t), alive(t)
        args = [clean[x] for x in ("q", "k", "v", "do")]
        O, _ = run_forward(binding, poison_padding(dict(t)))
        n = ops_of(d, dv, N) + 2 ** 7
        want, _ = oracle_forward(*args[:3], t["g"], s, t["lengths"], None)
        mag, _ = oracle_forward(*(a.abs() for a in args[:3]), t["g"], s, t["lengths"], None)
        check(torch.where(live, O.cpu().double(), 0.0), want, mag, n, torch.bfloat16, False, f"{N} O")
        got = run_backward(binding, poison_padding(dict(t)))
        want = oracle_backward(*args, t["g"], s, t["lengths"], None, None)
        mag = oracle_backward(*(a.abs() for a in args), t["g"], s, t["lengths"], None, None)
        for name, x, w, m in zip(("dQ", "dK", "dV"), got, want, mag):
            check(x, w, m, 2 * n, torch.bfloat16, False, f"{N} {name}")


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_segments_do_not_change_the_result(binding, dtype):
    """One head is cut into segments, the same head among many is not."""
    t = make(1, 1, 2500, 64, 64, 1, dtype, seed=12, decays=(-0.002,))
    many = {k: None if v is None else (v.repeat(300, 1, 1, 1) if v.dim() == 4 else v) for k, v in t.items()}
    n = ops_of(64, 64, 2500)
    mag, mS = oracle_forward(t["q"].abs(), t["k"].abs(), t["v"].abs(), t["g"], 0.125, None, t["S"].abs())
    for path in (binding.PATH_SIMT, binding.PATH_AUTO):
        O, S = run_forward(binding, t, path)
        O2, S2 = run_forward(binding, many, path)
        check(O[:1], O2[:1].double().cpu(), mag, 2 * n, t["q"].dtype, True, "O")
        check(S[:1], S2[:1].double().cpu(), mS, 2 * n, torch.float32, True, "S")
        assert torch.equal(O2[0], O2[299]) and torch.equal(S2[0], S2[123])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_two_calls_are_bitwise_alike(binding, dtype):
    t = make(2, 4, 900, 128, 128, 2, dtype, seed=13)
    for run in (run_forward, run_backward):
        assert all(torch.equal(a, b) for a, b in zip(run(binding, t), run(binding, t)))


@pytest.mark.gpu
@pytest.mark.parametrize("name", ["q", "k", "v", "S"])
def test_gradients_are_differences(binding, name):
    """L is linear in each argument: the difference over any step is the gradient. fp32: each loss is a sum of `mag` at most, off by
    ops 2^-23 of it; the sums over the outputs are taken in 64 bits."""
    t = make(1, 4, 260, 32, 24, 2, "f32", seed=14)
    grads = dict(zip(("q", "k", "v", "S"), run_backward(binding, t)))
    step = torch.randn(t[name].shape, generator=torch.Generator().manual_seed(5))

    def loss(x):
        O, S = run_forward(binding, x)
        return (O.double().cpu() * t["do"].double()).sum() + (S.double().cpu() * t["dS"].double()).sum()

    up, down = dict(t, **{name: t[name] + step}), dict(t, **{name: t[name] - step})
    diff = (loss(up) - loss(down)) / 2
    exact = ((up[name].double() - down[name].double()) / 2 * grads[name].double().cpu()).sum()
    big = {k: None if v is None or k == "lengths" else v.abs() for k, v in t.items()}
    big[name] = big[name] + step.abs()
    mO, mS = oracle_forward(big["q"], big["k"], big["v"], t["g"], 1 / math.sqrt(32), None, big["S"])
    mag = (mO * big["do"].double()).sum() + (mS * big["dS"].double()).sum()
    assert abs(diff - exact) <= 3 * ops_of(32, 24, 260) * 2.0 ** -23 * mag


# ------------------------------------------------------------------------------------------------ single tokens
STEPS = [(1, 1, 1, 1, 1), (3, 4, 5, 3, 2), (2, 8, 64, 64, 2), (5, 4, 128, 128, 4), (2, 2, 80, 100, 1), (1, 6, 300, 36, 1), (40, 16, 64, 128, 16)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", STEPS, ids=str)
def test_step(binding, shape, dtype):
    B, H, d, dv, Hk = shape
    t = make(B, H, 1, d, dv, Hk, dtype, seed=20 + B)
    D = dev(t)
    plan = binding.darkattn_decay_plan(B, H, 1, d, dv=dv, H_kv=Hk, dtype=binding.BF16 if dtype == "bf16" else binding.F32)
    pool = torch.full((B + 2, Hk, d, dv), 5.0, device="cuda")
    slots = torch.randperm(B + 2, generator=torch.Generator().manual_seed(3))[:B].to(torch.int32)
    for sl in (slots, None):
        at = slots.long() if sl is not None else torch.arange(B)
        pool.fill_(5.0)
        pool[at.cuda()] = D["S"]
        o = torch.full((B, H, dv), float("nan"), dtype=t["q"].dtype, device="cuda")
        binding.darkattn_decay_step(plan, D["q"][:, :, 0].contiguous(), D["k"][:, :, 0].contiguous(), D["v"][:, :, 0].contiguous(), D["g"], pool, o,
                                    slots=None if sl is None else sl.cuda())
        s = 1 / math.sqrt(d)
        want, wS = oracle_forward(t["q"], t["k"], t["v"], t["g"], s, None, t["S"])
        mag, mS = oracle_forward(t["q"].abs(), t["k"].abs(), t["v"].abs(), t["g"], s, None, t["S"].abs())
        check(o, want[:, :, 0], mag[:, :, 0], d + 8, t["q"].dtype, False, "o")
        check(pool[at.cuda()], wS, mS, 4, torch.float32, False, "S")
        rest = torch.ones(B + 2, dtype=torch.bool)
        rest[at] = False
        assert bool((pool[rest.cuda()] == 5.0).all())


@pytest.mark.gpu
def test_step_leaves_padding_alone(binding):
    B, H, d = 6, 2, 64
    t = dev(make(B, H, 1, d, seed=30))
    plan = binding.darkattn_decay_plan(B, H, 1, d)
    pool = t["S"].clone()
    slots = torch.tensor([2, -1, 0, 2, 6, 5], dtype=torch.int32, device="cuda")        # row 3 names row 0's slot again
    o = torch.full((B, H, d), 9.0, dtype=torch.bfloat16, device="cuda")
    args = [t[x][:, :, 0].contiguous() for x in ("q", "k", "v")]
    binding.darkattn_decay_step(plan, *args, t["g"], pool, o, slots=slots)
    assert bool((o[[1, 3, 4]] == 9).all()) and not bool((o[[0, 2, 5]] == 9).all(-1).all(-1).any())
    assert torch.equal(pool[[1, 3, 4]], t["S"][[1, 3, 4]])
    alone, o2 = t["S"].clone(), torch.empty_like(o)
    clean = torch.tensor([2, -1, 0, -1, -1, 5], dtype=torch.int32, device="cuda")
    binding.darkattn_decay_step(plan, *args, t["g"], alone, o2, slots=clean)
    assert torch.equal(pool, alone) and torch.equal(o[[0, 2, 5]], o2[[0, 2, 5]])


# ------------------------------------------------------------------------------------------------ 8-bit cache
def e4m3_values():
    v = []
    for c in range(127):                       # 0x7f is not a number
        e, m = c >> 3, c & 7
        v.append(Fraction(m, 8) * Fraction(2) ** -6 if e == 0 else (1 + Fraction(m, 8)) * Fraction(2) ** (e - 7))
    return v


E4M3 = e4m3_values()


def nearest_code(x, scale, fmt):
    """The code of x / scale by exact arithmetic."""
    if scale == 0:
        return 0
    u = Fraction(float(x)) / Fraction(float(scale))
    if fmt == 0:
        return max(-127, min(127, round(u))) & 0xff          # Fraction rounds ties to even
    a = abs(u)
    lo = max(i for i in range(127) if E4M3[i] <= a) if a <= 448 else 126
    if lo < 126:
        below, above = a - E4M3[lo], E4M3[lo + 1] - a
        if above < below or (above == below and lo & 1):
            lo += 1
    return lo | (0x80 if float(x) < 0 else 0)


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", [0, 1], ids=["i8", "e4m3"])
@pytest.mark.parametrize("rows,cols", [(3, 1), (5, 7), (4, 40), (33, 128), (2, 200), (3, 260), (2, 513)])
def test_codes_are_the_nearest(binding, fmt, rows, cols):
    gen = torch.Generator().manual_seed(rows + cols)
    S = torch.randn(2, rows, cols, generator=gen) * torch.exp(3 * torch.randn(2, rows, 1, generator=gen))
    S[0, 0] = 0                                                                  # a row of zeros
    top = 127.0 if fmt == 0 else 448.0
    S[1, 1] = torch.tensor([(top if i == 0 else (i % 60) + 0.5) for i in range(cols)])        # exact ties (scale 1)
    if cols > 2:                                                                 # next to ties, on either side
        base = torch.tensor([(i % 50) + 0.5 for i in range(cols)]) * 3.0
        S[1, 2 % rows] = torch.nextafter(base, base + torch.tensor([(-1.0) ** i for i in range(cols)]))
        S[1, 2 % rows, 0] = 3 * top
    dt = torch.int8 if fmt == 0 else torch.float8_e4m3fn
    codes, scales = torch.zeros(5, rows, cols, dtype=dt, device="cuda"), torch.full((5, rows), -1.0, device="cuda")
    slots = torch.tensor([4, 1], dtype=torch.int32, device="cuda")
    binding.darkattn_state_store(S.cuda(), codes, scales, slots=slots, format=fmt)
    raw, sc = codes.view(torch.uint8).cpu(), scales.cpu()
    for b, slot in ((0, 4), (1, 1)):
        for r in range(rows):
            s = np.float32(S[b, r].abs().max().numpy()) / np.float32(top)
            assert sc[slot, r].item() == float(s)
            want = [nearest_code(x, s, fmt) for x in S[b, r].tolist()]
            got = raw[slot, r].tolist()
            assert [g if fmt == 0 or g != 0x80 else 0 for g in got] == [w if fmt == 0 or w != 0x80 else 0 for w in want]
    rest = [0, 2, 3]
    assert bool((sc[rest] == -1).all()) and not raw[rest].any()
    back = torch.full((2, rows, cols), 7.0, device="cuda")
    binding.darkattn_state_load(codes, scales, back, slots=slots, format=fmt)
    value = codes.view(torch.int8).cpu().float() if fmt == 0 else codes.cpu().float()
    assert torch.equal(back.cpu(), (value * sc[..., None])[[4, 1]])


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", [0, 1], ids=["i8", "e4m3"])
def test_cache_rows_that_are_not_finite_tiny_or_padding(binding, fmt):
    S = torch.randn(5, 4, 64)
    S[0, 0, 3], S[0, 1, 5], S[0, 2, 7] = float("inf"), float("nan"), -float("inf")
    S[1, 0], S[1, 1] = 1e-45, torch.randn(64) * 1e-39
    S[1, 2, 0], S[1, 2, 1:] = 3e38, 1e-30
    codes = torch.zeros(4, 4, 64, dtype=torch.int8 if fmt == 0 else torch.float8_e4m3fn, device="cuda")
    scales = torch.zeros(4, 4, device="cuda")
    slots = torch.tensor([0, 3, -1, 0, 4], dtype=torch.int32, device="cuda")     # rows 2 and 4 are padding, row 3 names row 0's slot again
    binding.darkattn_state_store(S.cuda(), codes, scales, slots=slots, format=fmt)
    back = torch.full((5, 4, 64), 7.0, device="cuda")
    binding.darkattn_state_load(codes, scales, back, slots=slots, format=fmt)
    back = back.cpu()
    assert back[0, :3].isnan().all() and torch.equal(back[3].nan_to_num(5), back[0].nan_to_num(5)) and bool((back[[2, 4]] == 7).all())
    step = 1 / 254 if fmt == 0 else 2.0 ** -4
    assert ((back[0, 3] - S[0, 3]).abs() <= step * 1.0001 * S[0, 3].abs().max()).all()
    assert torch.isfinite(back[1]).all() and back[1, 2, 0] == pytest.approx(3e38, rel=1e-6)
    # denormal scales are whole steps of 2^-149: off by half a step of 127 (448) codes at most, beside the code's own half step
    assert ((back[1, :2] - S[1, :2]).abs() <= (224 + 0.5) * 2.0 ** -149 + step * S[1, :2].abs().amax(-1, keepdim=True)).all()


# ------------------------------------------------------------------------------------------------ together
@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_prompt_cache_and_steps_continue_one_another(binding, dtype):
    """A prompt, its state into the cache and back, a second prompt from there, then tokens one by one: as the oracle does from the state
    that was read back, and near to one long prompt."""
    B, H, Hk, N, M, T, d = 3, 4, 2, 150, 70, 4, 64
    t = make(B, H, N + M + T, d, d, Hk, dtype, seed=40, states=False)
    D = dev(t)
    kind = binding.BF16 if dtype == "bf16" else binding.F32
    cut = lambda x, i, j: D[x][:, :, i:j].contiguous()  # noqa: E731
    S, pool = torch.empty(B, Hk, d, d, device="cuda"), torch.zeros(B + 1, Hk, d, d, device="cuda")
    p1, p2, p3 = (binding.darkattn_decay_plan(B, H, n, d, H_kv=Hk, dtype=kind) for n in (N, M, 1))
    O1, O2 = (torch.empty(B, H, n, d, dtype=t["q"].dtype, device="cuda") for n in (N, M))
    binding.darkattn_decay_forward(p1, cut("q", 0, N), cut("k", 0, N), cut("v", 0, N), D["g"], O1, p1.alloc_workspace(), S_out=S)
    codes, scales = torch.empty(B + 2, Hk, d, d, dtype=torch.int8, device="cuda"), torch.empty(B + 2, Hk, d, device="cuda")
    where = torch.tensor([3, 0, 4], dtype=torch.int32, device="cuda")
    binding.darkattn_state_store(S, codes, scales, slots=where)
    kept = torch.empty_like(S)
    binding.darkattn_state_load(codes, scales, kept, slots=where)
    binding.darkattn_decay_forward(p2, cut("q", N, N + M), cut("k", N, N + M), cut("v", N, N + M), D["g"], O2, p2.alloc_workspace(), S_in=kept, S_out=S)
    slots = torch.tensor([1, 3, 0], dtype=torch.int32, device="cuda")
    pool[slots.long()] = S
    outs = []
    for i in range(N + M, N + M + T):
        o = torch.empty(B, H, d, dtype=t["q"].dtype, device="cuda")
        binding.darkattn_decay_step(p3, cut("q", i, i + 1)[:, :, 0].contiguous(), cut("k", i, i + 1)[:, :, 0].contiguous(), cut("v", i, i + 1)[:, :, 0].contiguous(),
                                    D["g"], pool, o, slots=slots)
        outs.append(o)
    got = torch.cat([O2] + [o[:, :, None] for o in outs], 2)
    rest = [t[x][:, :, N:] for x in ("q", "k", "v")]
    want, _ = oracle_forward(*rest, t["g"], 0.125, None, kept.cpu())
    mag, _ = oracle_forward(*(x.abs() for x in rest), t["g"], 0.125, None, kept.cpu().abs())
    check(got, want, mag, ops_of(d, d, M + T), t["q"].dtype, True, "continued")
    # one long prompt differs by what the codes left out: at most 1/254 of a row's largest number in each of its d rows
    whole, _ = oracle_forward(t["q"], t["k"], t["v"], t["g"], 0.125)
    first, S1 = oracle_forward(*(t[x][:, :, :N] for x in ("q", "k", "v")), t["g"], 0.125)
    off, _ = oracle_forward(rest[0].abs(), torch.zeros_like(rest[1]), torch.zeros_like(rest[2]), t["g"], 0.125, None,
                            (S1.abs().amax(-1, keepdim=True) / 254).expand(-1, -1, -1, d))
    n = ops_of(d, d, N + M + T)
    bound = 1.01 * off + (2.0 ** -8 + 2.0 ** -8 + n * 2.0 ** -22) * oracle_forward(*(t[x].abs() for x in ("q", "k", "v")), t["g"], 0.125)[0][:, :, N:]
    assert ((got.cpu().double() - whole[:, :, N:]).abs() <= bound).all()
    check(O1, first, oracle_forward(*(t[x][:, :, :N].abs() for x in ("q", "k", "v")), t["g"], 0.125)[0], n, t["q"].dtype, True, "first prompt")


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_captured_calls_on_a_side_stream(binding, dtype):
    """Prompt, backward pass, store, load and step captured into one graph and replayed on changed inputs; a second graph on the same
    workspace, replayed in turn, changes nothing."""
    B, H, N, d = 2, 4, 500, 64
    kind = binding.BF16 if dtype == "bf16" else binding.F32
    plan, one = binding.darkattn_decay_plan(B, H, N, d, dtype=kind), binding.darkattn_decay_plan(B, H, 1, d, dtype=kind)
    ws = plan.alloc_workspace()
    sets = [dev(make(B, H, N, d, dtype=dtype, seed=s)) for s in (50, 51, 52)]
    for x in sets:
        x["lengths"] = torch.tensor([N, 211], dtype=torch.int32, device="cuda")
    live = {k: v.clone() for k, v in sets[0].items()}

    def buffers():
        return {"O": torch.zeros_like(live["q"]), "dq": torch.zeros_like(live["q"]), "dk": torch.zeros_like(live["k"]), "dv": torch.zeros_like(live["v"]),
                "S": torch.zeros_like(live["S"]), "dS": torch.zeros_like(live["S"]), "back": torch.zeros_like(live["S"]), "o": torch.zeros_like(live["q"][:, :, 0]).contiguous(),
                "codes": torch.zeros(live["S"].shape, dtype=torch.int8, device="cuda"), "scales": torch.zeros(live["S"].shape[:-1], device="cuda")}

    token = [live[x][:, :, 0].contiguous() for x in "qkv"]

    def calls(out):
        binding.darkattn_decay_forward(plan, live["q"], live["k"], live["v"], live["g"], out["O"], ws, lengths=live["lengths"], S_in=live["S"], S_out=out["S"])
        binding.darkattn_decay_backward(plan, live["q"], live["k"], live["v"], live["g"], live["do"], out["dq"], out["dk"], out["dv"], ws, lengths=live["lengths"],
                                        S_in=live["S"], dS_out=live["dS"], dS_in=out["dS"])
        binding.darkattn_state_store(out["S"], out["codes"], out["scales"])
        binding.darkattn_state_load(out["codes"], out["scales"], out["back"])
        binding.darkattn_decay_step(one, *token, live["g"], out["back"], out["o"])

    a, b = buffers(), buffers()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graphs = []
    with torch.cuda.stream(side):
        calls(a)
        for out in (a, b):
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                calls(out)
            graphs.append(graph)
    torch.cuda.synchronize()
    for x in sets[1:]:
        for k in live:
            live[k].copy_(x[k])
        graphs[0].replay()
        graphs[1].replay()
        torch.cuda.synchronize()
        eager = buffers()
        calls(eager)
        torch.cuda.synchronize()
        for k in eager:
            assert torch.equal(eager[k], a[k]) and torch.equal(a[k], b[k]), k


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_two_calls_at_once(binding, dtype):
    """Two streams, a plan and a workspace each (and one plan for both): what each does by itself."""
    kind = binding.BF16 if dtype == "bf16" else binding.F32
    plan = binding.darkattn_decay_plan(2, 4, 3000, 64, dtype=kind)
    sets = [dev(make(2, 4, 3000, 64, dtype=dtype, seed=60 + i)) for i in range(2)]
    alone = []
    for x in sets:
        O, S = torch.empty_like(x["q"]), torch.empty_like(x["S"])
        binding.darkattn_decay_forward(plan, x["q"], x["k"], x["v"], x["g"], O, plan.alloc_workspace(), S_in=x["S"], S_out=S)
        torch.cuda.synchronize()
        alone.append((O, S))
    streams = [torch.cuda.Stream() for _ in sets]
    outs = [(torch.zeros_like(x["q"]), torch.zeros_like(x["S"])) for x in sets]
    spaces = [plan.alloc_workspace() for _ in sets]
    torch.cuda.synchronize()
    for _ in range(5):
        for x, st, (O, S), ws in zip(sets, streams, outs, spaces):
            binding.darkattn_decay_forward(plan, x["q"], x["k"], x["v"], x["g"], O, ws, S_in=x["S"], S_out=S, stream=st)
    torch.cuda.synchronize()
    for got, want in zip(outs, alone):
        assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.gpu
def test_offsets_past_32_bits(binding):
    """A pool of states, a cache and a batch of rows with more than 2^31 numbers: what lies at their ends comes out as by itself."""
    H, d = 4, 128
    n = (1 << 31) // (H * d * d) + 40
    t = dev(make(2, H, 1, d, seed=70))
    plan = binding.darkattn_decay_plan(2, H, 1, d)
    args = [t[x][:, :, 0].contiguous() for x in ("q", "k", "v")]
    pool = torch.empty(n, H, d, d, device="cuda")
    slots = torch.tensor([n - 1, 3], dtype=torch.int32, device="cuda")
    pool[slots.long()] = t["S"]
    o, o2 = (torch.empty(2, H, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    small = t["S"].clone()
    binding.darkattn_decay_step(plan, *args, t["g"], pool, o, slots=slots)
    binding.darkattn_decay_step(plan, *args, t["g"], small, o2)
    assert torch.equal(o, o2) and torch.equal(pool[slots.long()], small)
    del pool
    codes, scales = torch.zeros(n, H, d, d, dtype=torch.int8, device="cuda"), torch.zeros(n, H, d, device="cuda")
    back, c2, s2 = torch.empty_like(small), torch.zeros(2, H, d, d, dtype=torch.int8, device="cuda"), torch.zeros(2, H, d, device="cuda")
    binding.darkattn_state_store(small, codes, scales, slots=slots)
    binding.darkattn_state_store(small, c2, s2)
    binding.darkattn_state_load(codes, scales, back, slots=slots)
    assert torch.equal(codes[slots.long()], c2) and torch.equal(scales[slots.long()], s2) and torch.equal(back, c2.float() * s2[..., None])
    del codes, scales
    for dtype in ("bf16", "f32"):
        dt, N, heads = (torch.bfloat16, 1 << 17, 140) if dtype == "bf16" else (torch.float32, 1 << 15, 1025)
        w = 128 if dtype == "bf16" else 64
        gen = torch.Generator(device="cuda").manual_seed(1)
        x = torch.randn(1, heads, N, w, generator=gen, device="cuda", dtype=dt)
        assert x.numel() > 1 << 31
        big = binding.darkattn_decay_plan(1, heads, N, w, dtype=binding.BF16 if dtype == "bf16" else binding.F32)
        g = torch.full((heads,), -0.1, device="cuda")
        O = torch.empty_like(x)
        binding.darkattn_decay_forward(big, x, x, x, g, O, big.alloc_workspace())
        last = x[:, -1:, -700:].cpu()               # what lies before these is decayed by e^-40 where the last 300 are looked at
        want, _ = oracle_forward(last, last, last, g[:1].cpu(), 1 / math.sqrt(w))
        mag, _ = oracle_forward(last.abs(), last.abs(), last.abs(), g[:1].cpu(), 1 / math.sqrt(w))
        check(O[:, -1:, -300:], want[:, :, 400:], mag[:, :, 400:] * (1 + math.exp(-30)), ops_of(w, w, 700), dt, True, "last rows")
        del x, O


@pytest.mark.gpu
def test_the_binding_refuses_what_does_not_fit(binding):
    t = dev(make(1, 2, 20, 8, dtype="f32"))
    plan = binding.darkattn_decay_plan(1, 2, 20, 8, dtype=binding.F32)
    ws, O = plan.alloc_workspace(), torch.empty(1, 2, 20, 8, device="cuda")
    good = dict(Q=t["q"], K=t["k"], V=t["v"], log_decay=t["g"], O=O, workspace=ws)
    for k, v in [("Q", t["q"][:, :, :19]), ("K", t["k"].double()), ("V", t["v"].cpu()), ("O", O.transpose(1, 2).contiguous().transpose(1, 2)),
                 ("workspace", ws[:128]), ("log_decay", t["g"][:1]), ("Q", t["q"].transpose(-1, -2).contiguous().transpose(-1, -2))]:
        with pytest.raises(ValueError):
            binding.darkattn_decay_forward(plan, **{**good, k: v})
    with pytest.raises(ValueError):
        binding.darkattn_decay_forward(plan, **good, lengths=torch.zeros(1, dtype=torch.int64, device="cuda"))
    S = torch.zeros(2, 3, 8, device="cuda")
    with pytest.raises(ValueError):
        binding.darkattn_state_store(S, torch.zeros(2, 3, 8, device="cuda"), torch.zeros(2, 3, device="cuda"))
    with pytest.raises(ValueError):
        binding.darkattn_state_load(torch.zeros(2, 3, 8, dtype=torch.int8, device="cuda"), torch.zeros(2, 4, device="cuda"), S)
