"""Attention with a decay per head where a sequence is cut into segments of several chunks, and these into pieces: the cut that long prompts and
training steps have. With and without the optional states, against the quadratic form in 64 bits.

Bounds. FP32 arithmetic: `check` of test_decay.py, element by element. bf16 rows: beside that, which grows with the number of terms where errors of
either sign grow like its root, two on the norm of the error, for every head by itself.

1. Against `rounded`, the same sums in 64 bits with the kernels' documented roundings and no other: the masked scores times their decays, and the
   state that a chunk's rows read, to bf16. What is left is the rounding of the rows out, whose norm is known (`rounded` is at hand before it), and
   bits on which the kernel's scores and states fall to the other side of a rounding border. States are off by 2^-17 of their norm (two bf16
   parts of a token's share leave 2^-16 of it at most, in either direction; fp32 sums less), so that 2 2^-17 / 2^-8 = 2^-8 of them fall to the
   other side, by a step of 2^-7 at most: 2^-4 2^-7 = 2^-11 of the state's part. Scores, off by 2^-22, add 2^-14. The rows out being rounded
   with an error of 0.0015 to 0.0023 of their norm (a step over the root of 12: 2^-7 / 3.46 at the beginning of a binade), the sum is within
   sqrt(1 + (2^-11 / 0.0015)^2) = 1.06 of theirs alone; 1.15 leaves as much again for the sample. A second part that is lost adds 0.0017 of the state's part.
   (A kernel in FP32 arithmetic rounds the rows out alone: the same bound against the quadratic form.)
2. Against the quadratic form: one rounding of the rows out and one of each term, of rms 2^-7 / sqrt(12) = 0.00226 at most each. The terms are independent and
   of either sign, so that the errors' squares add up as their own do: sqrt(2) 0.00226 = 0.0032, and 5 % for the sample.
"""
import math

import pytest
import torch

from tests.test_decay import SHAPES, binding, blank_padding, check, dev, make, ops_of, oracle_backward, oracle_forward, poison_padding  # noqa: F401

C, FEW = 128, 32                                # a chunk of the tensor-core kernel; up to so many rows its scores are kept in two parts
AGAINST_ROUNDED, AGAINST_EXACT = 1.15, 0.0032 * 1.05


# ------------------------------------------------------------------------------------------------ the quadratic form in 64 bits, head by head
def _powers(g, n):
    """g^n by 64-bit exp; 0^0 = 1"""
    return torch.where(n == 0, 1.0, torch.exp(g * n.clamp(min=1).double()))


def quadratic(X, Y, Z, g, reverse, mul, S, row_mul):
    """sum_j mul lambda^|i-j| (x_i . y_j) z_j + row_mul lambda^(distance of i to the boundary) x_i S, of one head; j up to i, or from i on."""
    n = X.shape[0]
    i = torch.arange(n, device=X.device)
    out = torch.empty(n, Z.shape[1], dtype=torch.float64, device=X.device)
    for a in range(0, n, 1024):
        b = min(a + 1024, n)
        dist = (i[a:b, None] - i[None]) * (-1 if reverse else 1)
        out[a:b] = torch.where(dist >= 0, mul * _powers(g, dist.clamp(min=0)) * (X[a:b] @ Y.T), 0.0) @ Z
    if S is not None:
        out += row_mul * _powers(g, n - 1 - i if reverse else i + 1)[:, None] * (X @ S)
    return out


def states(Y, Z, g, reverse, mul, S):
    """The state behind the last row in the pass's direction."""
    n = Y.shape[0]
    i = torch.arange(n, device=Y.device)
    out = (mul * _powers(g, i + 1 if reverse else n - 1 - i)[:, None] * Y).T @ Z
    return out if S is None else out + _powers(g, torch.tensor(n, device=Y.device)) * S


def to_bf16(x):
    return x.float().bfloat16().double()


def rounded(X, Y, Z, g, reverse, mul, S, row_mul, tok_mul, cps, mistake=""):
    """As `quadratic`, in chunks, with the roundings of the bf16 kernel. X [n, a]; Y, Z [G, n, .] are summed over G. `mistake`: one to plant.
    Where neither width is above 64 the kernel keeps the state as the sum of two, of every chunk's first 64 tokens (and the state that a segment
    of `cps` chunks is entered by) and of its others, and rounds either."""
    n = X.shape[0]
    S = torch.zeros(X.shape[1], Z.shape[2], dtype=torch.float64, device=X.device) if S is None else S.clone()
    S2 = torch.zeros_like(S)
    half = 64 if max(X.shape[1], Z.shape[2]) <= 64 else C
    out = torch.empty(n, Z.shape[2], dtype=torch.float64, device=X.device)
    T = -(-n // C)
    for k in range(T):
        t0 = (T - 1 - k if reverse else k) * C
        x, y, z = X[t0:t0 + C], Y[:, t0:t0 + C], Z[:, t0:t0 + C]
        L = x.shape[0]
        if k % cps == 0:
            S, S2 = S + S2, torch.zeros_like(S)
        r = torch.arange(L, device=X.device)
        dist = (r[:, None] - r[None]) * (-1 if reverse else 1)
        P = torch.where(dist >= 0, mul * _powers(g, dist.clamp(min=0)) * (x @ y.transpose(1, 2)), 0.0)
        far = _powers(g, L - 1 - r if reverse else r + 1)
        out[t0:t0 + L] = ((P if L <= FEW else to_bf16(P)) @ z).sum(0) + row_mul * far[:, None] * (x @ (to_bf16(S) + to_bf16(S2)))
        share = tok_mul * _powers(g, r + 1 if reverse else L - 1 - r)[:, None] * y
        if mistake == "second part":
            share = to_bf16(share)
        keep = _powers(g, torch.tensor(L - (mistake == "power"), device=X.device))
        S, S2 = (keep * s + (share[:, i:j].transpose(1, 2) @ z[:, i:j]).sum(0) for s, i, j in ((S, 0, half), (S2, half, C)))
        if mistake == "state" and k == T // 2:
            S, S2 = torch.zeros_like(S), torch.zeros_like(S)
    return out


def both_forms(t, gradients, scale, cps):
    """{name: (quadratic form, the same with roundings; that without where cps is 0)} of all rows, zeros behind each end, and the state out."""
    t = {k: None if v is None else (v if k == "lengths" else v.double()) for k, v in t.items()}
    B, H, N, d = t["q"].shape
    Hk, dv = t["k"].shape[1], t["v"].shape[3]
    G = H // Hk
    at = t["q"].device
    zero = lambda *s: torch.zeros(*s, dtype=torch.float64, device=at)  # noqa: E731
    names = {"dq": (H, d), "dk": (Hk, d), "dv": (Hk, dv)} if gradients else {"o": (H, dv)}
    out = {x: (zero(B, h, N, w), zero(B, h, N, w)) for x, (h, w) in names.items()}
    S_out = zero(B, Hk, d, dv)
    for b in range(B):
        n = N if t["lengths"] is None else min(max(int(t["lengths"][b]), 0), N)
        for h in range(Hk):
            g = t["g"][h]
            S = None if t["S"] is None else t["S"][b, h]
            dS = None if t["dS"] is None else t["dS"][b, h]
            k, v = t["k"][b, h, :n], t["v"][b, h, :n]
            Q, D = t["q"][b, h * G:(h + 1) * G, :n], t["do"][b, h * G:(h + 1) * G, :n]
            ST, dST = (None if x is None else x.T for x in (S, dS))

            def put(name, hx, quad, *chunks):
                out[name][0][b, hx, :n] = quad
                out[name][1][b, hx, :n] = rounded(*chunks, cps) if cps else quad

            if gradients:
                for i in range(G):
                    put("dq", h * G + i, quadratic(D[i], v, k, g, False, scale, ST, scale), D[i], v[None], k[None], g, False, scale, ST, scale, 1.0)
                put("dk", h, sum(quadratic(v, D[i], Q[i], g, True, scale, dST if i == 0 else None, 1.0) for i in range(G)), v, D, Q, g, True, scale, dST, 1.0, scale)
                put("dv", h, sum(quadratic(k, Q[i], D[i], g, True, scale, dS if i == 0 else None, 1.0) for i in range(G)), k, Q, D, g, True, scale, dS, 1.0, scale)
                S_out[b, h] = sum(states(Q[i], D[i], g, True, scale, dS if i == 0 else None) for i in range(G))
            else:
                for i in range(G):
                    put("o", h * G + i, quadratic(Q[i], k, v, g, False, scale, S, scale), Q[i], k[None], v[None], g, False, scale, S, scale, 1.0)
                S_out[b, h] = states(k, v, g, False, 1.0, S)
    return out, S_out


def worst_norms(got, forms, lengths):
    """The largest shares of either bound over the heads, of all rows and of those behind the first chunk."""
    exact, before = forms
    worst = [0.0, 0.0]
    for b in range(got.shape[0]):
        n = got.shape[2] if lengths is None else min(max(int(lengths[b]), 0), got.shape[2])
        for first in (0, C):
            if n - first < 64:                  # (a sample)
                continue
            e, r, x = (y[b, :, first:n].double() for y in (exact, before, got))
            norm = lambda y: y.norm(dim=(1, 2))  # noqa: E731
            worst[0] = max(worst[0], (norm(x - r) / norm(to_bf16(r) - r)).max().item() / AGAINST_ROUNDED)
            worst[1] = max(worst[1], (norm(x - e) / norm(e)).max().item() / AGAINST_EXACT)
    return worst


# ------------------------------------------------------------------------------------------------ the bounds themselves (no GPU)
def _like_the_kernel(t, scale, mistake=""):
    B, H, N, _ = t["q"].shape
    O = torch.zeros(B, H, N, t["v"].shape[3], dtype=torch.float64)
    for h in range(H):
        S = None if t["S"] is None else t["S"][0, h].double()
        O[0, h] = rounded(t["q"][0, h].double(), t["k"][0, h:h + 1].double(), t["v"][0, h:h + 1].double(), t["g"][h].double(), False, scale, S, scale, 1.0, 5, mistake)
    return O.bfloat16()


def test_the_forms_agree_with_the_recurrence():
    t = make(2, 4, 300, 6, dv=5, Hk=2, dtype="f32", decays=(-0.01, -float("inf")))
    t["lengths"] = torch.tensor([300, 171])
    clean = blank_padding(t)
    (o, S), scale = oracle_forward(clean["q"], clean["k"], clean["v"], t["g"], 0.4, t["lengths"], t["S"]), 0.4
    forms, state = both_forms(t, False, scale, 0)
    assert torch.allclose(forms["o"][0], o, rtol=1e-12, atol=1e-12) and torch.allclose(state, S, rtol=1e-12, atol=1e-12)
    t["g"] = torch.tensor([-0.01, -0.3])
    want = oracle_backward(*(clean[x] for x in ("q", "k", "v", "do")), t["g"], scale, t["lengths"], t["S"], t["dS"])
    forms, state = both_forms(t, True, scale, 0)
    for x, w in zip(("dq", "dk", "dv"), want):
        assert torch.allclose(forms[x][0], w, rtol=1e-12, atol=1e-12)
    assert torch.allclose(state, want[3], rtol=1e-12, atol=1e-12)


def test_the_norms_see_what_the_elements_do_not():
    """Mistakes that the bound by elements lets pass; without one, either bound holds with room."""
    t = make(1, 2, 1100, 64, 64, 2, "bf16", seed=5, decays=(-math.log(2) / 60, -math.log(2) / 400))
    t["S"], t["dS"] = None, None
    forms, _ = both_forms(t, False, 0.125, 5)
    mag, _ = oracle_forward(t["q"].abs(), t["k"].abs(), t["v"].abs(), t["g"], 0.125)
    for mistake in ("", "second part", "power", "state"):
        got = _like_the_kernel(t, 0.125, mistake)
        a, b = worst_norms(got, forms["o"], None)
        if mistake != "state":
            check(got, forms["o"][0], mag, ops_of(64, 64, 1100), torch.bfloat16, True, mistake)
        if mistake:
            assert a > 1.1, (mistake, a, b)
            assert (b > 1.0) == (mistake in ("power", "state")), (mistake, a, b)
        else:
            assert a < 0.9 and b < 0.8, (a, b)


# ------------------------------------------------------------------------------------------------ on the GPU
#  B, H, N, d, dv, H_kv, type, path;  whether the forward, the backward pass has segments of several chunks, and pieces
CUT = [
    ((2, 12, 898, 96, 64, 3, "bf16", 0), (True, True), (True, True)),
    ((1, 8, 8000, 96, 64, 2, "bf16", 0), (True, True), (False, False)),
    ((1, 16, 5888, 128, 128, 16, "bf16", 0), (True, False), (True, True)),
    ((2, 16, 5888, 128, 128, 16, "bf16", 0), (True, True), None),
    ((1, 16, 8192, 64, 64, 4, "bf16", 0), (True, True), (True, True)),
    ((2, 24, 4000, 64, 64, 8, "bf16", 0), (True, True), (True, True)),
    ((2, 6, 4000, 64, 128, 6, "bf16", 0), (True, False), (True, True)),
    ((8, 16, 1100, 128, 128, 4, "bf16", 0), None, None),
    ((1, 16, 2757, 128, 128, 16, "f32", 0), (True, False), (True, False)),
    ((2, 24, 2000, 64, 64, 24, "f32", 0), (False, False), (True, False)),
    ((2, 8, 2000, 200, 136, 8, "f32", 0), (True, False), (True, False)),
    ((1, 16, 3000, 256, 256, 4, "bf16", 0), (True, False), (False, False)),
    ((2, 12, 1500, 96, 64, 3, "bf16", 1), None, None),
    # one segment, many chunks by one block, all stages in use
    ((2, 50, 2100, 64, 64, 50, "bf16", 0), None, None),
    ((2, 75, 1500, 128, 64, 75, "bf16", 0), None, None),
    ((2, 75, 1500, 64, 128, 75, "bf16", 0), None, None),
    ((2, 75, 1500, 128, 128, 75, "bf16", 0), None, None),
]


@pytest.mark.parametrize("shape,forward,backward", CUT, ids=str)
def test_the_cuts_are_what_these_tests_are_about(binding, shape, forward, backward):  # noqa: F811
    """(Refitting the estimate that cuts sequences may change these: then other shapes have to take their places.)"""
    plan, path = _plan(binding, *shape), shape[-1]
    for which, want in ((False, forward), (True, backward)):
        if want is not None:
            nseg, cps, sub = plan.split(which)
            assert nseg > 1 and (cps > 1, sub > 1) == want, (which, nseg, cps, sub)
            assert cps % sub == 0
        elif path == 0:
            assert plan.split(which)[0] == 1 or forward is not None
    plan.destroy()


def _plan(binding, B, H, N, d, dv, Hk, dtype, path):  # noqa: F811
    return binding.darkattn_decay_plan(B, H, N, d, dv=dv, H_kv=Hk, dtype=binding.BF16 if dtype == "bf16" else binding.F32, path=path)


def _inputs(shape, seed, states_in, lengths):
    B, H, N, d, dv, Hk, dtype, _ = shape
    t = make(B, H, N, d, dv, Hk, dtype, seed=seed)
    if "S" not in states_in:
        t["S"] = None
    if "dS" not in states_in:
        t["dS"] = None
    if lengths:
        t["lengths"] = torch.tensor([lengths[b % len(lengths)] for b in range(B)], dtype=torch.int32)
        t = poison_padding(t)
    return t


def _cases():
    out = []
    for shape, forward, _ in CUT:
        N = shape[2]
        # states: all four; none; those in without the one out, one of them in, and the other way round
        out.append((shape, None, (), False))
        out.append((shape, [N - 1, N // 3], ("S",), True))
        if forward is None:
            continue
        out.append((shape, None, ("S", "dS"), True))
        out.append((shape, None, ("S", "dS"), False))
        out.append((shape, [N * 7 // 10 + 1, N - 200], ("dS",), False))
        out.append((shape, [N // 2, 130], (), True))
    return out


@pytest.mark.gpu
@pytest.mark.parametrize("shape,lengths,states_in,state_out", _cases(), ids=str)
def test_forward_in_segments(binding, shape, lengths, states_in, state_out):  # noqa: F811
    B, H, N, d, dv, Hk, dtype, _ = shape
    t = _inputs(shape, N + d, states_in, lengths)
    plan, D = _plan(binding, *shape), dev(t)
    ws = torch.full((plan.workspace_bytes + 1024,), 0xff, dtype=torch.uint8, device="cuda")
    O = torch.full((B, H, N, dv), 7.0, dtype=t["q"].dtype, device="cuda")
    S_out = torch.full((B, Hk, d, dv), float("nan"), device="cuda") if state_out else None
    binding.darkattn_decay_forward(plan, D["q"], D["k"], D["v"], D["g"], O, ws[:plan.workspace_bytes], lengths=D["lengths"], S_in=D["S"], S_out=S_out)
    assert binding.darkattn_decay_last_device_status(plan, ws) == binding.OK and bool((ws[plan.workspace_bytes:] == 0xff).all())
    _compare(plan, binding, D, t, {"o": O}, S_out, False)


@pytest.mark.gpu
@pytest.mark.parametrize("shape,lengths,states_in,state_out", _cases(), ids=str)
def test_backward_in_segments(binding, shape, lengths, states_in, state_out):  # noqa: F811
    B, H, N, d, dv, Hk, dtype, _ = shape
    t = _inputs(shape, N + d + 1, states_in, lengths)
    plan, D = _plan(binding, *shape), dev(t)
    ws = torch.full((plan.workspace_bytes + 1024,), 0xff, dtype=torch.uint8, device="cuda")
    got = {"dq": torch.full_like(D["q"], float("nan")), "dk": torch.full_like(D["k"], float("nan")), "dv": torch.full_like(D["v"], float("nan"))}
    dS_in = torch.full((B, Hk, d, dv), float("nan"), device="cuda") if state_out else None
    binding.darkattn_decay_backward(plan, D["q"], D["k"], D["v"], D["g"], D["do"], got["dq"], got["dk"], got["dv"], ws[:plan.workspace_bytes], lengths=D["lengths"],
                                    S_in=D["S"], dS_out=D["dS"], dS_in=dS_in)
    assert binding.darkattn_decay_last_device_status(plan, ws) == binding.OK and bool((ws[plan.workspace_bytes:] == 0xff).all())
    _compare(plan, binding, D, t, got, dS_in, True)


def _within(got, want, mag, ops, dtype, tensor, what):
    """`check` of test_decay.py, on the GPU"""
    got = got.double()
    assert torch.isfinite(got).all(), f"{what}: not finite"
    bound = ops * 2.0 ** -23 * mag + 1e-37
    if dtype == torch.bfloat16:
        bound += 2.0 ** -8 * want.abs()
        if tensor:
            bound += (2.0 ** -8 + 2.0 ** -16) * mag
    worst = ((got - want).abs() / bound).max().item()
    assert worst <= 1.0, f"{what}: {worst:.3f} of the bound"


def _compare(plan, binding, D, t, got, state, gradients):  # noqa: F811
    B, H, N, d = t["q"].shape
    Hk, dv = t["k"].shape[1], t["v"].shape[3]
    scale, tensor = 1 / math.sqrt(d), plan.path == binding.PATH_TENSOR
    clean = {k: None if v is None else v.cuda() for k, v in {**t, **blank_padding(t)}.items()}
    forms, want_state = both_forms(clean, gradients, scale, plan.split(gradients)[1] if tensor else 0)
    mags, mag_state = both_forms({k: v if v is None or k in ("g", "lengths") else v.abs() for k, v in clean.items()}, gradients, scale, 0)
    n = ops_of(d, dv, N) * (H // Hk if gradients else 1)
    live = torch.arange(N, device="cuda")[None] < (torch.full((B,), N, device="cuda") if D["lengths"] is None else D["lengths"])[:, None]
    live = live[:, None, :, None]
    for name, x in got.items():
        if not gradients:
            assert bool((torch.where(live, 7.0, x.float()) == 7).all()), "rows behind the end were touched"
            x = torch.where(live, x, 0.0)
        _within(x, forms[name][0], mags[name][0], n, t["q"].dtype, tensor, name)
        if t["q"].dtype == torch.bfloat16:
            a, b = worst_norms(x, forms[name], t["lengths"])
            assert a <= 1 and b <= 1, f"{name}: {a:.3f} of the bound on the norm against the rounded form, {b:.3f} against the exact one"
    if state is not None:
        _within(state, want_state, mag_state, n, torch.float32, tensor, "state")


# ------------------------------------------------------------------------------------------------ short calls without states, growing states, the most heads
def _both_calls(binding, t, path, state_out):  # noqa: F811
    B, H, N, d = t["q"].shape
    Hk, dv = t["k"].shape[1], t["v"].shape[3]
    plan = binding.darkattn_decay_plan(B, H, N, d, dv=dv, H_kv=Hk, dtype=binding.BF16 if t["q"].dtype == torch.bfloat16 else binding.F32, path=path)
    D, ws = dev(t), plan.alloc_workspace()
    O = torch.full((B, H, N, dv), 7.0, dtype=t["q"].dtype, device="cuda")
    new = lambda x: torch.full_like(D[x], float("nan"))  # noqa: E731
    grads = {"dq": new("q"), "dk": new("k"), "dv": new("v")}
    S_out, dS_in = (torch.full((B, Hk, d, dv), float("nan"), device="cuda") if state_out else None for _ in range(2))
    binding.darkattn_decay_forward(plan, D["q"], D["k"], D["v"], D["g"], O, ws, lengths=D["lengths"], S_in=D["S"], S_out=S_out)
    assert binding.darkattn_decay_last_device_status(plan, ws) == binding.OK
    _compare(plan, binding, D, t, {"o": O}, S_out, False)
    binding.darkattn_decay_backward(plan, D["q"], D["k"], D["v"], D["g"], D["do"], *grads.values(), ws, lengths=D["lengths"], S_in=D["S"], dS_out=D["dS"], dS_in=dS_in)
    assert binding.darkattn_decay_last_device_status(plan, ws) == binding.OK
    _compare(plan, binding, D, t, grads, dS_in, True)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_calls_without_states_out(binding, shape, dtype):  # noqa: F811
    B, H, N, d, dv, Hk = shape
    for path in (binding.PATH_SIMT, binding.PATH_AUTO):
        for states_in in ((), ("S",), ("dS",), ("S", "dS")):
            t = _inputs((B, H, N, d, dv, Hk, dtype, path), 80 + N, states_in, [N // 2, N] if len(states_in) == 1 else None)
            _both_calls(binding, t, path, False)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d,dv", [(64, 64), (128, 72)])
def test_states_that_grow(binding, dtype, d, dv):  # noqa: F811
    """A decay above 1 is not refused."""
    for path in (binding.PATH_SIMT, binding.PATH_AUTO):
        for state_out in (False, True):
            _both_calls(binding, make(2, 4, 600, d, dv, 2, dtype, seed=90, decays=(0.004, 0.02)), path, state_out)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_as_many_heads_as_there_may_be(binding, dtype):  # noqa: F811
    """65535 of them: prompts, gradients, a step, a cache, whose last head is what it is by itself."""
    H, N, d = 65535, 3, 8
    gen = torch.Generator(device="cuda").manual_seed(3)
    rnd = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    kind = binding.BF16 if dtype == "bf16" else binding.F32
    q, k, v, do = (rnd(1, H, N, d).to(dt) for _ in range(4))
    S, g = rnd(1, H, d, d), -rnd(H).abs()

    def calls(*at):
        x = [t[:, at].contiguous() if at else t for t in (q, k, v, do, S)]
        decay = g[list(at)].contiguous() if at else g
        h = x[0].shape[1]
        plan, one = (binding.darkattn_decay_plan(1, h, n, d, dtype=kind) for n in (N, 1))
        ws = plan.alloc_workspace()
        O, S_out, dS_in = torch.empty_like(x[2]), torch.empty_like(x[4]), torch.empty_like(x[4])
        binding.darkattn_decay_forward(plan, *x[:3], decay, O, ws, S_in=x[4], S_out=S_out)
        grads = [torch.empty_like(y) for y in x[:3]]
        binding.darkattn_decay_backward(plan, *x[:3], decay, x[3], *grads, ws, S_in=x[4], dS_in=dS_in)
        pool, o = S_out.clone(), torch.empty_like(x[0][:, :, 0]).contiguous()
        binding.darkattn_decay_step(one, *(y[:, :, 0].contiguous() for y in x[:3]), decay, pool, o)
        kept = pool.reshape(h, 1, d, d)
        codes, scales, back = torch.empty(h, 1, d, d, dtype=torch.int8, device="cuda"), torch.empty(h, 1, d, device="cuda"), torch.empty_like(kept)
        binding.darkattn_state_store(kept, codes, scales)
        binding.darkattn_state_load(codes, scales, back)
        return [O, S_out, dS_in, *grads, pool, o[:, :, None], back.reshape(1, h, d, d)]

    for whole, part in zip(calls(), calls(0, 40000, 65534)):
        assert torch.equal(whole[:, [0, 40000, 65534]], part)
