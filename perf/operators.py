"""Performance cases of the attention with a decay per head and of the 8-bit state cache.

A case is one of four kinds of call:
  "prompt"    darkattn_decay_forward: the chunked form over a batch of prompts
  "backward"  darkattn_decay_backward: the gradients of a training step
  "step"      darkattn_decay_step: one token per sequence, the running states in a pool of slots
  "cache"     darkattn_state_store, then darkattn_state_load: running states kept in 8 bits, read back
With ``own`` unset ``run`` computes the same from elementary torch operations in 32 bits.
"""
import math

import torch

own = False

_FIELDS = ("kind", "dtype", "B", "H", "H_kv", "N", "d", "dv", "ragged", "states", "format")
_CHUNK = 128


def _case(kind, B, H, N, d, dtype="bf16", H_kv=0, dv=0, ragged=False, states=False, format="", name=None):
    c = dict(zip(_FIELDS, (kind, dtype, B, H, H_kv or H, N, d, dv or d, ragged, states, format)))
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # a short prompt of one request; prompt lengths are whatever the user typed
        _case("prompt", 1, 12, 333, 64, name="prompt_short_odd"),
        # a padded batch of prompts that continue earlier turns (state in, state out), four query heads to a key/value head
        _case("prompt", 8, 16, 2001, 128, H_kv=4, ragged=True, states=True, name="prompt_ragged_grouped"),
        # prefill of long prompts
        _case("prompt", 4, 16, 8192, 128, name="prefill_8k"),
        # prefill of one very long document: few heads, the state kept for the answer
        _case("prompt", 1, 8, 65536, 64, states=True, name="prefill_64k"),
        # single precision, an ordinary batch, a width that is no power of two
        _case("prompt", 2, 12, 1000, 80, dtype="f32", name="f32_prompt"),
        # training step of a small model
        _case("backward", 8, 12, 2048, 64, name="train_2k"),
        # training step of long sequences
        _case("backward", 4, 16, 8192, 128, name="train_8k"),
        # single-precision training over a piece of a longer sequence: gradients flow through the states at both ends
        _case("backward", 2, 8, 1000, 64, dtype="f32", states=True, name="f32_train"),
        # one decode step of a few sequences: one short launch, the caller waits for it at every token
        _case("step", 4, 16, 1, 128, name="decode_small"),
        # one decode step of many sequences: their states (134 MB) are read and written at every token
        _case("step", 128, 16, 1, 128, name="decode_large"),
        # one finished prompt's states go to the cache and back
        _case("cache", 1, 16, 1, 128, dtype="f32", format="i8", name="cache_one_prompt"),
        # a batch of them
        _case("cache", 96, 16, 1, 128, dtype="f32", format="e4m3", name="cache_batch"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("prompt", "prompt", "backward", "backward", "step", "cache"))
    H = rng.choice((8, 12, 16))
    d = rng.choice((64, 128, 64, 128, 80, 96))
    dv = rng.choice((d, d, d, 64, 128))
    H_kv = rng.choice((H, H, H, H // 4, H // 2))
    if kind == "step":
        B = max(1, min(_log_int(rng, 1, 128), 128 * 16 * 128 * 128 // (H_kv * d * dv)))
        return _case(kind, B, H, 1, d, dtype=rng.choice(("bf16", "bf16", "bf16", "f32")), H_kv=H_kv, dv=dv)
    if kind == "cache":
        rows = rng.choice((64, 128, 80, 256))
        B = max(1, min(_log_int(rng, 1, 96), 96 * 16 * 128 * 128 // (H * rows * dv)))
        return _case(kind, B, H, 1, rows, dtype="f32", dv=dv, format=rng.choice(("i8", "e4m3")))
    if rng.random() < 0.25:     # single precision: smaller problems
        N = _log_int(rng, 1, 4096)
        B = max(1, min(_log_int(rng, 1, 8), 2 * 12 * 2048 // (H * N)))
        return _case(kind, B, H, N, d, dtype="f32", H_kv=H_kv, dv=dv, ragged=rng.random() < 0.3, states=rng.random() < 0.5)
    N = _log_int(rng, 1, 65536 if kind == "prompt" else 8192)
    if rng.random() < 0.4 and N > 128:          # packed or padded to the chunk length
        N -= N % 128
    most = 4 * 16 * 8192
    B = max(1, min(_log_int(rng, 1, 16), most // (H * N)))
    while B * H * N > most:
        H, H_kv = H // 2, max(1, H_kv // 2)
    return _case(kind, B, H, N, d, H_kv=H_kv if H % H_kv == 0 else H, dv=dv, ragged=rng.random() < 0.3, states=rng.random() < 0.4)


def _dtype(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def prepare(case, seed):
    kind, B, H, Hkv, N, d, dv = (case[k] for k in ("kind", "B", "H", "H_kv", "N", "d", "dv"))
    dt = _dtype(case)
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, dtype=torch.float32):
        return torch.randn(*shape, generator=gen, device="cuda").to(dtype)

    def uniform(*shape):
        return torch.rand(*shape, generator=gen, device="cuda")

    s = {"kind": kind, "scale": 1.0 / math.sqrt(d), "format": case["format"]}
    if kind == "cache":
        slots = B + 3
        s.update(S=normal(B, H, d, dv) * torch.exp(normal(B, H, d, 1)), back=torch.empty(B, H, d, dv, device="cuda"),
                 slots=torch.randperm(slots, generator=gen, device="cuda")[:B].to(torch.int32),
                 codes=torch.zeros(slots, H, d, dv, dtype=torch.int8 if case["format"] == "i8" else torch.float8_e4m3fn, device="cuda"),
                 scales=torch.zeros(slots, H, d, device="cuda"))
        return s
    # half-lives from a few tokens to thousands, one per key/value head
    s["log_decay"] = -math.log(2) / torch.exp(math.log(4) + uniform(Hkv) * math.log(1024))
    if kind == "step":
        slots = B + 3
        s.update(q=normal(B, H, d, dtype=dt), k=normal(B, Hkv, d, dtype=dt), v=normal(B, Hkv, dv, dtype=dt), S=8 * normal(slots, Hkv, d, dv),
                 slots=torch.randperm(slots, generator=gen, device="cuda")[:B].to(torch.int32), o=torch.zeros(B, H, dv, dtype=dt, device="cuda"))
    else:
        s.update(Q=normal(B, H, N, d, dtype=dt), K=normal(B, Hkv, N, d, dtype=dt), V=normal(B, Hkv, N, dv, dtype=dt),
                 lengths=(1 + uniform(B) * N).to(torch.int32).clamp(1, N) if case["ragged"] else None,
                 S_in=8 * normal(B, Hkv, d, dv) if case["states"] else None)
        if kind == "prompt":
            s.update(O=torch.zeros(B, H, N, dv, dtype=dt, device="cuda"), S_out=torch.empty(B, Hkv, d, dv, device="cuda") if case["states"] else None)
        else:
            s.update(dO=normal(B, H, N, dv, dtype=dt), dS_out=normal(B, Hkv, d, dv) if case["states"] else None,
                     dQ=torch.empty(B, H, N, d, dtype=dt, device="cuda"), dK=torch.empty(B, Hkv, N, d, dtype=dt, device="cuda"),
                     dV=torch.empty(B, Hkv, N, dv, dtype=dt, device="cuda"), dS_in=torch.empty(B, Hkv, d, dv, device="cuda") if case["states"] else None)
    if own:
        from paper_2603_04127_b200 import binding
        s["plan"] = binding.darkattn_decay_plan(B, H, N, d, dv=dv, dtype=binding.F32 if case["dtype"] == "f32" else binding.BF16, H_kv=Hkv)
        s["workspace"] = s["plan"].alloc_workspace()
    return s


# ------------------------------------------------------------------------------------------------ the framework's calls
def _run_own(s):
    from paper_2603_04127_b200 import binding
    if s["kind"] == "cache":
        fmt = binding.STATE_I8 if s["format"] == "i8" else binding.STATE_E4M3
        binding.darkattn_state_store(s["S"], s["codes"], s["scales"], slots=s["slots"], format=fmt)
        binding.darkattn_state_load(s["codes"], s["scales"], s["back"], slots=s["slots"], format=fmt)
        return s["back"], s["scales"]
    if s["kind"] == "step":
        binding.darkattn_decay_step(s["plan"], s["q"], s["k"], s["v"], s["log_decay"], s["S"], s["o"], slots=s["slots"])
        return s["o"], s["S"]
    if s["kind"] == "prompt":
        binding.darkattn_decay_forward(s["plan"], s["Q"], s["K"], s["V"], s["log_decay"], s["O"], s["workspace"], lengths=s["lengths"],
                                       S_in=s["S_in"], S_out=s["S_out"])
        return s["O"], s["S_out"]
    binding.darkattn_decay_backward(s["plan"], s["Q"], s["K"], s["V"], s["log_decay"], s["dO"], s["dQ"], s["dK"], s["dV"], s["workspace"],
                                    lengths=s["lengths"], S_in=s["S_in"], dS_out=s["dS_out"], dS_in=s["dS_in"])
    return s["dQ"], s["dK"], s["dV"], s["dS_in"]


# ------------------------------------------------------------------------------------------------ the plain form
def _scan(x, y, z, g):
    """out_i = sum over j <= i of exp(g (i - j)) (x_i . y_j) z_j, in chunks; x, y [B, H, N, a], z [B, H, N, c], g [H]."""
    B, H, N, a = x.shape
    C, T = _CHUNK, -(-N // _CHUNK)
    x, y, z = (torch.nn.functional.pad(t, (0, 0, 0, T * C - N)).reshape(B, H, T, C, -1) for t in (x, y, z))
    pos = torch.arange(max(C, T), device=x.device)
    i = pos[:C]
    inside = torch.where(i[:, None] >= i, torch.exp(g.double()[:, None, None] * (i[:, None] - i).clamp(min=0)), 0.0).float()
    out = ((x @ y.transpose(-1, -2)) * inside[:, None]) @ z
    local = (y * torch.exp(g.double()[:, None] * (C - 1 - i)).float()[:, None, :, None]).transpose(-1, -2) @ z
    t = pos[:T]
    between = torch.where(t[:, None] > t, torch.exp(C * g.double()[:, None, None] * (t[:, None] - 1 - t).clamp(min=0)), 0.0).float()
    before = (between @ local.reshape(B, H, T, -1)).reshape(local.shape)
    out = out + torch.exp(g.double()[:, None] * (i + 1)).float()[:, None, :, None] * (x @ before)
    return out.reshape(B, H, T * C, -1)[:, :, :N]


def _flip(t):
    return t.flip(2)


def _masked(s, *tensors):
    """The tensors in 32 bits with zeros behind each sequence's end; positions, ends [B, 1, N, 1] and validity."""
    N = tensors[0].shape[2]
    at = torch.arange(N, device="cuda")[None, None, :, None]
    n = torch.full((tensors[0].shape[0],), N, device="cuda") if s["lengths"] is None else s["lengths"].long()
    n = n[:, None, None, None]
    return [torch.where(at < n, t.float(), 0.0) for t in tensors], at, n


def _shared(t, G):
    return t.repeat_interleave(G, 1)


def _grouped(t, G):
    return t.reshape(t.shape[0], -1, G, *t.shape[2:]).sum(2)


def _run_plain(s):
    kind, scale = s["kind"], s["scale"]
    if kind == "cache":
        # the scale is a number in 32 bits; the quotient is taken in 64, so that what lies next to a border goes to the nearer side
        sc = (s["S"].abs().amax(-1).double() / (127.0 if s["format"] == "i8" else 448.0)).float()
        units = torch.where(sc[..., None] > 0, s["S"].double() / sc[..., None].double(), 0.0)
        if s["format"] == "i8":
            codes = torch.round(units).clamp(-127, 127).to(torch.int8)
        else:                   # steps of an eighth of the leading power of two, of 2^-9 below 2^-6
            lead = torch.frexp(units)[1].clamp(min=-5) - 4
            codes = torch.ldexp(torch.round(torch.ldexp(units, -lead)), lead).clamp(-448, 448).float().to(torch.float8_e4m3fn)
        at = s["slots"].long()
        s["codes"].view(torch.int8).index_copy_(0, at, codes.view(torch.int8))
        s["scales"].index_copy_(0, at, sc)
        s["back"].copy_(s["codes"].view(torch.int8)[at].view(codes.dtype).float() * s["scales"][at][..., None])
        return s["back"], s["scales"]
    g = s["log_decay"]
    if kind == "step":
        at, G = s["slots"].long(), s["q"].shape[1] // s["k"].shape[1]
        S = torch.exp(g.double()).float()[:, None, None] * s["S"][at] + s["k"].float()[..., None] * s["v"].float()[..., None, :]
        s["S"].index_copy_(0, at, S)
        q = s["q"].float().reshape(S.shape[0], S.shape[1], G, -1)
        s["o"].copy_((scale * (q @ S)).reshape(s["o"].shape))
        return s["o"], s["S"]
    G = s["Q"].shape[1] // s["K"].shape[1]
    gh = g.repeat_interleave(G)
    if kind == "prompt":
        (q, k, v), at, n = _masked(s, s["Q"], s["K"], s["V"])
        out = _scan(q, _shared(k, G), _shared(v, G), gh)
        if s["S_in"] is not None:
            out = out + torch.exp(gh.double()[:, None, None] * (at + 1)).float() * (q @ _shared(s["S_in"], G))
            w = torch.where(at < n, torch.exp(g.double()[:, None, None] * (n - 1 - at).clamp(min=0)), 0.0).float()
            s["S_out"].copy_((w * k).transpose(-1, -2) @ v + torch.exp(g.double()[:, None, None] * n).float() * s["S_in"])
        s["O"].copy_(torch.where(at < n, (scale * out).to(s["O"].dtype), s["O"]))
        return s["O"], s["S_out"]
    (q, k, v, do), at, n = _masked(s, s["Q"], s["K"], s["V"], s["dO"])
    kq, vq = _shared(k, G), _shared(v, G)
    dq = _scan(do, vq, kq, gh)
    dk = _flip(_scan(_flip(vq), _flip(do), _flip(q), gh))
    dv = _flip(_scan(_flip(kq), _flip(q), _flip(do), gh))
    dk, dv = scale * _grouped(dk, G), scale * _grouped(dv, G)
    if s["S_in"] is not None:
        first = torch.exp(gh.double()[:, None, None] * (at + 1)).float()
        dq = dq + first * (do @ _shared(s["S_in"], G).transpose(-1, -2))
        last = torch.where(at < n, torch.exp(g.double()[:, None, None] * (n - 1 - at).clamp(min=0)), 0.0).float()
        dk = dk + last * (v @ s["dS_out"].transpose(-1, -2))
        dv = dv + last * (k @ s["dS_out"])
        s["dS_in"].copy_(scale * _grouped((first * q).transpose(-1, -2) @ do, G) + torch.exp(g.double()[:, None, None] * n).float() * s["dS_out"])
    s["dQ"].copy_(scale * dq)
    s["dK"].copy_(dk)
    s["dV"].copy_(dv)
    return s["dQ"], s["dK"], s["dV"], s["dS_in"]


def run(s):
    return _run_own(s) if own else _run_plain(s)


# ------------------------------------------------------------------------------------------------ counts and 64 bits
def work(case):
    """Bytes: every input read once, every output written once. Operations: the recurrence's own, 2 d dv to add a token to the
    state and 2 d dv to read a query out of it; the backward pass has both recurrences and three read-outs."""
    kind, B, H, Hkv, N, d, dv = (case[k] for k in ("kind", "B", "H", "H_kv", "N", "d", "dv"))
    e = 4 if case["dtype"] == "f32" else 2
    if kind == "cache":
        return {"bytes": 2 * B * H * d * (5 * dv + 4), "flops": 3 * B * H * d * dv}
    state = 4 * B * Hkv * d * dv
    rows = e * B * (H * (d + dv) + Hkv * (d + dv))
    if kind == "step":
        return {"bytes": 2 * state + rows, "flops": B * (3 * Hkv + 2 * H) * d * dv}
    mean = 0.5 if case["ragged"] else 1.0
    ends = state if case["states"] else 0
    if kind == "prompt":
        return {"bytes": mean * N * rows + 2 * ends, "flops": mean * B * N * (2 * Hkv + 2 * H) * d * dv}
    # Q, K, V, dO in; dQ, dK, dV out
    return {"bytes": N * (mean * rows + e * B * (H * d + Hkv * (d + dv))) + 3 * ends, "flops": mean * B * N * (2 * Hkv + 4 * H + 4 * Hkv) * d * dv}


def exact(case, seed):
    """The recurrence itself, token by token, in 64 bits."""
    s = prepare(case, seed)
    kind = s["kind"]
    if kind == "cache":
        top = 127.0 if s["format"] == "i8" else 448.0
        S = s["S"].double()
        sc = (S.abs().amax(-1, keepdim=True) / top).float().double()
        u = S / sc
        if s["format"] == "i8":
            u = torch.round(u)
        else:                   # e4m3: three bits behind the leading one, steps of 2^-9 below 2^-6
            step = torch.exp2(torch.floor(torch.log2(u.abs().clamp(min=2.0 ** -6))) - 3)
            u = torch.round(u / step) * step
        scales = s["scales"].double()
        scales[s["slots"].long()] = sc[..., 0]
        return u * sc, scales
    lam = torch.exp(s["log_decay"].double())
    scale = s["scale"]
    if kind == "step":
        G = s["q"].shape[1] // s["k"].shape[1]
        pool, o = s["S"].double(), []
        at = s["slots"].long()
        for b in range(len(at)):
            S = lam[:, None, None] * pool[at[b]] + torch.einsum("ha,hc->hac", s["k"][b].double(), s["v"][b].double())
            pool[at[b]] = S
            o.append(scale * torch.einsum("hga,hac->hgc", s["q"][b].double().reshape(S.shape[0], G, -1), S).reshape(-1, S.shape[2]))
        return torch.stack(o), pool
    Q, K, V = s["Q"].double(), s["K"].double(), s["V"].double()
    B, H, N, d = Q.shape
    Hkv, dv = K.shape[1], V.shape[3]
    G = H // Hkv
    n = torch.full((B,), N, device="cuda") if s["lengths"] is None else s["lengths"].long()
    live = (torch.arange(N, device="cuda")[:, None] < n).double()[:, :, None, None, None]       # [N, B, 1, 1, 1]
    # a state that its sequence's end has passed stays as it is
    fade = torch.where(live > 0, lam[:, None, None], torch.ones_like(lam)[:, None, None])       # [N, B, Hkv, 1, 1]
    Kt, Vt = (t.permute(2, 0, 1, 3).contiguous() * live[..., 0] for t in (K, V))                 # [N, B, Hkv, .]
    Qt = Q.reshape(B, Hkv, G, N, d).permute(3, 0, 1, 2, 4).contiguous() * live                   # [N, B, Hkv, G, d]
    S = torch.zeros(B, Hkv, d, dv, device="cuda", dtype=torch.float64) if s["S_in"] is None else s["S_in"].double()
    if kind == "prompt":
        O = torch.empty(N, B, Hkv, G, dv, device="cuda", dtype=torch.float64)
        for t in range(N):
            S = fade[t] * S + Kt[t][..., None] * Vt[t][..., None, :]
            torch.matmul(Qt[t], S, out=O[t])
        O = scale * (O * live).permute(1, 2, 3, 0, 4).reshape(B, H, N, dv)
        return O, S if s["S_in"] is not None else None
    Dt = s["dO"].double().reshape(B, Hkv, G, N, dv).permute(3, 0, 1, 2, 4).contiguous() * live
    dQ, dK, dV = torch.empty_like(Qt), torch.empty_like(Kt), torch.empty_like(Vt)
    for t in range(N):
        S = fade[t] * S + Kt[t][..., None] * Vt[t][..., None, :]
        torch.matmul(Dt[t], S.transpose(-1, -2), out=dQ[t])
    R = torch.zeros_like(S) if s["dS_out"] is None else s["dS_out"].double()
    for t in range(N - 1, -1, -1):
        R = R + scale * (Qt[t].transpose(-1, -2) @ Dt[t])
        dK[t] = (R @ Vt[t][..., None])[..., 0]
        dV[t] = (Kt[t][..., None, :] @ R)[..., 0, :]
        R = fade[t] * R
    dQ = scale * dQ.permute(1, 2, 3, 0, 4).reshape(B, H, N, d)
    return dQ, dK.permute(1, 2, 0, 3), dV.permute(1, 2, 0, 3), R if s["S_in"] is not None else None
