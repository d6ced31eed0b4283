"""The selective operators of a causal model and the group norm of its frames, one call per pass: the short convolution that mixes
neighbouring tokens of each channel, the selective scan whose decay and input the tokens choose themselves, and the group norm
(with its activation) of channels-last hidden states.

Two forms of each: the plain one in elementary torch operations, and (`own`) the library's calls.

  conv                a_t = bias + sum_j W_j x_{t-(K-1)+j} per channel, y = a or silu(a), with the last K-1 inputs in and out
  conv_token          the same for one token of each of a server's sequences, inputs kept in a pool
  conv_backward       gradients of conv for x, W, bias and the inputs it began from
  scan                D = softplus(dt + bias), h_t = exp(D A) h_{t-1} + D u_t B_t, y_t = (C_t . h_t + skip u_t) silu(z_t), state in and out
  scan_token          the same for one token of each of a server's sequences, states picked out of a pool
  scan_backward       gradients of scan for all of its inputs
  groupnorm           statistics over the rows of a frame (or clip) and a group of channels, y = w xh + b or its silu
  groupnorm_backward  its gradients for x, w and b
"""
from __future__ import annotations

import math

import torch

own = False

EPS = 1e-5


def _conv(name, op, B, H, N, d, taps, silu=True, dtype="bf16", layout="bhnd", ragged=False, cache=True):
    return {"name": name, "op": op, "B": B, "H": H, "N": N, "d": d, "taps": taps, "silu": silu, "dtype": dtype, "layout": layout,
            "ragged": ragged, "cache": cache}


def _conv_token(name, rows, idle, pool, H, d, taps, silu=True, dtype="bf16"):
    return {"name": name, "op": "conv_token", "B": rows, "idle": idle, "pool": pool, "H": H, "N": 1, "d": d, "taps": taps, "silu": silu,
            "dtype": dtype, "layout": "packed"}


def _scan(name, op, B, H, N, d, G=1, n=16, gate=True, dtype="bf16", layout="bhnd", ragged=False, state=True):
    return {"name": name, "op": op, "B": B, "H": H, "N": N, "d": d, "G": G, "n": n, "gate": gate, "dtype": dtype, "layout": layout,
            "ragged": ragged, "state": state}


def _scan_token(name, rows, idle, pool, H, d, G=1, n=16, gate=True, dtype="bf16"):
    return {"name": name, "op": "scan_token", "B": rows, "idle": idle, "pool": pool, "H": H, "N": 1, "d": d, "G": G, "n": n, "gate": gate,
            "dtype": dtype, "layout": "bhnd"}


def _group(name, op, B, H, N, d, groups, silu=True, dtype="bf16"):
    return {"name": name, "op": op, "B": B, "H": H, "N": N, "d": d, "groups": groups, "silu": silu, "dtype": dtype}


def listed():
    return [
        # the 2B model's hidden states of a 480p clip before a scan, from the beginning of the sequence
        _conv("conv_hidden_480p", "conv", 1, 1, 21 * 30 * 52, 2240, 4, layout="packed", cache=False),
        # a server's padded batch of prompts of unequal, odd lengths that go on from earlier ones, no activation, fp32
        _conv("conv_ragged_f32", "conv", 7, 8, 1501, 128, 3, silu=False, dtype="f32", layout="bnhd", ragged=True),
        # a server's step: 192 sequences of a pool of 256, some rows of the batch idle
        _conv_token("conv_token_batch", 192, 5, 256, 1, 2240, 4),
        # training step on the 2B model's heads (before q, k or v of a decayed attention), clips of different lengths
        _conv("conv_train_ragged", "conv_backward", 2, 20, 9 * 30 * 52, 112, 4, layout="bnhd", ragged=True),
        # a 480p clip at the 2B model's width, gate as a view of one projection's output, from an empty state
        _scan("scan_hidden_480p", "scan", 1, 1, 21 * 30 * 52, 2240, layout="packed", state=False),
        # fp32 twin with heads in two groups on a padded batch, state in and out, no gate
        _scan("scan_ragged_f32", "scan", 5, 4, 1501, 112, G=2, n=8, gate=False, dtype="f32", layout="bnhd", ragged=True),
        # one sequence's next token: launches and latency
        _scan_token("scan_token_single", 1, 0, 4, 1, 2240),
        # a server's step: 192 sequences of a pool of 256, some rows of the batch idle
        _scan_token("scan_token_batch", 192, 5, 256, 1, 2240),
        # training step on two blocks of the 480p clip
        _scan("scan_train_block", "scan_backward", 2, 1, 3 * 30 * 52, 2240, layout="packed"),
        # each frame of a 480p clip by itself, before the temporal convolution
        _group("group_frames_480p", "groupnorm", 1, 21, 30 * 52, 2240, 32),
        # small frames whose groups are ten channels, no activation, fp32
        _group("group_small_f32", "groupnorm", 3, 1, 901, 320, 32, silu=False, dtype="f32"),
        # training step with statistics over the whole clip
        _group("group_train_clip", "groupnorm_backward", 1, 1, 9 * 30 * 52, 2240, 32),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """Another case of the same ranges: every operator, lengths from one token to the 480p clip, narrow and wide channels, both types."""
    while True:
        op = rng.choice(["conv", "conv_token", "conv_backward", "scan", "scan", "scan_token", "scan_backward", "scan_backward", "groupnorm",
                         "groupnorm", "groupnorm_backward"])
        dtype = rng.choice(["bf16", "bf16", "f32"])
        if rng.random() < 0.5:
            H, d = 1, 8 * _log_int(rng, 2, 560)
        else:
            H, d = rng.choice([2, 4, 5, 8, 16, 20]), rng.choice([32, 64, 112, 128])
        B, N, layout, ragged = rng.choice([1, 1, 2, 3, 7]), _log_int(rng, 1, 32760), rng.choice(["bhnd", "bnhd", "packed"]), rng.random() < 0.4
        rows = _log_int(rng, 1, 256)
        idle, pool = rng.randint(0, rows // 8), rows + rng.randint(0, 64)
        n, gate, carried, silu = rng.choice([8, 16, 16]), rng.random() < 0.7, rng.random() < 0.6, rng.random() < 0.7
        G = rng.choice([g for g in range(1, H + 1) if H % g == 0])
        taps = rng.choice([2, 3, 4, 4])
        if op == "conv_token":
            c = _conv_token("", rows, idle, pool, H, d, taps, silu, dtype)
        elif op.startswith("conv"):
            c = _conv("", op, B, H, N, d, taps, silu, dtype, layout, ragged, carried)
        elif op == "scan_token":
            c = _scan_token("", rows, idle, pool, H, d, G, n, gate, dtype)
        elif op.startswith("scan"):
            c = _scan("", op, B, H, N, d, G, n, gate, dtype, layout, ragged, carried)
        else:
            d = 8 * _log_int(rng, 4, 560)
            c = _group("", op, rng.choice([1, 2, 3]), rng.choice([1, 1, 3, 21]), N, d, rng.choice([g for g in (1, 4, 8, 10, 16, 32, 40) if d % g == 0]),
                       silu, dtype)
        del c["name"]
        if work(c)["bytes"] > 4.4e8:
            continue
        if op in ("scan", "scan_backward") and B * N * H * d * n > (1.18e9 if op == "scan" else 3.36e8):
            continue
        return c


# ---- inputs -------------------------------------------------------------------------------------------------------

def _type(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def _randn(gen, *shape):
    return torch.randn(shape, generator=gen, device="cuda")


def _views(case, gen, count=1, layout=None):
    """`count` token tensors [B][H][N][d]: heads outside tokens ("bhnd"), token-major ("bnhd"), or views of one projection's output that
    holds two of them side by side ("packed")."""
    B, H, N, d, dt = case["B"], case["H"], case["N"], case["d"], _type(case)
    layout = layout or case.get("layout", "bhnd")
    if layout == "packed":
        return [_randn(gen, B, N, 2, H, d).to(dt)[:, :, i % 2].permute(0, 2, 1, 3) for i in range(count)]
    if layout == "bhnd":
        return [_randn(gen, B, H, N, d).to(dt) for _ in range(count)]
    return [_randn(gen, B, N, H, d).to(dt).permute(0, 2, 1, 3) for _ in range(count)]


def _dense(case):
    """The layout of a kernel's output: token-major where the inputs are views."""
    return "bhnd" if case.get("layout", "bhnd") == "bhnd" else "bnhd"


def _out(case):
    B, H, N, d, dt = case["B"], case["H"], case["N"], case["d"], _type(case)
    if _dense(case) == "bhnd":
        return torch.zeros((B, H, N, d), dtype=dt, device="cuda")
    return torch.zeros((B, N, H, d), dtype=dt, device="cuda").permute(0, 2, 1, 3)


def _as(x):
    """A zeroed tensor that lies as x does (a view of a projection's output: in one of its own)."""
    return torch.empty_strided(x.shape, x.stride(), dtype=x.dtype, device="cuda").zero_()


def _lengths(case):
    """Tokens of each sequence of a padded batch: the whole row, none, one, and lengths spread between."""
    B, N = case["B"], case["N"]
    if not case["ragged"]:
        return [N] * B
    return [N, 0, 1][:B if B < 3 else 3] + [N * (2 * b + 1) // (2 * B) for b in range(3, B)] if B != 2 else [N, (2 * N) // 3]


def _slots(case, seed):
    order = torch.randperm(case["pool"], generator=torch.Generator().manual_seed(int(seed)))[:case["B"]].to(torch.int32)
    order[case["B"] - case["idle"]:] = -1
    return order.cuda()


def _prepare_conv(case, seed, gen):
    B, H, d, K, dt = case["B"], case["H"], case["d"], case["taps"], _type(case)
    s = {"case": case, "W": _randn(gen, K, H, d) * K ** -0.5, "bias": 0.1 * _randn(gen, H, d)}
    s["x"], = _views(case, gen)
    if case["op"] == "conv_token":
        s["y"] = _out(case)
        s["slots"] = _slots(case, seed)
        s["cache_in"] = _randn(gen, case["pool"], H, K - 1, d).to(dt)
        s["cache_out"] = s["cache_in"].clone()
        return s
    s["lengths"] = torch.tensor(_lengths(case), dtype=torch.int32, device="cuda") if case["ragged"] else None
    s["cache_in"] = _randn(gen, B, H, K - 1, d).to(dt) if case["cache"] else None
    if case["op"] == "conv":
        s["y"], s["cache_out"] = _out(case), torch.zeros((B, H, K - 1, d), dtype=dt, device="cuda")
    else:
        s["dy"], = _views(case, gen, layout=_dense(case))
        s["dcache_out"] = _randn(gen, B, H, K - 1, d).to(dt) if case["cache"] else None
        s["dx"], s["dcache_in"] = _as(s["x"]), torch.zeros((B, H, K - 1, d), dtype=dt, device="cuda")
        s["dW"], s["dbias"] = torch.zeros((K, H, d), device="cuda"), torch.zeros((H, d), device="cuda")
    return s


def _prepare_scan(case, seed, gen):
    B, H, N, d, G, n, dt = case["B"], case["H"], case["N"], case["d"], case["G"], case["n"], _type(case)
    s = {"case": case}
    s["u"], s["dt"] = _views(case, gen, 2, _dense(case))
    s["z"] = _views(case, gen)[0] if case["gate"] else None
    bc = _randn(gen, B, N, 2, G, n).to(dt)                            # views of one projection's output
    s["Bm"], s["Cm"] = (bc[:, :, i].permute(0, 2, 1, 3) for i in range(2))
    # state i of a channel decays about i + 1 times as fast as its first; steps of a thousandth to a tenth
    s["A"] = -torch.arange(1, n + 1, dtype=torch.float32, device="cuda") * torch.exp(0.1 * _randn(gen, H, d, n))
    step = torch.exp(math.log(1e-3) + math.log(1e2) * torch.rand((H, d), generator=gen, device="cuda"))
    s["dt_bias"] = torch.log(torch.expm1(step))
    s["skip"] = 1.0 + 0.1 * _randn(gen, H, d)
    if case["op"] == "scan_token":
        s["y"], s["slots"] = _out(case), _slots(case, seed)
        s["S_in"] = _randn(gen, case["pool"], H, d, n)
        s["S_out"] = s["S_in"].clone()
        return s
    s["lengths"] = torch.tensor(_lengths(case), dtype=torch.int32, device="cuda") if case["ragged"] else None
    s["S_in"] = _randn(gen, B, H, d, n) if case["state"] else None
    if case["op"] == "scan":
        s["y"], s["S_out"] = _out(case), torch.zeros((B, H, d, n), device="cuda")
        return s
    s["dy"], = _views(case, gen, layout=_dense(case))
    s["dS_out"] = _randn(gen, B, H, d, n) if case["state"] else None
    s["du"], s["ddt"], s["dz"] = _as(s["u"]), _as(s["dt"]), _as(s["z"]) if case["gate"] else None
    s["dB"], s["dC"] = _as(s["Bm"]), _as(s["Cm"])
    s["dS_in"], s["dA"] = torch.zeros((B, H, d, n), device="cuda"), torch.zeros((H, d, n), device="cuda")
    s["ddt_bias"], s["dskip"] = torch.zeros((H, d), device="cuda"), torch.zeros((H, d), device="cuda")
    return s


def _prepare_group(case, gen):
    B, H, N, d, G, dt = case["B"], case["H"], case["N"], case["d"], case["groups"], _type(case)
    s = {"case": case, "w": 1.0 + 0.2 * _randn(gen, d), "b": 0.1 * _randn(gen, d)}
    # channels have levels and spreads of their own
    s["x"] = (_randn(gen, B, H, N, d) * torch.exp(0.3 * _randn(gen, d)) + 0.5 * _randn(gen, d)).to(dt)
    if case["op"] == "groupnorm":
        s["y"] = torch.zeros((B, H, N, d), dtype=dt, device="cuda")
        s["mean"], s["rstd"] = (torch.zeros((B, H, G), device="cuda") for _ in range(2))
    else:
        s["dy"] = _randn(gen, B, H, N, d).to(dt)
        s["mean"], s["rstd"] = _group_statistics(s["x"], G)
        s["dx"] = torch.zeros((B, H, N, d), dtype=dt, device="cuda")
        s["dw"], s["db"] = (torch.zeros(d, device="cuda") for _ in range(2))
    return s


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    if case["op"].startswith("conv"):
        return _prepare_conv(case, seed, gen)
    if case["op"].startswith("scan"):
        return _prepare_scan(case, seed, gen)
    return _prepare_group(case, gen)


# ---- plain forms ----------------------------------------------------------------------------------------------------

def _silu_slope(a):
    g = torch.sigmoid(a)
    return g * (1 + a * (1 - g))


def _kept(s):
    """Which rows are tokens [B][1][N][1], and the sequences' lengths."""
    B, N = s["case"]["B"], s["case"]["N"]
    lengths = s["lengths"].long() if s["lengths"] is not None else torch.full((B,), N, device="cuda")
    return (torch.arange(N, device="cuda")[None, :] < lengths[:, None])[:, None, :, None], lengths


def _extended(s, keep):
    """Cache and tokens one after the other, fp32: [B][H][K-1+N][d]."""
    x = torch.where(keep, s["x"].float(), torch.zeros((), device="cuda"))
    B, H, _, d = x.shape
    before = s["cache_in"].float() if s["cache_in"] is not None else x.new_zeros((B, H, s["case"]["taps"] - 1, d))
    return torch.cat([before, x], dim=2)


def _tail(s, lengths):
    """Rows of the extended tokens that the cache behind a call holds: [B][1][K-1][1]."""
    return (lengths[:, None] + torch.arange(s["case"]["taps"] - 1, device="cuda")[None])[:, None, :, None]


def _mixed(s, ext):
    N, K = s["case"]["N"], s["case"]["taps"]
    a = s["bias"][None, :, None, :].expand(ext.shape[0], -1, N, -1)
    for j in range(K):
        a = a + s["W"][j][None, :, None, :] * ext[:, :, j:j + N]
    return a


def _plain_conv(s):
    keep, lengths = _kept(s)
    ext = _extended(s, keep)
    a = _mixed(s, ext)
    y = a * torch.sigmoid(a) if s["case"]["silu"] else a
    dt = s["x"].dtype
    at = _tail(s, lengths).expand(-1, ext.shape[1], -1, ext.shape[3])
    return {"y": torch.where(keep, y, torch.zeros((), device="cuda")).to(dt), "cache_out": torch.gather(ext, 2, at).to(dt)}


def _plain_conv_token(s):
    rows = s["case"]["B"] - s["case"]["idle"]                       # the idle ones are the batch's last
    at = s["slots"][:rows].long()
    ext = torch.cat([s["cache_in"][at], s["x"][:rows]], dim=2)
    a = (s["W"].permute(1, 0, 2)[None] * ext.float()).sum(2) + s["bias"]
    y = a * torch.sigmoid(a) if s["case"]["silu"] else a
    s["y"][:rows, :, 0] = y.to(s["y"].dtype)
    s["cache_out"][at] = ext[:, :, 1:]
    return {"y": s["y"], "cache_out": s["cache_out"]}


def _plain_conv_backward(s):
    N, K, dt = s["case"]["N"], s["case"]["taps"], s["x"].dtype
    keep, lengths = _kept(s)
    ext = _extended(s, keep)
    da = torch.where(keep, s["dy"].float(), torch.zeros((), device="cuda"))
    if s["case"]["silu"]:
        da = da * _silu_slope(_mixed(s, ext))
    dext = torch.zeros_like(ext)
    for j in range(K):
        dext[:, :, j:j + N] += s["W"][j][None, :, None, :] * da
    if s["dcache_out"] is not None:
        dext.scatter_add_(2, _tail(s, lengths).expand(-1, ext.shape[1], -1, ext.shape[3]), s["dcache_out"].float())
    dW = torch.stack([(da * ext[:, :, j:j + N]).sum((0, 2)) for j in range(K)])
    dx = torch.where(keep, dext[:, :, K - 1:], torch.zeros((), device="cuda"))
    return {"dx": dx.to(dt), "dcache_in": dext[:, :, :K - 1].to(dt), "dW": dW, "dbias": da.sum((0, 2))}


def _softplus(x):
    return x.clamp_min(0) + torch.log1p(torch.exp(-x.abs()))


def _channels(x, G):
    """[B][H][N][d] -> [B][N][G][channels of a group], fp32."""
    B, H, N, d = x.shape
    return x.float().permute(0, 2, 1, 3).reshape(B, N, G, H // G * d)


def _tokens(x, like):
    """The way back, rounded."""
    B, H, N, d = like.shape
    return x.reshape(B, N, H, d).permute(0, 2, 1, 3).to(like.dtype)


def _shared(x):
    """[B][G][N][n] -> [B][N][G][1][n], fp32."""
    return x.float().permute(0, 2, 1, 3)[:, :, :, None]


def _recurrence(a, b, state):
    """x_t = a_t x_{t-1} + b_t over the second axis, from `state`: runs of tokens side by side, then one run after the other."""
    N = a.shape[1]
    T = max(1, math.isqrt(N))
    runs = -(-N // T)
    if runs * T != N:
        more = list(a.shape)
        more[1] = runs * T - N
        a, b = torch.cat([a, a.new_ones(more)], dim=1), torch.cat([b, b.new_zeros(more)], dim=1)
    a, b = a.unflatten(1, (runs, T)), b.unflatten(1, (runs, T))
    x, p = torch.empty_like(a), torch.empty_like(a)
    x[:, :, 0], p[:, :, 0] = b[:, :, 0], a[:, :, 0]
    for t in range(1, T):
        torch.addcmul(b[:, :, t], a[:, :, t], x[:, :, t - 1], out=x[:, :, t])
        torch.mul(a[:, :, t], p[:, :, t - 1], out=p[:, :, t])
    for r in range(runs):
        x[:, r].addcmul_(p[:, r], state[:, None])
        state = x[:, r, -1]
    return x.flatten(1, 2)[:, :N]


def _scan_terms(s):
    """What forward and backward share; rows that are no tokens keep the state (a = 1) and add nothing."""
    G = s["case"]["G"]
    keep, _ = _kept(s)
    keep = keep.permute(0, 2, 1, 3)                                   # [B][N][1][1]
    nothing = torch.zeros((), device="cuda")
    pre = _channels(s["dt"], G) + s["dt_bias"].view(G, -1)
    D = torch.where(keep, _softplus(pre), nothing)
    u = torch.where(keep, _channels(s["u"], G), nothing)
    A = s["A"].view(G, -1, s["case"]["n"])
    Bm, Cm = (torch.where(keep[..., None], _shared(s[k]), nothing) for k in ("Bm", "Cm"))
    a = torch.exp(D[..., None] * A)
    b = (D * u)[..., None] * Bm
    B = s["case"]["B"]
    state = s["S_in"].reshape(B, G, -1, s["case"]["n"]) if s["S_in"] is not None else a.new_zeros((B,) + tuple(A.shape))
    return keep, nothing, pre, D, u, A, Bm, Cm, a, b, state


def _plain_scan(s):
    G = s["case"]["G"]
    keep, nothing, _, _, u, _, _, Cm, a, b, state = _scan_terms(s)
    h = _recurrence(a, b, state)
    y = (h * Cm).sum(-1) + s["skip"].view(G, -1) * u
    if s["z"] is not None:
        z = _channels(s["z"], G)
        y = y * (z * torch.sigmoid(z))
    return {"y": _tokens(torch.where(keep, y, nothing), s["y"]), "S_out": h[:, -1].reshape(s["S_out"].shape).clone()}


def _plain_scan_token(s):
    case = s["case"]
    rows, G, n = case["B"] - case["idle"], case["G"], case["n"]
    at = s["slots"][:rows].long()
    u, D = (s[k][:rows, :, 0].float() for k in ("u", "dt"))          # [rows][H][d]
    D = _softplus(D + s["dt_bias"])
    Bm, Cm = (s[k][:rows, :, 0].float().repeat_interleave(case["H"] // G, dim=1)[:, :, None] for k in ("Bm", "Cm"))
    h = torch.exp(D[..., None] * s["A"]) * s["S_in"][at] + (D * u)[..., None] * Bm
    y = (h * Cm).sum(-1) + s["skip"] * u
    if s["z"] is not None:
        z = s["z"][:rows, :, 0].float()
        y = y * (z * torch.sigmoid(z))
    s["S_out"][at] = h
    s["y"][:rows, :, 0] = y.to(s["y"].dtype)
    return {"y": s["y"], "S_out": s["S_out"]}


def _plain_scan_backward(s):
    G, n = s["case"]["G"], s["case"]["n"]
    keep, nothing, pre, D, u, A, Bm, Cm, a, b, state = _scan_terms(s)
    h = _recurrence(a, b, state)
    del b
    skip = s["skip"].view(G, -1)
    dy = torch.where(keep, _channels(s["dy"], G), nothing)
    out = {}
    if s["z"] is not None:
        z = torch.where(keep, _channels(s["z"], G), nothing)
        out["dz"] = _tokens(dy * ((h * Cm).sum(-1) + skip * u) * _silu_slope(z), s["dz"])
        dy = dy * (z * torch.sigmoid(z))
    last = s["dS_out"].reshape(state.shape) if s["dS_out"] is not None else torch.zeros_like(state)
    behind = torch.cat([a[:, 1:], torch.ones_like(a[:, :1])], dim=1)
    g = _recurrence(behind.flip(1), (dy[..., None] * Cm).flip(1), last).flip(1)
    out["dC"] = (dy[..., None] * h).sum(3).permute(0, 2, 1, 3).to(s["dC"].dtype)
    out["dB"] = (g * (D * u)[..., None]).sum(3).permute(0, 2, 1, 3).to(s["dB"].dtype)
    along = (g * Bm).sum(-1)
    before = torch.cat([state[:, None], h[:, :-1]], dim=1)
    p = g * a * before
    dD = torch.where(keep, (p * A).sum(-1) + along * u, nothing)
    ddt = dD * torch.sigmoid(pre)
    shape = s["skip"].shape
    out["du"] = _tokens(D * along + skip * dy, s["du"])
    out["ddt"] = _tokens(ddt, s["ddt"])
    out["dA"] = (p * D[..., None]).sum((0, 1)).view(s["A"].shape)
    out["ddt_bias"], out["dskip"] = ddt.sum((0, 1)).view(shape), (dy * u).sum((0, 1)).view(shape)
    out["dS_in"] = (a[:, 0] * g[:, 0]).view(s["dS_in"].shape)
    return out


def _group_statistics(x, G):
    B, H, N, d = x.shape
    x = x.float().view(B, H, N, G, d // G)
    mean = x.mean((2, 4), keepdim=True)
    var = (x - mean).square().mean((2, 4))
    return mean.view(B, H, G), (var + EPS).rsqrt()


def _by_channel(p, d):
    """[B][H][G] -> [B][H][1][d]"""
    return p.repeat_interleave(d // p.shape[-1], dim=-1)[:, :, None]


def _plain_group(s):
    d = s["case"]["d"]
    mean, rstd = _group_statistics(s["x"], s["case"]["groups"])
    a = (s["x"].float() - _by_channel(mean, d)) * _by_channel(rstd, d) * s["w"] + s["b"]
    y = a * torch.sigmoid(a) if s["case"]["silu"] else a
    return {"y": y.to(s["y"].dtype), "mean": mean, "rstd": rstd}


def _plain_group_backward(s):
    case = s["case"]
    B, H, N, d = s["x"].shape
    rstd = _by_channel(s["rstd"], d)
    xh = (s["x"].float() - _by_channel(s["mean"], d)) * rstd
    da = s["dy"].float()
    if case["silu"]:
        da = da * _silu_slope(xh * s["w"] + s["b"])
    t = da * s["w"]

    def level(v):
        return _by_channel(v.view(B, H, N, case["groups"], -1).mean((2, 4)), d)
    dx = rstd * (t - level(t) - xh * level(t * xh))
    return {"dx": dx.to(s["dx"].dtype), "dw": (da * xh).sum((0, 1, 2)), "db": da.sum((0, 1, 2))}


# ---- the library's calls ----------------------------------------------------------------------------------------------

def _once(s, name, make):
    """A descriptor or workspace that a program makes once and keeps beside its buffers."""
    if name not in s:
        s[name] = make()
    return s[name]


def _desc(s, sv, name):
    return _once(s, "desc_" + name, lambda: sv.desc_of(s[name])) if s[name] is not None else None


def _space(nbytes):
    return torch.empty(nbytes, dtype=torch.uint8, device="cuda")


def _own_conv(s):
    import paper_2509_24695_amd as sv
    sv.sv_causal_conv(s["x"], _desc(s, sv, "x"), s["W"], s["bias"], s["case"]["taps"], s["case"]["silu"], s["lengths"], s["cache_in"],
                      s["cache_out"], s["y"], _desc(s, sv, "y"), stream=torch.cuda.current_stream())
    return {"y": s["y"], "cache_out": s["cache_out"]}


def _own_conv_token(s):
    import paper_2509_24695_amd as sv
    sv.sv_causal_conv_token(s["x"], _desc(s, sv, "x"), s["W"], s["bias"], s["case"]["taps"], s["case"]["silu"], s["slots"], s["case"]["pool"],
                            s["cache_in"], s["cache_out"], s["y"], _desc(s, sv, "y"), stream=torch.cuda.current_stream())
    return {"y": s["y"], "cache_out": s["cache_out"]}


def _own_conv_backward(s):
    import paper_2509_24695_amd as sv
    ws = _once(s, "ws", lambda: _space(sv.sv_causal_conv_backward_workspace_bytes(*s["x"].shape)))
    sv.sv_causal_conv_backward(s["x"], _desc(s, sv, "x"), s["dy"], _desc(s, sv, "dy"), s["W"], s["bias"], s["case"]["taps"], s["case"]["silu"],
                               s["lengths"], s["cache_in"], s["dcache_out"], s["dx"], _desc(s, sv, "dx"), s["dcache_in"], s["dW"], s["dbias"],
                               ws, stream=torch.cuda.current_stream())
    return {"dx": s["dx"], "dcache_in": s["dcache_in"], "dW": s["dW"], "dbias": s["dbias"]}


def _own_scan(s):
    import paper_2509_24695_amd as sv
    ws = _once(s, "ws", lambda: _space(sv.sv_selective_scan_workspace_bytes(*s["u"].shape, s["case"]["n"])))
    sv.sv_selective_scan(s["u"], s["dt"], _desc(s, sv, "u"), s["z"], _desc(s, sv, "z"), s["Bm"], s["Cm"], _desc(s, sv, "Bm"), s["A"], s["dt_bias"],
                         s["skip"], s["lengths"], s["S_in"], s["S_out"], s["y"], _desc(s, sv, "y"), ws, stream=torch.cuda.current_stream())
    return {"y": s["y"], "S_out": s["S_out"]}


def _own_scan_token(s):
    import paper_2509_24695_amd as sv
    sv.sv_selective_scan_token(s["u"], s["dt"], _desc(s, sv, "u"), s["z"], _desc(s, sv, "z"), s["Bm"], s["Cm"], _desc(s, sv, "Bm"), s["A"],
                               s["dt_bias"], s["skip"], s["slots"], s["case"]["pool"], s["S_in"], s["S_out"], s["y"], _desc(s, sv, "y"),
                               stream=torch.cuda.current_stream())
    return {"y": s["y"], "S_out": s["S_out"]}


def _own_scan_backward(s):
    import paper_2509_24695_amd as sv
    ws = _once(s, "ws", lambda: _space(sv.sv_selective_scan_backward_workspace_bytes(*s["u"].shape, s["case"]["G"], s["case"]["n"])))
    sv.sv_selective_scan_backward(s["u"], s["dt"], _desc(s, sv, "u"), s["z"], _desc(s, sv, "z"), s["Bm"], s["Cm"], _desc(s, sv, "Bm"), s["dy"],
                                  _desc(s, sv, "dy"), s["A"], s["dt_bias"], s["skip"], s["lengths"], s["S_in"], s["dS_out"], s["du"], s["ddt"],
                                  s["dz"], s["dB"], s["dC"], s["dS_in"], s["dA"], s["ddt_bias"], s["dskip"], ws,
                                  stream=torch.cuda.current_stream())
    names = ["du", "ddt", "dB", "dC", "dS_in", "dA", "ddt_bias", "dskip"] + (["dz"] if s["z"] is not None else [])
    return {k: s[k] for k in names}


def _own_group(s):
    import paper_2509_24695_amd as sv
    G = s["case"]["groups"]
    ws = _once(s, "ws", lambda: _space(sv.sv_groupnorm_workspace_bytes(*s["x"].shape, G)))
    sv.sv_groupnorm(s["x"], _desc(s, sv, "x"), s["w"], s["b"], G, EPS, s["case"]["silu"], s["y"], _desc(s, sv, "y"), s["mean"], s["rstd"], ws,
                    stream=torch.cuda.current_stream())
    return {"y": s["y"], "mean": s["mean"], "rstd": s["rstd"]}


def _own_group_backward(s):
    import paper_2509_24695_amd as sv
    G = s["case"]["groups"]
    ws = _once(s, "ws", lambda: _space(sv.sv_groupnorm_backward_workspace_bytes(*s["x"].shape, G)))
    sv.sv_groupnorm_backward(s["x"], _desc(s, sv, "x"), s["dy"], _desc(s, sv, "dy"), s["w"], s["b"], G, s["case"]["silu"], s["mean"], s["rstd"],
                             s["dx"], _desc(s, sv, "dx"), s["dw"], s["db"], ws, stream=torch.cuda.current_stream())
    return {"dx": s["dx"], "dw": s["dw"], "db": s["db"]}


_PLAIN = {"conv": _plain_conv, "conv_token": _plain_conv_token, "conv_backward": _plain_conv_backward, "scan": _plain_scan,
          "scan_token": _plain_scan_token, "scan_backward": _plain_scan_backward, "groupnorm": _plain_group,
          "groupnorm_backward": _plain_group_backward}
_OWN = {"conv": _own_conv, "conv_token": _own_conv_token, "conv_backward": _own_conv_backward, "scan": _own_scan,
        "scan_token": _own_scan_token, "scan_backward": _own_scan_backward, "groupnorm": _own_group, "groupnorm_backward": _own_group_backward}


def run(state):
    return (_OWN if own else _PLAIN)[state["case"]["op"]](state)


# ---- what a pass cannot do without ------------------------------------------------------------------------------------

def work(case):
    op, B, H, N, d = case["op"], case["B"], case["H"], case["N"], case["d"]
    elem, C = 4 if case["dtype"] == "f32" else 2, H * d
    if op == "conv_token":
        rows, K = B - case["idle"], case["taps"]
        return {"bytes": rows * C * elem * 2 * K + (K + 1) * C * 4 + B * 4, "flops": rows * C * (2 * K + 4)}
    if op.startswith("conv"):
        K, tokens = case["taps"], sum(_lengths(case)) * C
        caches = B * (K - 1) * C * elem * (1 + case["cache"] * (1 if op == "conv" else 2))
        if op == "conv":
            return {"bytes": tokens * 2 * elem + caches + (K + 1) * C * 4, "flops": tokens * (2 * K + 4)}
        return {"bytes": tokens * 3 * elem + caches + 2 * (K + 1) * C * 4, "flops": tokens * (6 * K + 10)}
    if op.startswith("scan"):
        n, G = case["n"], case["G"]
        params = C * (n + 2) * 4
        if op == "scan_token":
            rows = B - case["idle"]
            return {"bytes": rows * (C * (3 + case["gate"]) * elem + C * n * 8 + 2 * G * n * elem) + params + B * 4, "flops": rows * C * (7 * n + 20)}
        tokens = sum(_lengths(case))
        states = B * C * n * 4
        if op == "scan":
            return {"bytes": tokens * (C * (3 + case["gate"]) * elem + 2 * G * n * elem) + states * (1 + case["state"]) + params,
                    "flops": tokens * C * (7 * n + 20)}
        return {"bytes": tokens * (C * (5 + 2 * case["gate"]) * elem + 4 * G * n * elem) + states * (1 + 2 * case["state"]) + 2 * params,
                "flops": tokens * C * (21 * n + 40)}
    values, stats = B * H * N * d, 2 * B * H * case["groups"] * 4
    if op == "groupnorm":
        return {"bytes": values * 2 * elem + stats + 2 * d * 4, "flops": values * 12}
    return {"bytes": values * 3 * elem + stats + 4 * d * 4, "flops": values * 24}


# ---- the same in 64 bits, from the definitions ------------------------------------------------------------------------

def _exact_conv(s, backward):
    case = s["case"]
    B, H, N, d = s["x"].shape
    K = case["taps"]
    lengths = _lengths(case)
    W = s["W"].double().permute(1, 2, 0)                               # [H][d][K]
    y, dx = (torch.zeros((B, H, N, d), dtype=torch.float64, device="cuda") for _ in range(2))
    rows = torch.zeros((B, H, K - 1, d), dtype=torch.float64, device="cuda")
    cache_out, dcache_in = rows.clone(), rows.clone()
    dW, db = torch.zeros((K, H, d), dtype=torch.float64, device="cuda"), torch.zeros((H, d), dtype=torch.float64, device="cuda")
    for b in range(B):
        L = lengths[b]
        first = s["cache_in"][b].double() if s["cache_in"] is not None else rows[b]
        ext = torch.cat([first, s["x"][b, :, :L].double()], dim=1)     # [H][K-1+L][d]
        windows = ext.unfold(1, K, 1) if L else ext.new_zeros((H, 0, d, K))
        a = (windows * W[:, None]).sum(-1) + s["bias"].double()[:, None]
        if not backward:
            y[b, :, :L] = a / (1 + torch.exp(-a)) if case["silu"] else a
            cache_out[b] = ext[:, L:]
            continue
        da = s["dy"][b, :, :L].double()
        if case["silu"]:
            g = 1 / (1 + torch.exp(-a))
            da = da * (g + a * g * (1 - g))
        dext = torch.zeros_like(ext)
        for t in range(K):                                             # dext_m = sum_j W_j da_{m-j}
            dext[:, t:t + L] += da * W[:, None, :, t]
        if s["dcache_out"] is not None:
            dext[:, L:] += s["dcache_out"][b].double()
        dcache_in[b], dx[b, :, :L] = dext[:, :K - 1], dext[:, K - 1:]
        dW += (windows * da[..., None]).sum(1).permute(2, 0, 1)
        db += da.sum(1)
    return {"dx": dx, "dcache_in": dcache_in, "dW": dW, "dbias": db} if backward else {"y": y, "cache_out": cache_out}


def _exact_conv_token(s):
    y, cache = s["y"].double(), s["cache_out"].double()
    for row, slot in enumerate(s["slots"].tolist()):
        if slot < 0:
            continue
        window = torch.cat([s["cache_in"][slot].double(), s["x"][row].double()], dim=1)      # [H][K][d]
        a = s["bias"].double()
        for j in range(window.shape[1]):
            a = a + window[:, j] * s["W"][j].double()
        y[row, :, 0] = a / (1 + torch.exp(-a)) if s["case"]["silu"] else a
        cache[slot] = window[:, 1:]
    return {"y": y, "cache_out": cache}


def _exact_scan(s, backward):
    """The definition token by token, sequences side by side: one that has ended keeps its state."""
    case = s["case"]
    B, H, N, d, G, n = case["B"], case["H"], case["N"], case["d"], case["G"], case["n"]
    live = (torch.arange(N)[:, None] < torch.tensor(_lengths(case))[None]).cuda()[:, :, None, None]       # [N][B][1][1]

    def first(x):                                                      # [N][B][H][d], nothing where there is no token
        return torch.where(live, x.double().permute(2, 0, 1, 3), torch.zeros((), dtype=torch.float64, device="cuda")).contiguous()

    def heads(x):                                                      # [N][B][H][1][n]
        return first(x).repeat_interleave(H // G, dim=2)[:, :, :, None]
    u, pre = first(s["u"]), first(s["dt"]) + s["dt_bias"].double()
    D = torch.where(live, torch.log(1 + torch.exp(-pre.abs())) + pre.clamp_min(0), torch.zeros((), dtype=torch.float64, device="cuda"))
    Bm, Cm, A, skip = heads(s["Bm"]), heads(s["Cm"]), s["A"].double(), s["skip"].double()

    def begin(x):
        return x.double().clone() if x is not None else torch.zeros((B, H, d, n), dtype=torch.float64, device="cuda")

    def back(x):
        return x.permute(1, 2, 0, 3)
    h = begin(s["S_in"])
    y = skip * u
    states = [h] if backward else None
    for t in range(N):
        h = h * torch.exp(D[t][..., None] * A) + (D[t] * u[t])[..., None] * Bm[t]
        y[t] += (h * Cm[t]).sum(-1)
        if backward:
            states.append(h)
    z = first(s["z"]) if s["z"] is not None else None
    gate = 1 / (1 + torch.exp(-z)) if z is not None else None
    if not backward:
        y = torch.where(live, y, torch.zeros((), dtype=torch.float64, device="cuda"))
        return {"y": back(y if z is None else y * z * gate), "S_out": h}
    dy, out = first(s["dy"]), {}
    if z is not None:
        out["dz"] = back(dy * y * (gate + z * gate * (1 - gate)))
        dy = dy * z * gate
    g = begin(s["dS_out"])                                             # gradient of the state behind token t
    du, dD = skip * dy, torch.zeros_like(u)
    dB, dC = (torch.zeros((N, B, G, n), dtype=torch.float64, device="cuda") for _ in range(2))
    dA = torch.zeros_like(A)
    for t in range(N - 1, -1, -1):
        dC[t] = (states[t + 1] * dy[t][..., None]).view(B, G, -1, n).sum(2)
        g = g + Cm[t] * dy[t][..., None]
        dB[t] = (g * (D[t] * u[t])[..., None]).view(B, G, -1, n).sum(2)
        input_side = (g * Bm[t]).sum(-1)
        du[t] += D[t] * input_side
        g = g * torch.exp(D[t][..., None] * A)
        along = g * states[t]
        dA += (along * D[t][..., None]).sum(0)
        dD[t] = (along * A).sum(-1) + input_side * u[t]
    ddt = torch.where(live, dD / (1 + torch.exp(-pre)), torch.zeros((), dtype=torch.float64, device="cuda"))
    return {**out, "du": back(du), "ddt": back(ddt), "dB": dB.permute(1, 2, 0, 3), "dC": dC.permute(1, 2, 0, 3), "dS_in": g, "dA": dA,
            "ddt_bias": ddt.sum((0, 1)), "dskip": (dy * u).sum((0, 1))}


def _exact_scan_token(s):
    H, G = s["case"]["H"], s["case"]["G"]
    y, S = s["y"].double(), s["S_out"].double()
    for row, slot in enumerate(s["slots"].tolist()):
        if slot < 0:
            continue
        u, pre = s["u"][row, :, 0].double(), s["dt"][row, :, 0].double() + s["dt_bias"].double()
        D = torch.log(1 + torch.exp(-pre.abs())) + pre.clamp_min(0)
        Bm, Cm = (s[k][row, :, 0].double().repeat_interleave(H // G, dim=0)[:, None] for k in ("Bm", "Cm"))
        S[slot] = s["S_in"][slot].double() * torch.exp(D[..., None] * s["A"].double()) + (D * u)[..., None] * Bm
        out = (S[slot] * Cm).sum(-1) + s["skip"].double() * u
        if s["z"] is not None:
            z = s["z"][row, :, 0].double()
            out = out * z / (1 + torch.exp(-z))
        y[row, :, 0] = out
    return {"y": y, "S_out": S}


def _exact_group(s, backward):
    case = s["case"]
    B, H, N, d = s["x"].shape
    G = case["groups"]
    w, b = s["w"].double().view(G, 1, -1), s["b"].double().view(G, 1, -1)

    def grouped(x):                                                    # [B][H][G][N][d/G]
        return x.double().view(B, H, N, G, d // G).transpose(2, 3)

    def back(x):
        return x.transpose(2, 3).reshape(B, H, N, d)
    x = grouped(s["x"])
    count = N * (d // G)
    if not backward:
        mean = x.sum((3, 4)) / count
        rstd = (((x - mean[..., None, None]) ** 2).sum((3, 4)) / count + EPS) ** -0.5
        a = w * ((x - mean[..., None, None]) * rstd[..., None, None]) + b
        return {"y": back(a / (1 + torch.exp(-a)) if case["silu"] else a), "mean": mean, "rstd": rstd}
    mean, rstd, da = s["mean"].double()[..., None, None], s["rstd"].double()[..., None, None], grouped(s["dy"])
    xh = (x - mean) * rstd
    if case["silu"]:
        a = w * xh + b
        g = 1 / (1 + torch.exp(-a))
        da = da * (g + a * g * (1 - g))
    along, level = ((w * da * xh).sum((3, 4), keepdim=True) / count, (w * da).sum((3, 4), keepdim=True) / count)
    return {"dx": back((w * da - level - along * xh) * rstd), "dw": (da * xh).sum((0, 1, 3)).reshape(d), "db": da.sum((0, 1, 3)).reshape(d)}


def exact(case, seed):
    op = case["op"]
    if op == "scan_backward" and case["B"] * case["N"] * case["H"] * case["d"] * case["n"] * 8 > 4e10:
        return None                                                    # the states of all tokens
    s = prepare(case, seed)
    if op == "conv_token":
        return _exact_conv_token(s)
    if op.startswith("conv"):
        return _exact_conv(s, op == "conv_backward")
    if op == "scan_token":
        return _exact_scan_token(s)
    if op.startswith("scan"):
        return _exact_scan(s, op == "scan_backward")
    return _exact_group(s, op == "groupnorm_backward")
