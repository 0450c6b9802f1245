"""Performance cases of the operators around the step core's attention.

A block of a video diffusion transformer, run for the active frames of an asynchronous step, is
the step core's attention and three operators beside it:

  rope    rotary positions over time, height and width of the active frames' queries and keys
  cross   attention of the active frames' tokens to an encoder's states of another length
  linear  matrix product with bias, activation, gate and residual

``listed()`` gives the named cases and ``draw(rng)`` more of the same ranges; ``prepare`` makes
the inputs and output buffers a program holds before the call, ``run`` makes one pass (in plain
torch operations, or through the library's entry points where ``own`` is true), ``work`` states
the bytes and operations a pass cannot do without, and ``exact`` the result in 64 bits.

Shapes: F latent frames of N tokens (a grid of gh x gw), A of them active; H heads of dim d.
Rows of skipped frames are not computed: they keep what the output buffer holds (zeros).
"""
import math

import torch

own = False

DEV = "cuda"
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
SIZE = {"bf16": 2, "fp16": 2, "fp32": 4}
# exact() is left out above this many operations (64-bit rates: some seconds)
EXACT_FLOPS = 6.0e12


# ------------------------------------------------------------------------------ the cases
def listed():
    return [
        # Keyframe-only step of the smallest video, 4 frames of 8 x 8 tokens: a call's latency.
        dict(name="rope_tiny", kind="rope", F=4, A=2, gh=8, gw=8, H=2, Hk=2, d=64,
             dt=24, dh=20, dw=20, pairing="interleaved", inverse=False, fused=False, dtype="bf16"),
        # Queries and keys of the usual 81-frame 480p clip, every frame active.
        dict(name="rope_480p_all", kind="rope", F=21, A=21, gh=30, gw=52, H=12, Hk=12, d=128,
             dt=44, dh=42, dw=42, pairing="interleaved", inverse=False, fused=True, dtype="bf16"),
        # The widest: 720p, 40 heads, halves as pairs, fp16.
        dict(name="rope_720p_half", kind="rope", F=21, A=21, gh=45, gw=80, H=40, Hk=40, d=128,
             dt=32, dh=48, dw=48, pairing="half", inverse=False, fused=False, dtype="fp16"),
        # Rotation taken back (the gradient), odd grid, one key head for five query heads, part
        # of the head dim rotated, 32-bit data.
        dict(name="rope_odd_inverse", kind="rope", F=7, A=5, gh=17, gw=59, H=5, Hk=1, d=128,
             dt=16, dh=40, dw=40, pairing="half", inverse=True, fused=False, dtype="fp32"),
        # One token per sequence: 16 sequences with their own, ragged encoder states (a pooled
        # token per clip asking a long document): the form for single tokens.
        dict(name="cross_single", kind="cross", F=16, N=1, A=16, H=12, Hk=12, d=128, L=32000,
             ranges="lengths", kept=None, lse=False, fused=False, dtype="bf16"),
        # Keyframe-only step of a short 480p clip over a prompt of 512 text states.
        dict(name="cross_480p_keys", kind="cross", F=13, N=1560, A=4, H=12, Hk=12, d=128, L=512,
             ranges=None, kept=None, lse=False, fused=True, dtype="bf16"),
        # 720p clip with 40 heads, every frame active: the largest.
        dict(name="cross_720p_all", kind="cross", F=21, N=3600, A=21, H=40, Hk=40, d=128, L=512,
             ranges=None, kept=None, lse=False, fused=False, dtype="bf16"),
        # Each frame hears its own window of audio states, masked states among them; narrow
        # shared key heads, odd frame size, log-sum-exps kept for a merge.
        dict(name="cross_windows", kind="cross", F=33, N=1003, A=20, H=24, Hk=6, d=64, L=1500,
             ranges="windows", kept=1337, lse=True, fused=False, dtype="fp16"),
        # One row of time embedding to six modulation vectors: weights read once.
        dict(name="linear_row", kind="linear", F=1, N=1, A=1, K=1536, O=9216, dtype="bf16",
             out="fp32", bias=True, act="none", gate=None, residual=False),
        # First half of the feed-forward of a keyframe-only step of a short 480p clip.
        dict(name="linear_480p_keys", kind="linear", F=13, N=1560, A=4, K=1536, O=6144,
             dtype="bf16", out="bf16", bias=True, act="gelu_tanh", gate=None, residual=False),
        # Output projection of the 720p clip with 40 heads, gated per frame onto the stream.
        dict(name="linear_720p_gated", kind="linear", F=21, N=3600, A=21, K=5120, O=5120,
             dtype="bf16", out="bf16", bias=True, act="none", gate="frame", residual=True),
        # Odd sizes: a few prompt states projected to an odd width, 32-bit result.
        dict(name="linear_odd", kind="linear", F=1, N=333, A=1, K=1000, O=777, dtype="fp16",
             out="fp32", bias=True, act="silu", gate="shared", residual=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw_rope(rng):
    d = rng.choice([64, 128, 128])
    dh, dw = (2 * rng.randint(0, d // 6) for _ in range(2))
    rest = d - dh - dw
    dt = rest if rng.random() < 0.7 else 2 * rng.randint(1, rest // 2)
    H = _log_int(rng, 1, 40)
    F = _log_int(rng, 1, 33)
    return dict(kind="rope", F=F, A=rng.randint(1, F), gh=_log_int(rng, 1, 45),
                gw=_log_int(rng, 1, 80), H=H, Hk=rng.choice([0, 1, H, H]), d=d, dt=dt, dh=dh, dw=dw,
                pairing=rng.choice(["interleaved", "half"]), inverse=rng.random() < 0.3,
                fused=rng.random() < 0.5, dtype=rng.choice(["bf16", "bf16", "fp16", "fp32"]))


def _draw_cross(rng):
    F = _log_int(rng, 1, 33)
    Hk = _log_int(rng, 1, 40)
    H = Hk * rng.choice([1, 1, 2, 4]) if Hk <= 10 else Hk
    L = _log_int(rng, 1, 32000)
    N = rng.choice([1, _log_int(rng, 1, 3600), _log_int(rng, 64, 3600)])
    return dict(kind="cross", F=F, N=N,
                A=rng.randint(1, F), H=H, Hk=Hk, d=rng.choice([64, 128, 128]), L=L,
                ranges=rng.choice([None, None, "lengths", "windows"]),
                kept=rng.choice([None, rng.randint(0, L)]),
                lse=rng.random() < 0.5, fused=rng.random() < 0.5,
                dtype=rng.choice(["bf16", "bf16", "fp16"]))


def _draw_linear(rng):
    F = _log_int(rng, 1, 33)
    return dict(kind="linear", F=F, N=rng.choice([1, _log_int(rng, 1, 3600)]), A=rng.randint(1, F),
                K=_log_int(rng, 16, 8192), O=_log_int(rng, 8, 20480),
                dtype=rng.choice(["bf16", "bf16", "fp16"]),
                out=rng.choice(["same", "same", "fp32"]), bias=rng.random() < 0.7,
                act=rng.choice(["none", "none", "gelu_tanh", "gelu", "silu"]),
                gate=rng.choice([None, None, "shared", "frame"]), residual=rng.random() < 0.4)


def draw(rng):
    kind = rng.choice(["rope", "cross", "linear"])
    while True:
        c = {"rope": _draw_rope, "cross": _draw_cross, "linear": _draw_linear}[kind](rng)
        if kind == "linear" and c["out"] == "same":
            c["out"] = c["dtype"]
        w, most = work(c), {"rope": (3.0e9, 1e15), "cross": (1.5e9, 7e11),
                            "linear": (2.5e9, 3.8e12)}[kind]
        rows = c["F"] * _tokens(c)
        # plain attention holds the scores: rows x heads x keys in 32 bits
        scores = rows * c.get("H", 1) * c.get("L", 1) if kind == "cross" else 0
        if w["bytes"] <= most[0] and w["flops"] <= most[1] and scores <= 2.0e9:
            return c


# ------------------------------------------------------------------------------ inputs
def _tokens(c):
    return c["gh"] * c["gw"] if c["kind"] == "rope" else c["N"]


def _dims(c):
    """Rotated elements of a head per axis: time, height, width."""
    return c["dt"], c["dh"], c["dw"]


def _active(c):
    """The active frames, spread evenly."""
    return [i * c["F"] // c["A"] for i in range(c["A"])]


def _ranges(c):
    """Key rows [begin, end) of every frame, or None: all keys."""
    F, L = c["F"], c["L"]
    if c["ranges"] is None:
        return None
    if c["ranges"] == "lengths":  # packed sequences, ragged: frame f's share grows with f mod 3
        w = [1 + (f % 3) for f in range(F)]
        edge = [L * sum(w[:f]) // sum(w) for f in range(F + 1)]
        return [(edge[f], edge[f + 1]) for f in range(F)]
    half = max(1, L // 12)  # windows around each frame's instant, overlapping
    mid = [(2 * f + 1) * L // (2 * F) for f in range(F)]
    return [(max(0, m - half), min(L, m + half)) for m in mid]


def _keep(c, g):
    """uint8 [L]: `kept` of the encoder's states, scattered, or None: all of them."""
    if c["kept"] is None:
        return None
    keep = torch.zeros(c["L"], dtype=torch.uint8, device=DEV)
    keep[torch.randperm(c["L"], generator=g, device=DEV)[:c["kept"]]] = 1
    return keep


def _normal(g, *shape, dtype=torch.float32, std=1.0):
    return (torch.randn(*shape, generator=g, device=DEV) * std).to(dtype)


def _positions(c):
    return [torch.arange(n, dtype=torch.float64, device=DEV) for n in (c["F"], c["gh"], c["gw"])]


def _inputs(c, seed):
    """The random inputs by name; prepare() and exact() both start from these."""
    g = torch.Generator(device=DEV).manual_seed((seed * 1009 + 17) & 0x7FFFFFFFFFFF)
    dt, rows, t = DTYPES[c["dtype"]], c["F"] * _tokens(c), {}
    if c["kind"] == "rope":
        if c["fused"]:  # heads of one projection's rows: queries, keys, values
            b = _normal(g, rows, c["H"] + 2 * c["Hk"], c["d"], dtype=dt)
            t["Q"], t["K"] = b[:, :c["H"]], b[:, c["H"]:c["H"] + c["Hk"]] if c["Hk"] else None
        else:
            t["Q"] = _normal(g, rows, c["H"], c["d"], dtype=dt)
            t["K"] = _normal(g, rows, c["Hk"], c["d"], dtype=dt) if c["Hk"] else None
    elif c["kind"] == "cross":
        t["Q"] = _normal(g, rows, c["H"], c["d"], dtype=dt)
        if c["fused"]:  # one projection's rows: keys, values
            t["K"], t["V"] = _normal(g, c["L"], 2, c["Hk"], c["d"], dtype=dt).unbind(1)
        else:
            t["K"] = _normal(g, c["L"], c["Hk"], c["d"], dtype=dt)
            t["V"] = _normal(g, c["L"], c["Hk"], c["d"], dtype=dt)
        t["keep"] = _keep(c, g)
    else:
        t["X"] = _normal(g, rows, _padded(c["K"]), dtype=dt)[:, :c["K"]]
        t["W"] = _normal(g, c["O"], _padded(c["K"]), dtype=dt, std=c["K"] ** -0.5)[:, :c["K"]]
        t["bias"] = _normal(g, c["O"], dtype=dt) if c["bias"] else None
        t["gate"] = None if c["gate"] is None else _normal(
            g, *((c["F"], c["O"]) if c["gate"] == "frame" else (c["O"],)))
        t["R"] = _normal(g, rows, c["O"], dtype=DTYPES[c["out"]]) if c["residual"] else None
    return t


def _padded(n):
    """Rows of matrices start on 16-byte boundaries."""
    return (n + 7) // 8 * 8


def prepare(case, seed):
    c = dict(case)
    s = {"case": c, **_inputs(c, seed)}
    act = _active(c)
    s["frames"] = act
    s["active"] = torch.tensor(act + [0] * (c["F"] - c["A"]), dtype=torch.int32, device=DEV)
    n = _tokens(c)
    s["counts"] = torch.tensor([c["A"], c["A"] * n], dtype=torch.int32, device=DEV)
    s["rows"] = (torch.tensor(act, device=DEV)[:, None] * n + torch.arange(n, device=DEV)).flatten()
    if c["kind"] == "rope":
        # (cos, sin) of every pair at every position of an axis
        s["tables"] = [None if dim == 0 else _table(pos, dim).to(torch.float32)
                       for pos, dim in zip(_positions(c), _dims(c))]
        s["Yq"], s["Yk"] = (None if x is None else torch.zeros(x.shape, dtype=x.dtype, device=DEV)
                            for x in (s["Q"], s["K"]))
    elif c["kind"] == "cross":
        r = _ranges(c)
        s["ranges"] = r
        s["kv_range"] = None if r is None else torch.tensor(r, dtype=torch.int32, device=DEV)
        s["O"] = torch.zeros_like(s["Q"])
        s["lse"] = torch.zeros(c["H"], c["F"] * n, device=DEV) if c["lse"] else None
        s["status"] = torch.zeros(1, dtype=torch.int32, device=DEV)
    else:
        s["Y"] = torch.zeros(c["F"] * n, c["O"], dtype=DTYPES[c["out"]], device=DEV)
        s["status"] = torch.zeros(1, dtype=torch.int32, device=DEV)
    return s


def _table(pos, dim):
    freq = 10000.0 ** (-torch.arange(0, dim, 2, dtype=torch.float64, device=pos.device) / dim)
    a = pos[:, None] * freq
    return torch.stack([a.cos(), a.sin()], dim=-1)


# ------------------------------------------------------------------------------ one pass
def run(state):
    kind = state["case"]["kind"]
    if own:
        return {"rope": _own_rope, "cross": _own_cross, "linear": _own_linear}[kind](state)
    return {"rope": _plain_rope, "cross": _plain_cross, "linear": _plain_linear}[kind](state)


def _own_rope(s):
    import paper_2606_06309_gb300 as rf
    c = s["case"]
    rf.rf_rope(s["Yq"], s["Q"], s["Yk"], s["K"], c["F"], c["gh"], c["gw"], _dims(c), s["tables"],
               pairing=c["pairing"], inverse=c["inverse"], active=s["active"], counts=s["counts"])
    return [s["Yq"]] if s["Yk"] is None else [s["Yq"], s["Yk"]]


def _own_cross(s):
    import paper_2606_06309_gb300 as rf
    c = s["case"]
    rf.rf_cross_attn(s["O"], s["lse"], s["Q"], s["K"], s["V"], c["F"], c["N"], c["d"] ** -0.5,
                     kv_range=s["kv_range"], key_mask=s["keep"], active=s["active"],
                     counts=s["counts"], status=s["status"])
    return [s["O"]] if s["lse"] is None else [s["O"], s["lse"]]


def _own_linear(s):
    import paper_2606_06309_gb300 as rf
    c = s["case"]
    rf.rf_linear(s["Y"], s["X"], s["W"], c["F"], c["N"], bias=s["bias"], act=c["act"],
                 gate=s["gate"], residual=s["R"], active=s["active"], counts=s["counts"],
                 status=s["status"])
    return [s["Y"]]


def _plain_rope(s):
    c = s["case"]
    F, gh, gw = c["F"], c["gh"], c["gw"]
    grids = ((F, 1, 1), (1, gh, 1), (1, 1, gw))
    cs = torch.cat([t.view(*grids[i], -1, 2).expand(F, gh, gw, -1, 2)
                    for i, t in enumerate(s["tables"]) if t is not None], dim=3)
    cs = cs.reshape(F * gh * gw, 1, -1, 2)[s["rows"]]
    cos, sin = cs[..., 0], cs[..., 1]
    if c["inverse"]:
        sin = -sin
    R = sum(_dims(c))
    out = []
    for X, Y in ((s["Q"], s["Yq"]), (s["K"], s["Yk"])):
        if X is None:
            continue
        x = X[s["rows"]].float()
        y = x.clone()
        if c["pairing"] == "interleaved":
            a, b = x[..., 0:R:2], x[..., 1:R:2]
            y[..., 0:R:2], y[..., 1:R:2] = a * cos - b * sin, a * sin + b * cos
        else:
            a, b = x[..., :R // 2], x[..., R // 2:R]
            y[..., :R // 2], y[..., R // 2:R] = a * cos - b * sin, a * sin + b * cos
        Y[s["rows"]] = y.to(Y.dtype)
        out.append(Y)
    return out


def _attend(q, k, v, keep, scale):
    """q [n, H, d], k, v [L, Hk, d], keep [L] or None -> O [n, H, d], lse [H, n], 32 bits."""
    n, H, d = q.shape
    L, Hk = k.shape[0], k.shape[1]
    if L == 0:
        return (torch.zeros(n, H, d, device=q.device),
                torch.full((H, n), -math.inf, device=q.device))
    qg = q.float().view(n, Hk, H // Hk, d).permute(1, 2, 0, 3).reshape(Hk, -1, d)
    s = torch.matmul(qg, k.float().permute(1, 2, 0)) * scale
    if keep is not None:
        s = s.masked_fill(keep == 0, -math.inf)
    m = s.amax(dim=-1, keepdim=True)
    m = torch.where(m == -math.inf, torch.zeros_like(m), m)
    p = torch.exp(s - m)
    l = p.sum(dim=-1, keepdim=True)
    vf = v.float().permute(1, 0, 2)
    if keep is not None:
        vf = vf * keep[:, None].float()
    o = torch.matmul(p, vf) / torch.where(l == 0, torch.ones_like(l), l)
    o = o.view(Hk, H // Hk, n, d).permute(2, 0, 1, 3).reshape(n, H, d)
    return o, (l.log() + m).view(H, n)


def _plain_cross(s):
    c = s["case"]
    n, scale, O, lse = c["N"], c["d"] ** -0.5, s["O"], s["lse"]
    if s["ranges"] is None:
        parts = [(s["rows"], 0, c["L"])]
    else:
        parts = [(slice(f * n, f * n + n), *s["ranges"][f]) for f in s["frames"]]
    for rows, b, e in parts:
        keep = None if s["keep"] is None else s["keep"][b:e]
        o, l = _attend(s["Q"][rows], s["K"][b:e], s["V"][b:e], keep, scale)
        O[rows] = o.to(O.dtype)
        if lse is not None:
            lse[:, rows] = l
    return [O] if lse is None else [O, lse]


def _act(y, act):
    if act == "gelu":
        return 0.5 * y * (1.0 + torch.erf(y * math.sqrt(0.5)))
    if act == "gelu_tanh":
        return 0.5 * y * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (y + 0.044715 * y * y * y)))
    if act == "silu":
        return y / (1.0 + torch.exp(-y))
    return y


def _plain_linear(s):
    c = s["case"]
    n, A, rows, Y = c["N"], c["A"], s["rows"], s["Y"]
    y = torch.matmul(s["X"][rows].float(), s["W"].float().t())
    if s["bias"] is not None:
        y = y + s["bias"].float()
    y = _act(y, c["act"])
    if s["gate"] is not None:
        g = s["gate"]
        y = y * g if g.dim() == 1 else (y.view(A, n, -1) * g[s["frames"]][:, None]).flatten(0, 1)
    if s["R"] is not None:
        y = y + s["R"][rows].float()
    Y[rows] = y.to(Y.dtype)
    return [Y]


# ------------------------------------------------------------------------------ the work
def work(case):
    c = case
    rows, es = c["A"] * _tokens(c), SIZE[c["dtype"]]
    if c["kind"] == "rope":
        heads = c["H"] + c["Hk"]
        return {"bytes": 2 * rows * heads * c["d"] * es, "flops": 3 * rows * heads * sum(_dims(c))}
    if c["kind"] == "cross":
        r = _ranges(c)
        if r is None:
            pairs, keys = rows * c["L"], c["L"]
        else:
            act = [r[f] for f in _active(c)]
            pairs = c["N"] * sum(max(0, e - b) for b, e in act)
            keys, at = 0, 0  # rows of the union of the (ascending) ranges
            for b, e in act:
                keys += max(0, e - max(at, b))
                at = max(at, e)
        if c["kept"] is not None:
            pairs, keys = pairs * c["kept"] / c["L"], keys * c["kept"] / c["L"]
        b = es * c["d"] * (2 * rows * c["H"] + 2 * keys * c["Hk"])
        if c["lse"]:
            b += 4 * rows * c["H"]
        return {"bytes": int(b), "flops": int(4 * pairs * c["H"] * c["d"])}
    K, O, eo = c["K"], c["O"], SIZE[c["out"]]
    b = es * (rows * K + O * K) + eo * rows * O * (2 if c["residual"] else 1)
    if c["bias"]:
        b += es * O
    if c["gate"] is not None:
        b += 4 * O * (c["A"] if c["gate"] == "frame" else 1)
    return {"bytes": b, "flops": 2 * rows * K * O}


# ------------------------------------------------------------------------------ 64 bits
def exact(case, seed):
    c = dict(case)
    if work(c)["flops"] > EXACT_FLOPS:
        return None
    t = _inputs(c, seed)
    n = _tokens(c)
    if c["kind"] == "rope":
        return _exact_rope(c, t, n)
    if c["kind"] == "cross":
        return _exact_cross(c, t, n)
    Y = torch.zeros(c["F"] * n, c["O"], dtype=torch.float64, device=DEV)
    W = t["W"].double()
    for f in _active(c):
        at = slice(f * n, f * n + n)
        z = t["X"][at].double() @ W.T
        if t["bias"] is not None:
            z += t["bias"].double()
        if c["act"] == "gelu":  # x Phi(x)
            z = z * torch.special.ndtr(z)
        elif c["act"] == "gelu_tanh":
            z = z * torch.sigmoid(2.0 * math.sqrt(2.0 / math.pi) * (z + 0.044715 * z ** 3))
        elif c["act"] == "silu":
            z = z * torch.sigmoid(z)
        if t["gate"] is not None:
            z = z * (t["gate"][f] if c["gate"] == "frame" else t["gate"]).double()
        if t["R"] is not None:
            z = z + t["R"][at].double()
        Y[at] = z
    return [Y]


def _exact_rope(c, t, n):
    """Each pair as a complex number times e^(i angle)."""
    sign = -1.0 if c["inverse"] else 1.0
    pt, ph, pw = _positions(c)
    bands = [10000.0 ** (-torch.arange(0, dim, 2, dtype=torch.float64, device=DEV) / max(dim, 1))
             for dim in _dims(c)]
    half, out = sum(_dims(c)) // 2, []
    for X in (t["Q"], t["K"]):
        if X is None:
            continue
        Y = torch.zeros(X.shape, dtype=torch.float64, device=DEV)
        for f in _active(c):
            a = torch.cat([(pt[f] * bands[0]).expand(c["gh"], c["gw"], -1),
                           (ph[:, None, None] * bands[1]).expand(-1, c["gw"], -1),
                           (pw[None, :, None] * bands[2]).expand(c["gh"], -1, -1)], dim=-1)
            turn = torch.polar(torch.ones_like(a), sign * a).reshape(n, 1, half)
            at = slice(f * n, f * n + n)
            x = X[at].double()
            if c["pairing"] == "interleaved":
                z = torch.view_as_complex(x[..., :2 * half].reshape(n, -1, half, 2).contiguous())
                y = torch.view_as_real(z * turn).reshape(n, -1, 2 * half)
            else:
                z = torch.complex(x[..., :half].contiguous(), x[..., half:2 * half].contiguous())
                z = z * turn
                y = torch.cat([z.real, z.imag], dim=-1)
            Y[at] = torch.cat([y, x[..., 2 * half:]], dim=-1)
        out.append(Y)
    return out


def _exact_cross(c, t, n):
    H, Hk, d = c["H"], c["Hk"], c["d"]
    O = torch.zeros(c["F"] * n, H, d, dtype=torch.float64, device=DEV)
    lse = torch.zeros(H, c["F"] * n, dtype=torch.float64, device=DEV)
    ranges = _ranges(c)
    for f in _active(c):
        b, e = (0, c["L"]) if ranges is None else ranges[f]
        keys = torch.arange(b, max(b, e), device=DEV)
        if t["keep"] is not None:
            keys = keys[t["keep"][keys] != 0]
        at = slice(f * n, f * n + n)
        if len(keys) == 0:
            lse[:, at] = -math.inf
            continue
        for h in range(H):
            k, v = t["K"][keys, h * Hk // H].double(), t["V"][keys, h * Hk // H].double()
            z = (t["Q"][at, h].double() @ k.T) / math.sqrt(d)
            lse[h, at] = torch.logsumexp(z, dim=-1)
            O[at, h] = torch.softmax(z, dim=-1) @ v
    return [O, lse] if c["lse"] else [O]
