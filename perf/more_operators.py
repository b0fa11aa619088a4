"""Timing cases of what stands around the mixer in a block: a gated recurrence of channels (one state a channel instead of a
matrix a head), the norm of queries and keys with the rotation in the same pass, and the gated feed-forward product.

Sizes are those of ``paper_2405_18428_amd/inputs.py`` and the tests (384 and 1152 channels a token, grids of 16 to 128 tokens a
side, 16 heads of 128) and generic ones (2048 channels, four times as many inside the feed-forward block).  Where ``own`` is
false ``run`` takes the operators in their plain form, elementary torch operations in 32 bits (sums of gates, angles and sums over
all rows in 64), where it is true the library's entry points.
"""
import math

import torch

own = False

BHTD, BTHD = 0, 1
ROW_FWD, ROW_REV, COL_FWD, COL_REV = 0, 1, 2, 3
ADJACENT, HALVES = 0, 1
LOG, PRE = 0, 1                      # a gate's logarithm, or its pre-activation
SILU, GELU, GELU_TANH = 0, 1, 2
EPS = 1e-6
BASE = 10000.0


def listed():
    return [
        # one conversation being answered: the next token of one sequence, all latency
        {"name": "recur_step_one", "op": "step", "B": 1, "D": 2048, "gate": PRE, "tau": 16.0, "rest": True, "dtype": "bf16"},
        # a batch of prompts of their own lengths, padded to the longest, each continued from its conversation's state
        {"name": "recur_prompts", "op": "fwd", "B": 8, "gh": 1, "gw": 2047, "D": 2048, "gate": PRE, "tau": 16.0, "rest": True,
         "dtype": "bf16", "scan": ROW_FWD, "ragged": True, "state": True},
        # one long document: a single sequence, many tokens
        {"name": "recur_long", "op": "fwd", "B": 1, "gh": 1, "gw": 65536, "D": 2048, "gate": PRE, "tau": 1.0, "rest": False,
         "dtype": "bf16", "scan": ROW_FWD, "ragged": False, "state": False},
        # a training step over text
        {"name": "recur_train", "op": "train", "B": 4, "gh": 1, "gw": 4096, "D": 2048, "gate": PRE, "tau": 16.0, "rest": True,
         "dtype": "bf16", "scan": ROW_FWD, "ragged": False, "state": False},
        # the same in 32 bits for small images, in a block whose scan runs up the columns, gates given as logarithms
        {"name": "recur_train_grid_f32", "op": "train", "B": 4, "gh": 32, "gw": 32, "D": 384, "gate": LOG, "tau": 1.0, "rest": False,
         "dtype": "f32", "scan": COL_REV, "ragged": False, "state": True},
        # queries and keys of a serving batch's next tokens, at positions that the caller holds, four queries a key head
        {"name": "qk_step", "op": "qk", "B": 64, "H": 16, "Hk": 4, "frames": 1, "gh": 1, "gw": 1, "sections": "128", "d": 128,
         "dtype": "bf16", "layout": BTHD, "pairing": HALVES, "given": True, "packed": True, "affine": True, "train": False},
        # a training step's queries and keys, slices of one projection's rows, both directions
        {"name": "qk_train", "op": "qk", "B": 4, "H": 16, "Hk": 16, "frames": 1, "gh": 1, "gw": 4095, "sections": "128", "d": 128,
         "dtype": "bf16", "layout": BTHD, "pairing": HALVES, "given": False, "packed": True, "affine": True, "train": True},
        # feed-forward block of one next token: every weight is read for a single row
        {"name": "glu_step", "op": "glu", "M": 1, "K": 2048, "F": 8192, "act": SILU, "dtype": "bf16", "train": False},
        # the next tokens of a serving batch
        {"name": "glu_batch", "op": "glu", "M": 33, "K": 2048, "F": 8192, "act": SILU, "dtype": "bf16", "train": False},
        # the tokens of a 1024 px image
        {"name": "glu_image", "op": "glu", "M": 4096, "K": 1152, "F": 4608, "act": GELU_TANH, "dtype": "bf16", "train": False},
        # a training step of 8192 tokens
        {"name": "glu_train", "op": "glu", "M": 8192, "K": 2048, "F": 8192, "act": SILU, "dtype": "bf16", "train": True},
        # a training step of a small model in 32 bits, odd numbers of rows and channels
        {"name": "glu_train_odd_f32", "op": "glu", "M": 1021, "K": 381, "F": 1531, "act": GELU, "dtype": "f32", "train": True},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    """A case of the same ranges, at most as large as the largest listed one of its kind."""
    op = rng.choice(["step", "fwd", "fwd", "train", "train", "qk", "qk", "qk", "glu", "glu", "glu", "glu"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if op in ("step", "fwd", "train"):
        D = rng.choice([384, 1152, 2048, _log(rng, 1, 4096)])
        c = {"op": op, "D": D, "gate": rng.choice([LOG, PRE, PRE]), "tau": rng.choice([1.0, 16.0]), "rest": rng.random() < 0.5, "dtype": dtype}
        if op == "step":
            return {**c, "B": _log(rng, 1, 1024)}
        rows = {"fwd": 100000000, "train": 30000000}[op] // D // (2 if dtype == "f32" else 1)   # over all batches
        T = _log(rng, 1, min(65536, rows))
        B = _log(rng, 1, max(1, min(64, rows // T)))
        gh = rng.choice([1, 1, max(1, int(T ** 0.5))])
        return {**c, "B": B, "gh": gh, "gw": max(1, T // gh), "scan": rng.randrange(2 if gh == 1 else 4),
                "ragged": gh == 1 and rng.random() < 0.4, "state": rng.random() < 0.5}
    if op == "qk":
        axes = rng.choice([0, 1, 1, 2, 3])
        sections = [2 * rng.randint(1, 20) for _ in range(axes)]
        if axes == 1:
            sections = [rng.choice([32, 64, 128, 2 * rng.randint(1, 64)])]
        d = sum(sections) + rng.choice([0, 0, 8, 2 * rng.randint(0, 16)])
        d = d if axes else rng.choice([32, 36, 64, 128, rng.randint(1, 256)])
        frames, gh, gw = (1, 1, _log(rng, 1, 8192)) if axes <= 1 else (_log(rng, 1, 12) if axes == 3 else 1, _log(rng, 2, 90), _log(rng, 2, 90))
        Hk = rng.choice([1, 4, 6, 16])
        H = Hk * rng.choice([1, 1, 2, 4])
        B = _log(rng, 1, max(1, min(64, 30000000 // (frames * gh * gw * (H + Hk) * d))))
        return {"op": op, "B": B, "H": H, "Hk": Hk, "frames": frames, "gh": gh, "gw": gw, "sections": ",".join(map(str, sections)), "d": d,
                "dtype": dtype, "layout": rng.choice([BHTD, BTHD]), "pairing": rng.choice([ADJACENT, HALVES]), "given": axes > 0 and rng.random() < 0.4,
                "packed": rng.random() < 0.6, "affine": rng.random() < 0.8, "train": rng.random() < 0.5}
    K, F = rng.choice([(384, 1536), (1152, 4608), (2048, 8192), (_log(rng, 32, 2048), _log(rng, 32, 8192))])
    M = _log(rng, 1, 8192 if dtype == "bf16" else max(1, min(8192, 10 ** 10 // (K * F))))
    return {"op": "glu", "M": M, "K": K, "F": F, "act": rng.choice([SILU, GELU, GELU_TANH]), "dtype": dtype, "train": rng.random() < 0.5}


def _dt(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _sections(c):
    return tuple(int(n) for n in c["sections"].split(",") if n)


def _inputs(case, seed):
    """The tensors of a case, from its sizes and the seed alone, and the buffers that a program keeps."""
    c, g = case, torch.Generator(device="cuda").manual_seed(seed)
    dt = _dt(c["dtype"])
    randn = lambda *n: torch.randn(*n, generator=g, device="cuda")  # noqa: E731
    s = {"case": c}
    if c["op"] in ("step", "fwd", "train"):
        B, D = c["B"], c["D"]
        T = 1 if c["op"] == "step" else c["gh"] * c["gw"]
        lead = (B,) if c["op"] == "step" else (B, T)
        s["x"] = randn(*lead, D).to(dt)
        z = randn(*lead, D) + 2.0
        s["g"] = z.to(dt) if c["gate"] == PRE else torch.nn.functional.logsigmoid(z) / 16.0
        if c["op"] == "step" or c["state"]:
            s["s0"] = 2.0 * randn(B, D)
        if c["op"] == "step":
            s["s1"] = torch.empty_like(s["s0"])
            return s
        if c["ragged"]:
            n = torch.randint(0, T + 1, (B,), generator=g, device="cuda", dtype=torch.int32)
            n[B // 2] = T
            s["lens"] = n
        s["out"] = torch.zeros(B, T, D, dtype=dt, device="cuda")     # rows behind a prompt's end keep what they hold
        if c["op"] == "train":
            s["do"] = randn(B, T, D).to(dt)
            if c["state"]:
                s["df"] = randn(B, D)
    elif c["op"] == "qk":
        B, T, H, Hk, d = c["B"], c["frames"] * c["gh"] * c["gw"], c["H"], c["Hk"], c["d"]
        turn = lambda x: x.transpose(1, 2) if c["layout"] == BHTD else x  # noqa: E731
        if c["packed"]:              # rows of one projection: queries, keys, values
            rows = (1.5 * randn(B, T, (H + 2 * Hk) * d)).to(dt)
            s["q"], s["k"] = turn(rows[..., :H * d].view(B, T, H, d)), turn(rows[..., H * d:(H + Hk) * d].view(B, T, Hk, d))
        else:
            s["q"], s["k"] = ((1.5 * randn(*((B, n, T) if c["layout"] == BHTD else (B, T, n)), d)).to(dt) for n in (H, Hk))
        s["qw"], s["kw"] = (1.0 + 0.1 * randn(d), 1.0 + 0.1 * randn(d)) if c["affine"] else (None, None)
        if c["given"]:
            s["pos"] = torch.randint(0, 32768, (B, T, len(_sections(c))), generator=g, device="cuda", dtype=torch.int32)
        if c["train"]:
            s["dq"], s["dk"] = (randn(*s[n].shape).to(dt) for n in ("q", "k"))
    else:
        M, K, F = c["M"], c["K"], c["F"]
        s["x"] = randn(M, K).to(dt)
        s["wg"], s["wu"] = (randn(F, K) * K ** -0.5).to(dt), (randn(F, K) * K ** -0.5).to(dt)
        if c["train"]:
            s["do"] = randn(M, F).to(dt)
    return s


def prepare(case, seed):
    """Inputs, and with the library the workspaces that its calls take."""
    s = _inputs(case, seed)
    if own:
        _workspaces(s)
    return s


def _workspaces(s):
    import paper_2405_18428_amd as gla
    c = s["case"]
    code = gla.DT_BF16 if c["dtype"] == "bf16" else gla.DT_F32
    room = lambda n: torch.empty(max(n, 16), dtype=torch.uint8, device="cuda")  # noqa: E731
    if c["op"] in ("fwd", "train"):
        sizes = (c["B"], c["gh"] * c["gw"], c["D"])
        s["ws"] = room(gla.gla_recur_fwd_workspace_bytes(*sizes))
        if c["op"] == "train":
            s["ws_back"] = room(gla.gla_recur_bwd_workspace_bytes(*sizes))
    elif c["op"] == "qk" and c["train"]:
        s["ws"] = room(gla.gla_qk_norm_bwd_workspace_bytes(c["B"], c["H"], c["Hk"], c["frames"] * c["gh"] * c["gw"], c["d"]))
    elif c["op"] == "glu":
        sizes = (c["M"], c["K"], c["F"], code)
        s["ws"] = room(gla.gla_glu_fwd_workspace_bytes(*sizes))
        if c["train"]:               # what the forward pass hands to the backward pass, and the latter's room
            s["pre"] = torch.empty(2, c["M"], c["F"], device="cuda")
            s["ws_back"] = room(gla.gla_glu_bwd_workspace_bytes(*sizes))


def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_own(s):
    import paper_2405_18428_amd as gla
    c, dt = s["case"], _dt(s["case"]["dtype"])
    if c["op"] in ("step", "fwd", "train"):
        how = {"gate_kind": c["gate"], "tau": c["tau"], "complement": c["rest"]}
        if c["op"] == "step":
            return gla.gla_recur_step(s["x"], s["g"], s["s0"], out_dtype=dt, state_out=s["s1"], **how)
        how.update(scan_dir=c["scan"], seq_lens=s.get("lens"), initial_state=s.get("s0"))
        out, fin = gla.gla_recur_fwd(s["x"], s["g"], c["gh"], c["gw"], out=s["out"], workspace=s["ws"], **how)
        if c["op"] == "fwd":
            return out, fin
        dx, dg, ds = gla.gla_recur_bwd(s["x"], s["g"], s["do"], c["gh"], c["gw"], d_final_state=s.get("df"), grad_dtype=dt,
                                       want_d_initial_state=c["state"], workspace=s["ws_back"], **how)
        return (out, fin, dx, dg) + ((ds,) if c["state"] else ())
    if c["op"] == "qk":
        how = {"sections": _sections(c), "eps": EPS, "positions": s.get("pos"), "base": BASE, "pairing": c["pairing"], "layout": c["layout"],
               "grid_h": c["gh"], "grid_w": c["gw"]}
        y = gla.gla_qk_norm_fwd(s["q"], s["k"], s["qw"], s["kw"], **how)
        if not c["train"]:
            return y
        back = gla.gla_qk_norm_bwd(s["q"], s["k"], s["dq"], s["dk"], s["qw"], s["kw"], grad_dtype=dt, workspace=s["ws"], **how)
        return (*y, *(t for t in back if t is not None))
    if not c["train"]:
        return gla.gla_glu_fwd(s["x"], s["wg"], s["wu"], c["act"], workspace=s["ws"])
    y = gla.gla_glu_fwd(s["x"], s["wg"], s["wu"], c["act"], pre=s["pre"], workspace=s["ws"])
    return (y, *gla.gla_glu_bwd(s["x"], s["wg"], s["wu"], s["do"], c["act"], pre=s["pre"], workspace=s["ws_back"]))


# --- plain forms -----------------------------------------------------------------------------------------------------

def _run_plain(s):
    return {"step": _plain_step, "fwd": _plain_recur, "train": _plain_recur, "qk": _plain_qk, "glu": _plain_glu}[s["case"]["op"]](s)


def _log_gate(s):
    """The gates' logarithms in 64 bits."""
    c = s["case"]
    if c["gate"] == LOG:
        return s["g"].double()
    z = s["g"].double()
    return (torch.minimum(z, torch.zeros_like(z)) - torch.log1p(torch.exp(-z.abs()))) / c["tau"]


def _plain_step(s):
    lg, x = _log_gate(s), s["x"].float()
    u = x * (-torch.expm1(lg)).float() if s["case"]["rest"] else x
    h = torch.exp(lg).float() * s["s0"] + u
    return h.to(s["x"].dtype), h


def _order(c):
    """Scan step -> token, for the four scan orders of the grid."""
    n = torch.arange(c["gh"] * c["gw"], device="cuda")
    if c["scan"] >= COL_FWD:
        n = n.view(c["gh"], c["gw"]).t().reshape(-1)
    return n.flip(0) if c["scan"] & 1 else n


def _to_scan(x, c):
    return x if c["scan"] == ROW_FWD else x.index_select(1, _order(c))


def _from_scan(x, c, dt):
    if c["scan"] != ROW_FWD:
        y = torch.empty_like(x)
        y[:, _order(c)] = x
        x = y
    return x.to(dt).contiguous()


def _recur(lg, u, s0):
    """h_t = exp(lg_t) h_{t-1} + u_t over dimension 1 by doubling: after the pass of width w every step has the sum over the 2 w
    steps up to it.  lg in 64 bits, u and h in 32."""
    h, w = u.clone(), 1
    if s0 is not None:
        h[:, 0] += torch.exp(lg[:, 0]).float() * s0
    lg = lg.clone()
    while w < h.shape[1]:
        more = torch.exp(lg[:, w:]).float() * h[:, :-w]
        h[:, w:] += more
        more = lg[:, :-w].clone()
        lg[:, w:] += more
        w *= 2
    return h


def _plain_recur(s):
    c, dt = s["case"], s["x"].dtype
    lg, x = _to_scan(_log_gate(s), c), _to_scan(s["x"].float(), c)
    T, inside = x.shape[1], None
    if "lens" in s:                  # steps behind the end add nothing and do not decay
        inside = torch.arange(T, device="cuda")[None] < s["lens"][:, None]
        inside = (inside if c["scan"] == ROW_FWD else inside.flip(1))[..., None]
        x, lg = torch.where(inside, x, torch.zeros_like(x)), torch.where(inside, lg, torch.zeros_like(lg))
    rest = (-torch.expm1(lg)).float() if c["rest"] else None
    h = _recur(lg, x * rest if c["rest"] else x, s.get("s0"))
    fin = h[:, -1].clone()
    mask = lambda t: t if inside is None else torch.where(inside, t, torch.zeros_like(t))  # noqa: E731
    out = _from_scan(mask(h), c, dt)
    if c["op"] == "fwd":
        return out, fin
    # the adjoint of h is the same recurrence from the end, where step t meets the gate of step t + 1
    do = mask(_to_scan(s["do"].float(), c))
    if "df" in s:
        do[:, -1] += s["df"]
    back = torch.cat([torch.zeros_like(lg[:, :1]), lg.flip(1)[:, :-1]], 1)
    G = _recur(back, do.flip(1), None).flip(1)
    first = s["s0"][:, None] if "s0" in s else torch.zeros_like(h[:, :1])
    before = torch.cat([first, h[:, :-1]], 1)
    a = torch.exp(lg).float()
    dlg = a * ((before - x) if c["rest"] else before) * G
    if c["gate"] == PRE:
        dlg = dlg * (1.0 / (1.0 + torch.exp(_to_scan(s["g"].float(), c)))) * (1.0 / c["tau"])
    res = [out, fin, _from_scan(mask(G * rest if c["rest"] else G), c, dt), _from_scan(mask(dlg), c, dt)]
    return tuple(res + ([a[:, 0] * G[:, 0]] if c["state"] else []))


def _angles(c, s):
    """[B or 1, T, pairs] angles in 64 bits and the two channels of each pair."""
    sections = _sections(c)
    if c["given"]:
        pos = s["pos"].double()
    else:
        n = torch.arange(c["frames"] * c["gh"] * c["gw"], device="cuda")
        cell = n % (c["gh"] * c["gw"])
        axes = [n] if len(sections) == 1 else [cell // c["gw"], cell % c["gw"]]
        if len(sections) == 3:
            axes = [n // (c["gh"] * c["gw"])] + axes
        pos = torch.stack(axes, -1)[None].double()
    ang, first, second, at = [], [], [], 0
    for a, w in enumerate(sections):
        i = torch.arange(w // 2, device="cuda")
        ang.append(pos[..., a:a + 1] * torch.pow(torch.tensor(BASE, dtype=torch.float64, device="cuda"), -2.0 * i.double() / w))
        first.append(at + (2 * i if c["pairing"] == ADJACENT else i))
        second.append(at + (2 * i + 1 if c["pairing"] == ADJACENT else i + w // 2))
        at += w
    return torch.cat(ang, -1), torch.cat(first), torch.cat(second)


def _plain_qk(s):
    c = s["case"]
    turned = len(_sections(c)) > 0
    if turned:
        ang, i0, i1 = _angles(c, s)
        ang = ang[:, None] if c["layout"] == BHTD else ang[:, :, None]
        cs, sn = torch.cos(ang).float(), torch.sin(ang).float()

    def turn(y, sign):
        if not turned:
            return y
        z, a, b = y.clone(), y[..., i0], y[..., i1]
        z[..., i0], z[..., i1] = a * cs - b * (sign * sn), b * cs + a * (sign * sn)
        return z

    ys, dxs, dws = [], [], []
    for x, w, do in ((s["q"], s["qw"], s.get("dq")), (s["k"], s["kw"], s.get("dk"))):
        dt, x = x.dtype, x.float()
        rstd = 1.0 / torch.sqrt((x * x).mean(-1, keepdim=True) + EPS)
        n = x * rstd
        ys.append(turn(n if w is None else n * w, 1.0).to(dt).contiguous())
        if do is not None:
            dy = turn(do.float(), -1.0)
            dn = dy if w is None else dy * w
            dxs.append((rstd * (dn - n * (dn * n).mean(-1, keepdim=True))).to(dt).contiguous())
            if w is not None:
                dws.append((dy * n).sum((0, 1, 2), dtype=torch.float64).float())
    return tuple(ys + dxs + dws)


def _act(kind, g):
    """The activation and its derivative."""
    if kind == SILU:
        sg = 1.0 / (1.0 + torch.exp(-g))
        return g * sg, sg * (1.0 + g * (1.0 - sg))
    if kind == GELU:
        phi = 0.5 * torch.erfc(-g * 0.5 ** 0.5)
        return g * phi, phi + g * torch.exp(-0.5 * g * g) * (2.0 * math.pi) ** -0.5
    k = (2.0 / math.pi) ** 0.5
    sg = 1.0 / (1.0 + torch.exp(-2.0 * k * (g + 0.044715 * g * g * g)))      # (1 + tanh) / 2
    return g * sg, sg + 2.0 * g * sg * (1.0 - sg) * k * (1.0 + 3.0 * 0.044715 * g * g)


def _plain_glu(s):
    c, dt = s["case"], s["x"].dtype
    x, wg, wu = s["x"].float(), s["wg"].float(), s["wu"].float()
    g, u = x @ wg.t(), x @ wu.t()
    act, slope = _act(c["act"], g)
    y = (act * u).to(dt)
    if not c["train"]:
        return y
    do = s["do"].float()
    dg, du = do * u * slope, do * act
    return y, (dg @ wg + du @ wu).to(dt), (dg.t() @ x).to(dt), (du.t() @ x).to(dt)


# --- work ------------------------------------------------------------------------------------------------------------

def work(case):
    c = case
    e = 2 if c["dtype"] == "bf16" else 4
    if c["op"] in ("step", "fwd", "train"):
        B, D, T = c["B"], c["D"], 1 if c["op"] == "step" else c["gh"] * c["gw"]
        rows = B * T
        if c.get("ragged"):          # lengths are uniform over 0 .. T and one is T
            rows = T + (B - 1) * T / 2
        n, eg = rows * D, 4 if c["gate"] == LOG else e
        moved = n * (2 * e + eg) + 4 * B * D * (2 if c["op"] == "step" or c["state"] else 1)
        done = n * 10
        if c["op"] == "train":
            moved += n * 3 * e + (8 * B * D if c["state"] else 0)
            done += n * 20
        return {"bytes": float(moved), "flops": float(done)}
    if c["op"] == "qk":
        rows = c["B"] * c["frames"] * c["gh"] * c["gw"]
        n = rows * (c["H"] + c["Hk"]) * c["d"]
        given = 4 * rows * len(_sections(c)) if c["given"] else 0
        moved, done = 2 * n * e + given + (8 * c["d"] if c["affine"] else 0), 8 * n
        if c["train"]:
            moved, done = moved + 2 * n * e + (8 * c["d"] if c["affine"] else 0), done + 20 * n
        return {"bytes": float(moved), "flops": float(done)}
    M, K, F = c["M"], c["K"], c["F"]
    moved, done = e * (M * K + 2 * F * K + M * F), 4.0 * M * K * F
    if c["train"]:
        moved, done = moved + e * (M * F + M * K + 2 * F * K), 3 * done
    return {"bytes": float(moved), "flops": float(done)}


# --- the definitions in 64 bits ----------------------------------------------------------------------------------------

def exact(case, seed):
    s = _inputs(case, seed)
    return {"step": _exact_recur, "fwd": _exact_recur, "train": _exact_recur, "qk": _exact_qk, "glu": _exact_glu}[case["op"]](s)


def _exact_recur(s):
    """The recurrence one step after the other, and the gradients by the chain rule from the last step to the first."""
    c = s["case"]
    one = c["op"] == "step"
    x, z = (s[n][:, None] if one else s[n] for n in ("x", "g"))
    B, T, D = x.shape
    lens = s["lens"].tolist() if "lens" in s else [T] * B
    token = torch.arange(T)
    if not one and c["scan"] in (COL_FWD, COL_REV):
        token = torch.cat([torch.arange(col, T, c["gw"]) for col in range(c["gw"])])
    if not one and c["scan"] in (ROW_REV, COL_REV):
        token = token.flip(0)
    here = [torch.tensor([1.0 if t < n else 0.0 for n in lens], dtype=torch.float64, device="cuda")[:, None] for t in token.tolist()] \
        if "lens" in s else [None] * T
    token = token.tolist()

    def at(t):
        v = z[:, t].double()
        lg = v if c["gate"] == LOG else -torch.nn.functional.softplus(-v) / c["tau"]
        return torch.exp(lg), -torch.expm1(lg)

    state = s["s0"].double() if "s0" in s else torch.zeros(B, D, dtype=torch.float64, device="cuda")
    out = torch.zeros(B, T, D, dtype=torch.float64, device="cuda")
    before = torch.zeros_like(out) if c["op"] == "train" else None
    for t, m in zip(token, here):
        a, b = at(t)
        if before is not None:
            before[:, t] = state
        new = a * state + (x[:, t].double() * b if c["rest"] else x[:, t].double())
        state = new if m is None else m * new + (1.0 - m) * state
        out[:, t] = new if m is None else m * new
    if one:
        return out[:, 0], state
    if c["op"] == "fwd":
        return out, state
    adj = s["df"].double() if "df" in s else torch.zeros_like(state)
    dx, dg = torch.zeros_like(out), torch.zeros_like(out)
    for t, m in zip(reversed(token), reversed(here)):
        a, b = at(t)
        G = adj + s["do"][:, t].double()
        dx[:, t] = G * b if c["rest"] else G
        dl = G * a * (before[:, t] - (x[:, t].double() if c["rest"] else 0.0))
        dg[:, t] = dl if c["gate"] == LOG else dl * torch.sigmoid(-z[:, t].double()) / c["tau"]
        if m is None:
            adj = a * G
        else:
            dx[:, t] *= m
            dg[:, t] *= m
            adj = m * (a * G) + (1.0 - m) * adj
    return (out, state, dx, dg) + ((adj,) if c["state"] else ())


def _exact_qk(s):
    """Rows over their root mean square, each pair as a complex number turned by its token's angle, gradients by differentiation."""
    c = s["case"]
    B, T, sections = c["B"], c["frames"] * c["gh"] * c["gw"], _sections(c)
    if c["given"]:
        pos = s["pos"].double()
    elif sections:
        t, r, w = torch.meshgrid(*(torch.arange(n, device="cuda", dtype=torch.float64) for n in (c["frames"], c["gh"], c["gw"])), indexing="ij")
        axes = {1: [(t * c["gh"] + r) * c["gw"] + w], 2: [r, w], 3: [t, r, w]}[len(sections)]
        pos = torch.stack([a.reshape(-1) for a in axes], -1).expand(B, T, len(sections))
    lie = (lambda x: x) if c["layout"] == BHTD else (lambda x: x.transpose(1, 2))
    ys, dxs, dws = [], [], []
    for name, weight, up in (("q", "qw", "dq"), ("k", "kw", "dk")):
        x = lie(s[name]).double().detach().requires_grad_(c["train"])
        w = s[weight].double().requires_grad_(c["train"]) if s[weight] is not None else None
        n = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS)
        n = n * w if w is not None else n
        parts, at = [], 0
        for a, width in enumerate(sections):
            part = n[..., at:at + width]
            v = (torch.complex(part[..., 0::2].contiguous(), part[..., 1::2].contiguous()) if c["pairing"] == ADJACENT
                 else torch.complex(part[..., :width // 2].contiguous(), part[..., width // 2:].contiguous()))
            turn = pos[:, None, :, a, None] / torch.tensor([BASE ** (2.0 * i / width) for i in range(width // 2)], dtype=torch.float64, device="cuda")
            v = v * torch.polar(torch.ones_like(turn), turn)
            parts.append(torch.stack([v.real, v.imag], -1).flatten(-2) if c["pairing"] == ADJACENT else torch.cat([v.real, v.imag], -1))
            at += width
        y = torch.cat(parts + [n[..., at:]], -1)
        ys.append(lie(y.detach()))
        if c["train"]:
            y.backward(lie(s[up]).double())
            dxs.append(lie(x.grad))
            if w is not None:
                dws.append(w.grad)
    return tuple(ys + dxs + dws)


def _exact_glu(s):
    """The block as a composition, its gradients by differentiation."""
    c, F = s["case"], torch.nn.functional
    x, wg, wu = (s[n].double().requires_grad_(c["train"]) for n in ("x", "wg", "wu"))
    g = F.linear(x, wg)
    a = F.silu(g) if c["act"] == SILU else F.gelu(g, approximate="none" if c["act"] == GELU else "tanh")
    y = a * F.linear(x, wu)
    if not c["train"]:
        return y
    return (y.detach(), *torch.autograd.grad(y, (x, wg, wu), s["do"].double()))
