"""Cases for measuring two operators: rotary positions with several axes, and differential attention.

Multi-axis rotary positions turn pairs of features of q and k by angles that come from several
coordinates of a token (time, height, width).  Differential attention is
``out = (softmax(Q1 K1^T s) - lambda softmax(Q2 K2^T s)) V`` with ``Q = [Q1 | Q2]``, ``K = [K1 | K2]``,
grouped KV heads, an optional causal flag and valid lengths; query rows stand at the end of the keys.

``own`` false: the operators in their plain form (elementary torch operations in 32 bits);
true: the framework's calls.  ``exact`` is the definition in 64 bits.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    return [
        # one new token in each of 64 running requests, text and image positions (three axes): latency
        dict(name="rotary_decode_64", op="rotary", B=64, H=32, H_kv=8, N=1, D=128, dtype="bf16", parts=1,
             sections="16,24,24", dims="", ladder="shared", layout="halves", train=False),
        # prompt of 32k tokens seen as a 32 x 32 x 32 tensor, one ladder of frequencies per axis
        dict(name="rotary_32k", op="rotary", B=1, H=32, H_kv=8, N=32768, D=128, dtype="bf16", parts=1,
             sections="22,21,21", dims="32,32,32", ladder="axis", layout="halves", train=False),
        # training step of a small fp32 model on images of ragged token counts, two sub-heads per head,
        # part of the features left without position: forward and gradients
        dict(name="rotary_train_f32", op="rotary", B=2, H=12, H_kv=12, N=1531, D=64, dtype="f32", parts=2,
             sections="6,7", dims="", ladder="axis", layout="pairs", train=True),
        # the smallest call of a bidirectional encoder: latency
        dict(name="diff_encoder_256", op="diff", B=1, H=8, H_kv=8, Nq=256, Nk=256, D=128, dtype="bf16", causal=False,
             lens="full", train=False),
        # encoder batch padded to the longest text, head dim 64
        dict(name="diff_encoder_ragged", op="diff", B=4, H=12, H_kv=12, Nq=1531, Nk=1531, D=64, dtype="bf16",
             causal=False, lens="both", train=False),
        # ordinary prompt at Llama-8B head shapes
        dict(name="diff_prompt_4k", op="diff", B=1, H=32, H_kv=8, Nq=4096, Nk=4096, D=128, dtype="bf16", causal=True,
             lens="full", train=False),
        # the largest prompt: a quarter of those heads (one of four ranks) over 16k tokens
        dict(name="diff_prompt_16k", op="diff", B=1, H=8, H_kv=2, Nq=16384, Nk=16384, D=128, dtype="bf16", causal=True,
             lens="full", train=False),
        # one new token per request against caches of different fill
        dict(name="diff_decode_batch", op="diff", B=32, H=32, H_kv=8, Nq=1, Nk=4099, D=128, dtype="bf16", causal=True,
             lens="keys", train=False),
        # one new token of one request against a 128k cache
        dict(name="diff_decode_128k", op="diff", B=1, H=32, H_kv=8, Nq=1, Nk=131072, D=128, dtype="bf16", causal=True,
             lens="full", train=False),
        # training step: forward and gradients of q, k, v and lambda
        dict(name="diff_train_2k", op="diff", B=2, H=8, H_kv=8, Nq=2048, Nk=2048, D=128, dtype="bf16", causal=True,
             lens="full", train=True),
        dict(name="diff_train_8k", op="diff", B=1, H=8, H_kv=2, Nq=8192, Nk=8192, D=128, dtype="bf16", causal=True,
             lens="full", train=True),
        # the same in fp32 at an odd length, padded batch
        dict(name="diff_train_f32", op="diff", B=2, H=4, H_kv=2, Nq=777, Nk=777, D=64, dtype="f32", causal=True,
             lens="both", train=True),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    H_kv = rng.choice([1, 2, 4, 8])
    H = H_kv * rng.choice([1, 2, 4])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    D = rng.choice([64, 128])
    if rng.random() < 0.35:
        parts = rng.choice([1, 2])
        half = D // parts // 2
        axes = rng.choice([1, 2, 3])
        cut = sorted(rng.sample(range(1, half), axes))
        sections = [b - a for a, b in zip([0] + cut[:-1], cut)]
        dims = ""
        N = _log(rng, 1, 32768)
        if rng.random() < 0.4:
            shape = [_log(rng, 2, 32) for _ in sections]
            N, dims = math.prod(shape), ",".join(map(str, shape))
        return dict(op="rotary", B=rng.choice([1, 2, 3]), H=H, H_kv=H_kv, N=N, D=D, dtype=dtype, parts=parts,
                    sections=",".join(map(str, sections)), dims=dims, ladder=rng.choice(["shared", "axis"]),
                    layout=rng.choice(["halves", "pairs"]), train=rng.random() < 0.4)
    kind = rng.choice(["prompt", "prompt", "decode", "train", "train", "chunk"])
    B = rng.choice([1, 1, 2, 3])
    if kind == "decode":
        B, Nq, Nk = _log(rng, 1, 64), 1, _log(rng, 64, 32768)
    elif kind == "chunk":                      # a chunk of a prompt, or drafted tokens, behind a cache
        Nk = _log(rng, 256, 8192)
        Nq = _log(rng, 2, Nk)
    else:
        Nq = Nk = _log(rng, 16, 4096)
    causal = kind in ("decode", "chunk") or rng.random() < 0.7
    lens = rng.choice(["full", "keys"]) if kind in ("decode", "chunk") else rng.choice(["full", "full", "both"])
    case = dict(op="diff", B=B, H=H, H_kv=H_kv, Nq=Nq, Nk=Nk, D=D, dtype=dtype, causal=causal, lens=lens,
                train=kind == "train")
    while work(case)["flops"] > 5e11 or work(case)["bytes"] > 5e8:     # the largest listed case is the most
        if case["B"] > 1:
            case["B"] -= 1
        else:
            case["Nk"] = 3 * case["Nk"] // 4
            case["Nq"] = min(case["Nq"], case["Nk"]) if kind in ("decode", "chunk") else case["Nk"]
    return case


def _ints(text):
    return [int(x) for x in text.split(",") if x]


def _lens(case):
    """Valid keys and valid query rows per batch entry, as lists (None: all of them)."""
    if case["lens"] == "full":
        return None, None
    B, Nk, Nq = case["B"], case["Nk"], case["Nq"]
    keys = [Nk if i == 0 else Nq + (Nk - Nq) * ((37 * i + 11) % 64) // 63 for i in range(B)]
    if case["lens"] == "keys":
        return keys, None
    keys = [Nk if i == 0 else 1 + (Nk - 1) * ((37 * i + 11) % 64) // 63 for i in range(B)]
    return keys, list(keys)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dt = DTYPES[case["dtype"]]

    def normal(*shape):
        return torch.randn(*shape, device="cuda", generator=gen).to(dt)

    B, H, H_kv, D = case["B"], case["H"], case["H_kv"], case["D"]
    st = {"case": case}
    if case["op"] == "rotary":
        N = case["N"]
        st["q"], st["k"] = normal(B, H, N, D), normal(B, H_kv, N, D)
        st["sections"], st["dims"], st["positions"] = _ints(case["sections"]), None, None
        if case["dims"]:
            st["dims"] = _ints(case["dims"])
        else:
            st["positions"] = torch.randint(0, 131072, (len(st["sections"]), B, N), device="cuda", generator=gen,
                                            dtype=torch.int32)
        if case["train"]:
            st["dq"], st["dk"] = normal(B, H, N, D), normal(B, H_kv, N, D)
        return st
    Nq, Nk = case["Nq"], case["Nk"]
    st["q"], st["k"], st["v"] = normal(B, H, Nq, D), normal(B, H_kv, Nk, D), normal(B, H_kv, Nk, D)
    st["lam"] = 0.2 + 0.6 * torch.rand(H, device="cuda", generator=gen)
    keys, rows = _lens(case)
    st["kv_lens"] = None if keys is None else torch.tensor(keys, dtype=torch.int32, device="cuda")
    st["q_lens"] = None if rows is None else torch.tensor(rows, dtype=torch.int32, device="cuda")
    if case["train"]:
        st["dout"] = normal(B, H, Nq, D)
    return st


# ------------------------------------------------------------------ plain forms

def _angles(st, dtype=torch.float64):
    """Angle of every (batch entry, token, pair), in 64 bits: positions reach 10^5."""
    case, sec = st["case"], st["sections"]
    dev = st["q"].device
    half = sum(sec)
    axis = torch.repeat_interleave(torch.arange(len(sec), device=dev), torch.tensor(sec, device=dev))
    c = torch.arange(half, device=dev, dtype=dtype)
    if case["ladder"] == "axis":
        size = torch.tensor(sec, device=dev, dtype=dtype)
        start = torch.cumsum(size, 0) - size
        freq = 10000.0 ** (-(c - start[axis]) / size[axis])
    else:
        freq = 10000.0 ** (-c / half)
    if st["dims"] is not None:
        shape = torch.tensor(st["dims"], device=dev)
        stride = torch.flip(torch.cumprod(torch.flip(shape, [0]), 0), [0]) // shape
        n = torch.arange(case["N"], device=dev)
        pos = ((n[None, :] // stride[:, None]) % shape[:, None])[:, None, :].expand(-1, case["B"], -1)
    else:
        pos = st["positions"]
    return pos.to(dtype)[axis].permute(1, 2, 0) * freq                 # [B, N, half]


def _turn(x, cos, sin, case, half):
    B, heads, N, D = x.shape
    y = x.float().view(B, heads, N, case["parts"], D // case["parts"])
    r = y[..., :2 * half]
    if case["layout"] == "halves":
        x1, x2 = r[..., :half], r[..., half:]
        turned = torch.cat([x1 * cos - x2 * sin, x2 * cos + x1 * sin], -1)
    else:
        x1, x2 = r[..., 0::2], r[..., 1::2]
        turned = torch.stack([x1 * cos - x2 * sin, x2 * cos + x1 * sin], -1).flatten(-2)
    return torch.cat([turned, y[..., 2 * half:]], -1).reshape(B, heads, N, D).to(x.dtype)


def _plain_rotary(st):
    case, half = st["case"], sum(st["sections"])
    ang = _angles(st)[:, None, :, None, :]
    cos, sin = ang.cos().float(), ang.sin().float()
    out = [_turn(st["q"], cos, sin, case, half), _turn(st["k"], cos, sin, case, half)]
    if case["train"]:
        out += [_turn(st["dq"], cos, -sin, case, half), _turn(st["dk"], cos, -sin, case, half)]
    return out


def _visible(st):
    """Which keys each query row sees, [B or 1, Nq, Nk]."""
    case, dev = st["case"], st["q"].device
    B, Nq, Nk = case["B"], case["Nq"], case["Nk"]
    t = torch.arange(Nq, device=dev)[None, :, None]
    u = torch.arange(Nk, device=dev)[None, None, :]
    kl = torch.full((1,), Nk, device=dev) if st["kv_lens"] is None else st["kv_lens"].long()
    ql = torch.full((1,), Nq, device=dev) if st["q_lens"] is None else st["q_lens"].long()
    kl, ql = kl[:, None, None], ql[:, None, None]
    vis = (u < kl) & (t < ql)
    return vis & (u <= kl - ql + t) if case["causal"] else vis


def _plain_diff(st):
    case = st["case"]
    B, H, Hk, Nq, Nk, D = (case[x] for x in ("B", "H", "H_kv", "Nq", "Nk", "D"))
    g, d = H // Hk, D // 2
    scale = 1.0 / math.sqrt(d)
    q = st["q"].float().view(B, Hk, g, Nq, 2, d).permute(0, 1, 4, 2, 3, 5).reshape(B, Hk, 2, g * Nq, d)
    k = st["k"].float().view(B, Hk, Nk, 2, d).transpose(2, 3)                    # [B, Hk, 2, Nk, d]
    v = st["v"].float()
    lam = st["lam"].view(1, Hk, g, 1, 1)
    hidden = ~_visible(st)[:, None, None, None]
    s = (q @ k.transpose(-1, -2)).mul_(scale).view(B, Hk, 2, g, Nq, Nk).masked_fill_(hidden, -math.inf)
    s = s.sub_(s.amax(-1, keepdim=True).clamp_(min=-1e30)).exp_()
    p = s.div_(s.sum(-1, keepdim=True).clamp_(min=1e-30))
    a = (p[:, :, 0] - lam * p[:, :, 1]).view(B, Hk, g * Nq, Nk)
    out = (a @ v).view(B, H, Nq, D).to(st["q"].dtype)
    if not case["train"]:
        return out
    do = st["dout"].float().view(B, Hk, g * Nq, D)
    dv = a.transpose(-1, -2) @ do
    del a
    da = (do @ v.transpose(-1, -2)).view(B, Hk, 1, g, Nq, Nk)
    delta = (p * da).sum(-1, keepdim=True)                                      # [B, Hk, 2, g, Nq, 1]
    dlam = -delta[:, :, 1].double().sum((0, 3, 4)).view(H).float()
    sign = torch.stack([torch.ones_like(lam), -lam], 2)
    ds = ((da - delta) * p * (sign * scale)).view(B, Hk, 2, g * Nq, Nk)
    dq = (ds @ k).view(B, Hk, 2, g, Nq, d).permute(0, 1, 3, 4, 2, 5).reshape(B, H, Nq, D)
    dk = (ds.transpose(-1, -2) @ q).transpose(2, 3).reshape(B, Hk, Nk, D)
    dt = st["q"].dtype
    return [out, dq.to(dt), dk.to(dt), dv.to(dt), dlam]


# ------------------------------------------------------------------ one pass

def run(st):
    case = st["case"]
    if not own:
        return _plain_rotary(st) if case["op"] == "rotary" else _plain_diff(st)
    import paper_2410_20926_b200 as ta
    if case["op"] == "rotary":
        q, k = st["q"], st["k"]
        if case["train"]:
            q, k = q.detach().requires_grad_(), k.detach().requires_grad_()
        out = ta.multi_axis_rotary(q, k, st["sections"], positions=st["positions"], dims=st["dims"],
                                   base=10000.0, parts=case["parts"], interleaved=case["layout"] == "pairs",
                                   per_axis_ladder=case["ladder"] == "axis")
        if not case["train"]:
            return out
        grads = torch.autograd.grad(out, (q, k), (st["dq"], st["dk"]))
        return [x.detach() for x in out] + list(grads)
    q, k, v, lam = st["q"], st["k"], st["v"], st["lam"]
    if case["train"]:
        q, k, v, lam = (x.detach().requires_grad_() for x in (q, k, v, lam))
    out = ta.differential_attention(q, k, v, lam, causal=case["causal"], q_lens=st["q_lens"], kv_lens=st["kv_lens"])
    if not case["train"]:
        return out
    return [out.detach()] + list(torch.autograd.grad(out, (q, k, v, lam), st["dout"]))


def _pairs(case):
    """Visible (query row, key) pairs of one head, summed over the batch, and the rows and keys that count."""
    keys, rows = _lens(case)
    keys = keys or [case["Nk"]] * case["B"]
    rows = rows or [case["Nq"]] * case["B"]
    pairs = 0
    for kl, ql in zip(keys, rows):
        pairs += ql * kl - (ql * (ql - 1) // 2 if case["causal"] else 0)
    return pairs, sum(rows), sum(keys)


def work(case):
    e = 4 if case["dtype"] == "f32" else 2
    B, H, H_kv, D = case["B"], case["H"], case["H_kv"], case["D"]
    times = 2 if case["train"] else 1
    if case["op"] == "rotary":
        n = B * (H + H_kv) * case["N"] * D
        rotated = 2 * sum(_ints(case["sections"])) * case["parts"] / D
        pos = 0 if case["dims"] else 4 * len(_ints(case["sections"])) * B * case["N"]
        return {"bytes": times * 2 * e * n + pos, "flops": times * 3 * n * rotated}
    pairs, rows, keys = _pairs(case)
    every = B * H * case["Nq"] * D                                    # rows beyond a length are written too
    read = rows * H * D + 2 * keys * H_kv * D
    if not case["train"]:
        return {"bytes": e * (read + every), "flops": 4 * D * H * pairs}
    grads = every + 2 * B * H_kv * case["Nk"] * D
    return {"bytes": e * (read + rows * H * D + every + grads), "flops": 14 * D * H * pairs}


# ------------------------------------------------------------------ the definition in 64 bits

def _exact_rotary(st):
    """Every pair as a complex number, multiplied by the unit number of its angle."""
    case, sec = st["case"], st["sections"]
    half, parts = sum(sec), case["parts"]
    N = case["N"]
    if st["dims"] is not None:
        pos = np.stack(np.unravel_index(np.arange(N), st["dims"]))[:, None, :].repeat(case["B"], 1)
    else:
        pos = st["positions"].cpu().numpy()
    phase = np.empty((case["B"], N, half))
    c = 0
    for a, size in enumerate(sec):
        for i in range(size):
            expo = i / size if case["ladder"] == "axis" else c / half
            phase[..., c] = pos[a].astype(np.float64) * 10000.0 ** -expo
            c += 1
    unit = torch.polar(torch.ones(phase.shape, dtype=torch.float64), torch.from_numpy(phase)).cuda()
    unit = unit[:, None, :, None, :]

    def turned(x, by):
        B, heads, _, D = x.shape
        y = x.double().reshape(B, heads, N, parts, D // parts)
        res = y.clone()
        first, second = (slice(0, half), slice(half, 2 * half)) if case["layout"] == "halves" else \
            (slice(0, 2 * half, 2), slice(1, 2 * half, 2))
        z = torch.complex(y[..., first], y[..., second]) * by
        res[..., first], res[..., second] = z.real, z.imag
        return res.reshape(B, heads, N, D)

    out = [turned(st["q"], unit), turned(st["k"], unit)]
    if case["train"]:
        out += [turned(st["dq"], unit.conj()), turned(st["dk"], unit.conj())]
    return out


def _exact_diff(st):
    """Head by head over the valid rows and keys alone; the gradients by differentiating the definition."""
    case = st["case"]
    B, H, Hk, Nq, Nk, D = (case[x] for x in ("B", "H", "H_kv", "Nq", "Nk", "D"))
    g, d = H // Hk, D // 2
    keys, rows = _lens(case)
    q, k, v = (st[x].double() for x in ("q", "k", "v"))
    out = torch.zeros_like(q)
    train = case["train"]
    if train:
        dq, dk, dv, dlam = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v), [0.0] * H
    for b in range(B):
        kl = Nk if keys is None else keys[b]
        ql = Nq if rows is None else rows[b]
        for h in range(H):
            kh = h // g
            lam = st["lam"][h].double().requires_grad_(train)
            for t0 in range(0, ql, 4096):
                t1 = min(ql, t0 + 4096)
                see = kl - ql + t1 if case["causal"] else kl          # no row of the block sees further
                qq = q[b, h, t0:t1].clone().requires_grad_(train)
                kk = k[b, kh, :see].clone().requires_grad_(train)
                vv = v[b, kh, :see].clone().requires_grad_(train)
                bias = 0.0
                if case["causal"]:
                    at = torch.arange(t0, t1, device=q.device)[:, None] + (kl - ql)
                    bias = torch.zeros(t1 - t0, see, dtype=torch.float64, device=q.device)
                    bias.masked_fill_(torch.arange(see, device=q.device)[None] > at, -math.inf)
                one = torch.softmax(qq[:, :d] @ kk[:, :d].T / math.sqrt(d) + bias, -1) @ vv
                two = torch.softmax(qq[:, d:] @ kk[:, d:].T / math.sqrt(d) + bias, -1) @ vv
                o = one - lam * two
                out[b, h, t0:t1] = o.detach()
                if train:
                    gq, gk, gv, gl = torch.autograd.grad(o, (qq, kk, vv, lam), st["dout"][b, h, t0:t1].double())
                    dq[b, h, t0:t1] = gq
                    dk[b, kh, :see] += gk
                    dv[b, kh, :see] += gv
                    dlam[h] += gl
    if not train:
        return out
    return [out, dq, dk, dv, torch.stack(dlam)]


def exact(case, seed):
    st = prepare(case, seed)
    return _exact_rotary(st) if case["op"] == "rotary" else _exact_diff(st)
