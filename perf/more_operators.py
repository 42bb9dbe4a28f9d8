"""What a transformer block runs between its matrix products, as measurable cases.

A placement rests on what every operation costs on the machine that runs it,
and a user measures these by running them.  Besides attention over the batch
itself and the embedding, a block has four kinds of pass:

- ``rotary``, ``rotary_grad``: positions turn the pairs of each head's
  dimensions, of one axis (text) or several (time, height, width);
- ``dropout``: values dropped and the others scaled, from a counter-based
  generator, so that no mask is stored; its gradient is the same pass;
- ``norm``, ``norm_grad``: the end of one block and the beginning of the next:
  the norm of a block's output, its gate, dropout, the residual stream with
  its scale, and the norm before the next block;
- ``cross``, ``cross_train``: attention to an encoder's states, which have
  lengths of their own, and the same with its backward pass.

Sizes are the repository's own configurations (16 heads of 64 and 64 heads of
128, 4 sequences of 1024 tokens, hidden 1024 and 8192, 4 times that inside a
block) or generic ones.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DEVICE = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
SIZE = {"bf16": 2, "f16": 2, "f32": 4}
EPS = 1e-5


def _rotary(work, dtype, heads, dim, turned, tokens, axes, pairs=False, far=4096):
    return dict(work=work, dtype=dtype, heads=heads, dim=dim, turned=turned, tokens=tokens, axes=axes, pairs=pairs, far=far)


def _dropout(dtype, tokens, hidden, p=0.1):
    return dict(work="dropout", dtype=dtype, tokens=tokens, hidden=hidden, p=p)


def _norm(work, dtype, tokens, hidden, stream="", params="f32", center=False, bias=False, post=False, gate="", seqs=1, mix=0,
          pad=0, p=0.0, scale=1.0):
    return dict(work=work, dtype=dtype, stream=stream or dtype, params=params, tokens=tokens, hidden=hidden, center=center,
                bias=bias, post=post, gate=gate, seqs=seqs, mix=mix, pad=pad, p=p, scale=scale)


def _cross(work, dtype, heads, kv_heads, dim, seqs, tokens, source, mix=0, pad=0):
    return dict(work=work, dtype=dtype, heads=heads, kv_heads=kv_heads, dim=dim, seqs=seqs, tokens=tokens, source=source, mix=mix,
                pad=pad)


def listed():
    return [
        # a debugging batch, where a call's latency is all
        dict(name="rotary-small", **_rotary("rotary", "bf16", 16, 64, 64, 61, 1)),
        # transformer-96's queries with 8 key heads beside them, tokens of text and pictures
        dict(name="rotary-96", **_rotary("rotary", "bf16", 72, 128, 128, 4096, 3)),
        # backwards over packed documents at far positions, some dimensions left alone
        dict(name="rotary-grad-ragged", **_rotary("rotary_grad", "f16", 28, 80, 64, 9973, 2, pairs=True, far=1 << 20)),
        # a small layer's dropout, and that inside transformer-96's blocks
        dict(name="dropout-small", **_dropout("bf16", 512, 1024)),
        dict(name="dropout-96", **_dropout("bf16", 4096, 32768)),
        # transformer-24: layer norms with biases before each block, dropout behind it
        dict(name="norm-24", **_norm("norm", "bf16", 4096, 1024, center=True, bias=True, p=0.1)),
        # transformer-96 with norms on both sides, a gate for each channel and a 32-bit stream
        dict(name="norm-96", **_norm("norm", "bf16", 4096, 8192, stream="f32", post=True, gate="channel")),
        dict(name="norm-grad-24", **_norm("norm_grad", "bf16", 4096, 1024, center=True, bias=True, p=0.1)),
        # gates of each sequence's own, as conditioned blocks have them
        dict(name="norm-grad-96", **_norm("norm_grad", "bf16", 4096, 8192, post=True, gate="sequence", seqs=4, p=0.1, scale=0.5)),
        # a debugging batch of translations, one without a source; ordinary and long ones, trained
        dict(name="cross-small", **_cross("cross", "bf16", 8, 2, 64, 5, 211, 307, mix=1, pad=3)),
        dict(name="cross-train-ragged", **_cross("cross_train", "f16", 24, 4, 80, 37, 9973, 12011, mix=3, pad=27)),
        dict(name="cross-train-long", **_cross("cross_train", "bf16", 32, 8, 128, 2, 8192, 8192)),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rotary", "rotary_grad", "dropout", "norm", "norm", "norm_grad", "norm_grad", "cross", "cross_train"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    if kind.startswith("rotary"):
        dim = rng.choice([64, 128, 64, 128, 40, 80, 96, 256])
        tokens = _log(rng, 1, 16384)
        return _rotary(kind, dtype, _log(rng, 1, max(2, min(80, 2 ** 26 // (dim * tokens)))), dim, rng.choice([dim, dim, dim // 2, 2 * (dim // 6)]),
                       tokens, rng.choice([1, 1, 2, 3]), pairs=rng.random() < 0.5, far=_log(rng, 1000, 1 << 22))
    hidden = rng.choice([_log(rng, 64, 8192) // 8 * 8, _log(rng, 64, 8192) | 1])
    if kind == "dropout":
        times = rng.choice([1, 4])
        return _dropout(dtype, _log(rng, 1, 8192 // times), hidden * times, p=rng.choice([0.05, 0.1, 0.2, 0.5]))
    if kind.startswith("norm"):
        tokens = _log(rng, 1, 8192)
        gate = rng.choice(["", "", "channel", "sequence"])
        pad = tokens // 40 if gate == "sequence" else 0
        return _norm(kind, dtype, tokens, hidden, stream=rng.choice([dtype, "f32"]), params=rng.choice([dtype, "f32"]),
                     center=rng.random() < 0.4, bias=rng.random() < 0.3, post=rng.random() < 0.5, gate=gate,
                     seqs=min(_log(rng, 1, 60), tokens - pad) if gate == "sequence" else 1, mix=rng.randrange(1, 10 ** 6),
                     pad=pad, p=rng.choice([0.0, 0.1, 0.3]), scale=rng.choice([1.0, 0.5, 1.7]))
    kv, group = rng.choice([1, 2, 3, 4, 8]), rng.choice([1, 2, 4, 5, 8])
    dim = rng.choice([64, 128, 64, 128, 32, 40, 80, 96])
    most = max(300, min(8192, 8192 * 32 // (kv * group)))
    tokens, source = _log(rng, 100, most), _log(rng, 100, most)
    return _cross(kind, rng.choice(["bf16", "f16"]), kv * group, kv, dim, min(_log(rng, 1, 60), tokens // 2), tokens, source,
                  mix=rng.randrange(1, 10 ** 6), pad=rng.choice([0, 0, tokens // 40]))


def _lengths(total, n, mix, least=1):
    """n lengths in order with this sum: equal, or of a wide spread."""
    if not mix:
        return [total * (i + 1) // n - total * i // n for i in range(n)]
    share = np.random.default_rng([7, mix]).lognormal(0.0, 1.2, n)
    ends = np.floor(np.cumsum(share) / share.sum() * (total - least * n)).astype(np.int64)
    ends[-1] = total - least * n
    return [int(x) + least for x in np.diff(ends, prepend=0)]


def _sources(case):
    """The sources' lengths, apart from the targets'; of a mixed batch one has none."""
    n, total = case["seqs"], case["source"]
    if not case["mix"] or n < 3:
        return _lengths(total, n, case["mix"] and case["mix"] + 1)
    some = _lengths(total, n - 1, case["mix"] + 1)
    return some[:1] + [0] + some[1:]


def _pointers(lengths):
    return torch.from_numpy(np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32)).to(DEVICE)


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(1000003 * int(seed) + 29)
    dtype, T, kind = TYPES[case["dtype"]], case["tokens"], case["work"]

    def normal(*shape, dtype=dtype, by=1.0, at=0.0):
        return (torch.randn(shape, generator=gen, device=DEVICE, dtype=torch.float32) * by + at).to(dtype)

    if kind.startswith("rotary"):
        H, d, P, A = case["heads"], case["dim"], case["turned"] // 2, case["axes"]
        # one behind the other from some place on; the further axes' positions lie in a picture
        pos = torch.arange(T, device=DEVICE).repeat(A, 1) + int(seed) % 7 + case["far"] - min(T, case["far"])
        pos[1:] = torch.randint(0, 200, (A - 1, T), generator=gen, device=DEVICE)
        state = dict(case=case, x=normal(T, H, d), positions=pos.int() if T % 2 else pos,
                     freqs=(10000.0 ** (-torch.arange(P, device=DEVICE, dtype=torch.float64) / P)).float(),
                     axes=(torch.arange(P, device=DEVICE) * A // max(P, 1)).int() if A > 1 else None)
        return state
    rng = dict(seed=(int(seed) * 6364136223846793005 + 1442695040888963407) % 2 ** 63,
               step=torch.tensor([int(seed) + 5], dtype=torch.int64, device=DEVICE))
    if kind == "dropout":
        return dict(case=case, x=normal(T, case["hidden"]), **rng)
    if kind.startswith("norm"):
        h, stream, params = case["hidden"], TYPES[case["stream"]], TYPES[case["params"]]
        state = dict(case=case, f=normal(T, h, by=1.5, at=0.1), pre=normal(h, dtype=params, by=0.2, at=1.0), post=None,
                     pre_bias=None, post_bias=None, gate=None, ptr=None, lengths=None, **rng)
        if kind == "norm":
            state["x"] = normal(T, h, dtype=stream, by=2.0, at=-0.1)
        else:
            state.update(y=normal(T, h, dtype=stream, by=2.0, at=-0.1), dy=normal(T, h, dtype=stream), dz=normal(T, h))
        if case["bias"]:
            state["pre_bias"] = normal(h, dtype=params, by=0.1)
        if case["post"]:
            state["post"] = normal(h, dtype=params, by=0.2, at=1.0)
            if case["bias"]:
                state["post_bias"] = normal(h, dtype=params, by=0.1)
        if case["gate"] == "channel":
            state["gate"] = normal(h, dtype=params, by=0.5)
        elif case["gate"] == "sequence":
            state["lengths"] = _lengths(T - case["pad"], case["seqs"], case["mix"])
            state["ptr"], state["gate"] = _pointers(state["lengths"]), normal(case["seqs"], h, dtype=params, by=0.5)
        return state
    H, K, d, U = case["heads"], case["kv_heads"], case["dim"], case["source"]
    lengths, sources = _lengths(T - case["pad"], case["seqs"], case["mix"]), _sources(case)
    fused = normal(U, 2 * K * d)  # keys and values of the encoder's states, from one projection
    state = dict(case=case, lengths=lengths, sources=sources, q=normal(T, H, d), k=fused[:, :K * d].view(U, K, d),
                 v=fused[:, K * d:].view(U, K, d), q_ptr=_pointers(lengths), k_ptr=_pointers(sources))
    if kind == "cross_train":
        state["dout"] = normal(T, H, d)
    return state


# ------------------------------------------------------------------ plain form
def _plain_rotary(s, sign):
    case, x = s["case"], s["x"]
    P = case["turned"] // 2
    pos = s["positions"].double()
    pos = pos[0, :, None] if s["axes"] is None else pos[s["axes"].long()].T
    a = (pos * s["freqs"].double()).unsqueeze(1)
    c, w = torch.cos(a).float(), (torch.sin(a) * sign).float()
    out = x.float()
    if case["pairs"]:
        u, v = out[..., 0:2 * P:2], out[..., 1:2 * P:2]
        turned = torch.stack([u * c - v * w, v * c + u * w], 3).flatten(2)
    else:
        u, v = out[..., :P], out[..., P:2 * P]
        turned = torch.cat([u * c - v * w, v * c + u * w], 2)
    return torch.cat([turned, out[..., 2 * P:]], 2).to(x.dtype)


def _kept(rows, columns, p, seed, step):
    """Which values stay, [rows, columns]: 16 bits a value of Philox4x32-10, a block of the generator for
    eight columns of a row."""
    low = 0xffffffff
    c = [torch.arange((columns + 7) // 8, device=DEVICE).repeat(rows, 1), torch.arange(rows, device=DEVICE)[:, None],
         (step & low).reshape(1, 1), (step >> 32 & low).reshape(1, 1)]
    key = [seed & low, seed >> 32]
    for _ in range(10):
        a, b = c[0] * 0xd2511f53, c[2] * 0xcd9e8d57  # modulo 2^64: the lower halves are whole, the upper ones after a mask
        c = [(b >> 32 & low) ^ c[1] ^ key[0], b & low, (a >> 32 & low) ^ c[3] ^ key[1], a & low]
        key = [(key[0] + 0x9e3779b9) & low, (key[1] + 0xbb67ae85) & low]
    words = torch.stack(c, 2)
    bits = torch.stack([words & 0xffff, words >> 16], 3).reshape(rows, -1)[:, :columns]
    return bits >= round(p * 65536)


def _dropped(x, s):
    p = s["case"]["p"]
    if not p:
        return x
    keep = _kept(x.shape[0], x.shape[1], p, s["seed"], s["step"])
    return torch.where(keep, x * (65536.0 / (65536 - round(p * 65536))), torch.zeros((), device=x.device))


def _unit(v, center):
    """Rows of mean square 1 (or variance 1 around 0), and the factors that made them so."""
    v = v - v.mean(1, keepdim=True) if center else v
    r = 1.0 / torch.sqrt((v * v).mean(1, keepdim=True) + EPS)
    return v * r, r


def _unit_grad(g, unit, r, center):
    g = g - unit * (g * unit).mean(1, keepdim=True)
    return (g - g.mean(1, keepdim=True) if center else g) * r


def _gates(s):
    """The gate of every row, in 32 bits: 0 for a row of no sequence."""
    gate = s["gate"]
    if gate is None or s["ptr"] is None:
        return gate if gate is None else gate.float()
    rows = torch.zeros(s["f"].shape, device=gate.device)
    n = torch.diff(s["ptr"]).long()
    rows[:s["case"]["tokens"] - s["case"]["pad"]] = gate.float().repeat_interleave(n, 0, output_size=sum(s["lengths"]))
    return rows


def _plain_norm(s):
    case = s["case"]
    n = s["f"].float()
    if s["post"] is not None:
        n = _unit(n, case["center"])[0] * s["post"].float()
        n = n if s["post_bias"] is None else n + s["post_bias"].float()
    n, gate = _dropped(n, s), _gates(s)
    y = s["x"].float() * case["scale"] + (n if gate is None else n * gate)
    z = _unit(y, case["center"])[0] * s["pre"].float()
    z = z if s["pre_bias"] is None else z + s["pre_bias"].float()
    return dict(y=y.to(s["x"].dtype), z=z.to(s["f"].dtype))


def _plain_norm_grad(s):
    case, out = s["case"], {}
    center, gate = case["center"], _gates(s)
    dz = s["dz"].float()
    Y, r = _unit(s["y"].float(), center)
    dyt = s["dy"].float() + _unit_grad(dz * s["pre"].float(), Y, r, center)
    out["pre"] = (dz * Y).sum(0)
    if s["pre_bias"] is not None:
        out["pre_bias"] = dz.sum(0)
    out["dx"] = (dyt * case["scale"]).to(s["y"].dtype)
    n = s["f"].float()
    if s["post"] is not None:
        N, rf = _unit(n, center)
        n = N * s["post"].float()
        n = n if s["post_bias"] is None else n + s["post_bias"].float()
    if gate is not None:
        per_row = dyt * _dropped(n, s)
        if s["ptr"] is None:
            out["gate"] = per_row.sum(0)
        else:
            at = torch.repeat_interleave(torch.arange(case["seqs"], device=DEVICE), torch.diff(s["ptr"]).long(), output_size=sum(s["lengths"]))
            out["gate"] = torch.zeros(case["seqs"], n.shape[1], device=DEVICE).index_add_(0, at, per_row[:len(at)])
    dn = _dropped(dyt if gate is None else dyt * gate, s)
    if s["post"] is not None:
        out["post"] = (dn * N).sum(0)
        if s["post_bias"] is not None:
            out["post_bias"] = dn.sum(0)
        dn = _unit_grad(dn * s["post"].float(), N, rf, center)
    out["df"] = dn.to(s["f"].dtype)
    return out


def _grouped(x, heads):
    """Rows of one sequence [L, kv heads, d] as [heads, L, d] in 32 bits."""
    L, K, d = x.shape
    return x.float().permute(1, 0, 2).reshape(K, 1, L, d).expand(K, heads // K, L, d).reshape(heads, L, d)


def _plain_cross(s, train):
    q, k, v = s["q"], s["k"], s["v"]
    (T, H, d), K = q.shape, k.shape[1]
    c = 1.0 / math.sqrt(d)
    out, lse = torch.zeros_like(q), torch.full((H, T), -math.inf, device=q.device)
    dq, dk, dv = (torch.zeros(x.shape, dtype=q.dtype, device=q.device) for x in (q, k, v))
    at = k_at = 0
    for L, M in zip(s["lengths"], s["sources"]):
        rows, keys, at, k_at = slice(at, at + L), slice(k_at, k_at + M), at + L, k_at + M
        if not M:
            continue
        Q, KK, VV = _grouped(q[rows], H), _grouped(k[keys], H), _grouped(v[keys], H)
        x = torch.matmul(Q, KK.transpose(1, 2).contiguous()).mul_(c)
        top = x.amax(2, keepdim=True)
        p = torch.exp(x.sub_(top))
        total = p.sum(2, keepdim=True)
        lse[:, rows] = (torch.log(total) + top)[:, :, 0]
        p /= total
        o = torch.matmul(p, VV)
        out[rows] = o.permute(1, 0, 2).to(q.dtype)
        if not train:
            continue
        do = _grouped(s["dout"][rows], H)
        dV = torch.matmul(p.transpose(1, 2).contiguous(), do)
        dp = torch.matmul(do, VV.transpose(1, 2).contiguous())
        ds = p.mul_(dp - (do * o).sum(2, keepdim=True)).mul_(c)
        dQ, dK = torch.matmul(ds, KK), torch.matmul(ds.transpose(1, 2).contiguous(), Q)
        dq[rows] = dQ.permute(1, 0, 2).to(q.dtype)
        dk[keys] = dK.view(K, H // K, M, d).sum(1).permute(1, 0, 2).to(q.dtype)
        dv[keys] = dV.view(K, H // K, M, d).sum(1).permute(1, 0, 2).to(q.dtype)
    return dict(out=out, dq=dq, dk=dk, dv=dv) if train else dict(out=out, lse=lse)


def _plain(state, kind):
    if kind.startswith("rotary"):
        return _plain_rotary(state, -1.0 if kind == "rotary_grad" else 1.0)
    if kind == "dropout":
        return _dropped(state["x"].float(), state).to(state["x"].dtype)
    if kind.startswith("norm"):
        return _plain_norm(state) if kind == "norm" else _plain_norm_grad(state)
    return _plain_cross(state, kind == "cross_train")


def run(state):
    s, case = state, state["case"]
    kind = case["work"]
    if not own:
        return _plain(s, kind)
    import paper_2208_00184_amd as cel
    if kind.startswith("rotary"):
        f = cel.rotary if kind == "rotary" else cel.rotary_grad
        return f(s["x"], s["positions"], s["freqs"], axes=s["axes"], pairs=case["pairs"])
    if kind == "dropout":
        return cel.dropout(s["x"], case["p"], s["seed"], step=s["step"])
    if kind.startswith("norm"):
        how = dict(post=s["post"], gate=s["gate"], seq_ptr=s["ptr"], pre_bias=s["pre_bias"], post_bias=s["post_bias"],
                   scale=case["scale"], p=case["p"], seed=s["seed"], step=s["step"], eps=EPS, center=case["center"])
        if kind == "norm":
            y, z = cel.residual_norm(s["f"], s["x"], s["pre"], **how)
            return dict(y=y, z=z)
        dx, df, grads = cel.residual_norm_grad(s["dy"], s["dz"], s["f"], s["y"], s["pre"], **how)
        return dict(dx=dx, df=df, **grads)
    args = s["q"], s["k"], s["v"]
    out, lse = cel.cross_attention(*args, s["q_ptr"], s["k_ptr"])
    if kind == "cross":
        return dict(out=out, lse=lse)
    dq, dk, dv = cel.cross_attention_grad(s["dout"], *args, out, lse, s["q_ptr"], s["k_ptr"])
    return dict(out=out, dq=dq, dk=dk, dv=dv)


def work(case):
    T, size, kind = case["tokens"], SIZE[case["dtype"]], case["work"]
    if kind.startswith("rotary"):
        values = T * case["heads"] * case["dim"]
        return dict(bytes=2 * values * size + T * case["axes"] * (4 if T % 2 else 8) + 2 * case["turned"],
                    flops=3 * T * case["heads"] * case["turned"])
    h = case.get("hidden", 0)
    if kind == "dropout":
        return dict(bytes=2 * T * h * size, flops=T * h)
    if kind.startswith("norm"):
        stream, few = SIZE[case["stream"]], 1 + case["post"]
        few += case["bias"] * few
        few += {"": 0, "channel": 1, "sequence": case["seqs"]}[case["gate"]]
        if kind == "norm":  # f, x in; y, z out
            return dict(bytes=2 * T * h * (size + stream) + few * h * SIZE[case["params"]], flops=T * h * (7 + 4 * case["post"]))
        # dy, dz, y in, and f where a gradient needs it; dx, df out, and the parameters' gradients in 32 bits
        f = size * bool(case["post"] or case["gate"])
        return dict(bytes=T * h * (3 * stream + 2 * size + f) + few * h * (SIZE[case["params"]] + 4), flops=T * h * (13 + 12 * case["post"]))
    H, K, d, U = case["heads"], case["kv_heads"], case["dim"], case["source"]
    pairs = sum(a * b for a, b in zip(_lengths(T - case["pad"], case["seqs"], case["mix"]), _sources(case)))
    rows, few = 2 * T * H * d, 2 * U * K * d
    if kind == "cross":  # q, k, v in; out and lse out
        return dict(bytes=2 * rows + 2 * few + 4 * T * H, flops=4 * d * H * pairs)
    # q, k, v, dout in; out, dq, dk, dv out
    return dict(bytes=4 * rows + 4 * few, flops=14 * d * H * pairs)


# ------------------------------------------------------- definition in 64 bits
def _stays(rows, columns, p, seed, step):
    """The same generator, from products of 16-bit pieces, a row of blocks for each of its four words."""
    def wide(m, x):  # -> the upper and lower 32 bits of m x
        ml, mh, xl, xh = m & 65535, m >> 16, x & 65535, x >> 16
        ll, lh, hl, hh = ml * xl, ml * xh, mh * xl, mh * xh
        mid = (ll >> 16) + (lh & 65535) + (hl & 65535)
        return hh + (lh >> 16) + (hl >> 16) + (mid >> 16), (mid & 65535) << 16 | ll & 65535

    blocks = -(-columns // 8)
    n = torch.arange(rows * blocks, device=DEVICE)
    step = int(step)
    x0, x1 = n % blocks, torch.div(n, blocks, rounding_mode="floor")
    x2, x3 = torch.full_like(n, step % 2 ** 32), torch.full_like(n, (step >> 32) % 2 ** 32)
    for i in range(10):
        k0, k1 = (seed % 2 ** 32 + i * 0x9e3779b9) % 2 ** 32, (seed // 2 ** 32 + i * 0xbb67ae85) % 2 ** 32
        h0, l0 = wide(0xd2511f53, x0)
        h1, l1 = wide(0xcd9e8d57, x2)
        x0, x1, x2, x3 = h1 ^ x1 ^ k0, l1, h0 ^ x3 ^ k1, l0
    least, keep = int(p * 65536 + 0.5), torch.empty(rows, blocks, 8, dtype=torch.bool, device=DEVICE)
    for j, x in enumerate((x0, x1, x2, x3)):
        keep[:, :, 2 * j] = ((x & 65535) >= least).view(rows, blocks)
        keep[:, :, 2 * j + 1] = ((x >> 16) >= least).view(rows, blocks)
    return keep.view(rows, 8 * blocks)[:, :columns], 1.0 / (1.0 - least / 65536.0)


def _exact_norm(case, s):
    def up(name):
        return None if s.get(name) is None else s[name].double()

    T, h, center = case["tokens"], case["hidden"], case["center"]
    step = max(1, 2 ** 25 // h)  # rows at a time
    pre, post, pre_bias, post_bias, gate = (up(n) for n in ("pre", "post", "pre_bias", "post_bias", "gate"))
    of = torch.full((T,), -1, dtype=torch.int64, device=DEVICE)  # each row's gate
    if case["gate"] == "channel":
        of[:], gate = 0, gate[None]
    elif case["gate"]:
        for i, (a, b) in enumerate(zip(s["ptr"].tolist(), s["ptr"].tolist()[1:])):
            of[a:b] = i
    if case["p"]:
        keep, by = _stays(T, h, case["p"], s["seed"], s["step"])

    def normed(v):
        v = v - v.mean(1, keepdim=True) if center else v
        return v * (v.square().mean(1, keepdim=True) + EPS).rsqrt()

    parts = []
    names = ["pre"] + ["pre_bias"] * case["bias"] + ["post"] * case["post"] + ["post_bias"] * (case["post"] and case["bias"])
    sums = {n: torch.zeros(h, dtype=torch.float64, device=DEVICE) for n in names}
    if gate is not None:
        sums["gate"] = torch.zeros_like(gate)
    for a in range(0, T, step):
        rows = slice(a, min(T, a + step))
        leaves = {n: t.clone().requires_grad_() for n, t in (("pre", pre), ("pre_bias", pre_bias), ("post", post),
                                                            ("post_bias", post_bias)) if t is not None}
        f = s["f"][rows].double().requires_grad_()

        def branch():
            n = f
            if post is not None:
                n = normed(f) * leaves["post"]
                n = n + leaves["post_bias"] if post_bias is not None else n
            return torch.where(keep[rows], n * by, 0.0) if case["p"] else n

        gates = None
        if gate is not None:
            gates = torch.where(of[rows, None] >= 0, gate[of[rows].clamp(min=0)], 0.0).requires_grad_()
        n = branch()
        if case["work"] == "norm":
            y = s["x"][rows].double() * case["scale"] + (n if gates is None else n * gates)
            z = normed(y) * pre
            parts.append((y.detach(), (z + pre_bias if pre_bias is not None else z).detach()))
            continue
        y = s["y"][rows].double().requires_grad_()
        z = normed(y) * leaves["pre"]
        z = z + leaves["pre_bias"] if pre_bias is not None else z
        first = [n for n in ("pre", "pre_bias") if n in leaves]
        g = torch.autograd.grad(z, [y] + [leaves[n] for n in first], s["dz"][rows].double())
        total = s["dy"][rows].double() + g[0]
        second = [n for n in ("post", "post_bias") if n in leaves]
        b = n if gates is None else n * gates
        g2 = torch.autograd.grad(b, [f] + [leaves[n] for n in second] + ([] if gates is None else [gates]), total)
        parts.append((total * case["scale"], g2[0]))
        for name, t in zip(first + second, g[1:] + g2[1:]):
            sums[name] += t
        if gates is not None:
            there = of[rows] >= 0
            sums["gate"].index_add_(0, of[rows][there], g2[-1][there])
    one, two = (torch.cat(x) for x in zip(*parts))
    if case["work"] == "norm":
        return dict(y=one, z=two)
    if case["gate"] == "channel":
        sums["gate"] = sums["gate"][0]
    return dict(dx=one, df=two, **sums)


def _cross64(q, k, v, c):
    x = (q @ k.transpose(1, 2)) * c
    lse = torch.logsumexp(x, 2)
    return torch.exp(x - lse[:, :, None]) @ v, lse


def exact(case, seed):
    s, kind = prepare(case, seed), case["work"]
    if kind.startswith("rotary"):
        x, P = s["x"].double(), case["turned"] // 2
        out = x.clone()
        for p in range(P):
            axis = 0 if s["axes"] is None else int(s["axes"][p])
            turn = torch.polar(torch.ones(case["tokens"], dtype=torch.float64, device=DEVICE),
                               s["positions"][axis].double() * float(s["freqs"][p]))[:, None]
            i, j = (2 * p, 2 * p + 1) if case["pairs"] else (p, p + P)
            w = torch.complex(x[:, :, i], x[:, :, j]) * (turn.conj() if kind == "rotary_grad" else turn)
            out[:, :, i], out[:, :, j] = w.real, w.imag
        return out
    if kind == "dropout":
        keep, by = _stays(case["tokens"], case["hidden"], case["p"], s["seed"], s["step"])
        return torch.where(keep, s["x"].double() * by, 0.0)
    if kind.startswith("norm"):
        return _exact_norm(case, s)
    T, U, H, K, d = case["tokens"], case["source"], case["heads"], case["kv_heads"], case["dim"]
    train, c = kind == "cross_train", 1.0 / math.sqrt(d)
    out = torch.zeros(T, H, d, dtype=torch.float64, device=DEVICE)
    lse = torch.full((H, T), -math.inf, dtype=torch.float64, device=DEVICE)
    dq, dk, dv = (torch.zeros(t, n, d, dtype=torch.float64, device=DEVICE) for t, n in ((T, H), (U, K), (U, K)))
    kv_of = torch.arange(H, device=DEVICE) * K // H
    q_ptr, k_ptr = s["q_ptr"].tolist(), s["k_ptr"].tolist()
    for i in range(case["seqs"]):
        rows, keys = slice(q_ptr[i], q_ptr[i + 1]), slice(k_ptr[i], k_ptr[i + 1])
        L, M = rows.stop - rows.start, keys.stop - keys.start
        if not M:
            continue
        step = max(1, 2 ** 28 // (L * M))
        for a in range(0, H, step):
            heads = torch.arange(a, min(H, a + step), device=DEVICE)
            x = [t.transpose(0, 1).contiguous().requires_grad_(train) for t in (
                s["q"][rows, a:a + step].double(), s["k"][keys][:, kv_of[heads]].double(), s["v"][keys][:, kv_of[heads]].double())]
            o, z = _cross64(*x, c)
            out[rows, a:a + step] = o.detach().transpose(0, 1)
            lse[a:a + step, rows] = z.detach()
            if train:
                gq, gk, gv = torch.autograd.grad(o, x, s["dout"][rows, a:a + step].double().transpose(0, 1).contiguous())
                dq[rows, a:a + step] = gq.transpose(0, 1)
                dk[keys].index_add_(1, kv_of[heads], gk.transpose(0, 1).contiguous())
                dv[keys].index_add_(1, kv_of[heads], gv.transpose(0, 1).contiguous())
    return dict(out=out, dq=dq, dk=dk, dv=dv) if train else dict(out=out, lse=lse)
