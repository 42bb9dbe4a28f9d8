"""The operators of a transformer training step, as measurable cases.

A placement rests on what every operation costs on the machine that runs it,
and a user measures these by running them.  Four kinds of pass:

- ``attend``: causal attention over a packed batch (sequences one behind the
  other, query heads sharing key/value heads), as a forward pass calls it;
- ``attend_train``: the same with its backward pass, as a training step
  calls the two;
- ``embed``: rows of an embedding table by token id, scaled;
- ``embed_grad``: the table's gradient, dense, from the gradient of the rows.

Queries, keys and values are views of one fused projection, as a model's
linear layer writes them.  Token ids follow Zipf's law, as words do; an id of
-1 is padding.  Sizes are the repository's own configurations (16 heads of 64
and 64 heads of 128, 4 sequences of 1024 tokens, hidden 1024 and 8192) or
generic ones.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DEVICE = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


def _attend(work, dtype, heads, kv_heads, dim, seqs, tokens, mix=0, pad=0):
    return dict(work=work, dtype=dtype, heads=heads, kv_heads=kv_heads, dim=dim, seqs=seqs, tokens=tokens, mix=mix,
                pad=pad)


def _embed(work, dtype, vocab, hidden, tokens, pad=0, grad="", wide=False):
    return dict(work=work, dtype=dtype, vocab=vocab, hidden=hidden, tokens=tokens, pad=pad, grad=grad or dtype,
                wide_ids=wide)


def listed():
    return [
        # a debugging batch: a few short sequences, where a call's latency is all
        dict(name="attend-small", **_attend("attend", "bf16", 8, 2, 64, 5, 211, mix=1, pad=3)),
        # transformer-24's attention: 16 heads of 64, 4 sequences of 1024
        dict(name="attend-24", **_attend("attend", "bf16", 16, 16, 64, 4, 4096)),
        # a packed batch of documents of very different lengths, padded
        dict(name="attend-ragged", **_attend("attend", "f16", 32, 8, 128, 61, 16301, mix=2, pad=83)),
        # one long context
        dict(name="attend-long", **_attend("attend", "bf16", 16, 4, 128, 1, 16384)),
        # training: transformer-24 as it is, and transformer-96's 64 heads of 128
        dict(name="train-24", **_attend("attend_train", "bf16", 16, 16, 64, 4, 4096)),
        dict(name="train-96", **_attend("attend_train", "bf16", 64, 64, 128, 4, 4096)),
        # training on packed documents with grouped heads of an uneven size
        dict(name="train-ragged", **_attend("attend_train", "f16", 24, 4, 80, 37, 9973, mix=3, pad=27)),
        # training on one long sequence
        dict(name="train-long", **_attend("attend_train", "bf16", 32, 8, 128, 1, 8192)),
        # the lookup of a small batch, and of a large one into the wide model
        dict(name="embed-small", **_embed("embed", "bf16", 32000, 1024, 512)),
        dict(name="embed-96", **_embed("embed", "bf16", 131072, 8192, 32768, pad=500, wide=True)),
        # the gradient of transformer-24's table, summed into 32 bits, and of the wide model's
        dict(name="embed-grad-24", **_embed("embed_grad", "bf16", 50001, 1024, 4096, grad="f32")),
        dict(name="embed-grad-96", **_embed("embed_grad", "bf16", 131072, 8192, 32768, pad=500, wide=True)),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["attend", "attend", "attend_train", "attend_train", "embed", "embed_grad"])
    if kind.startswith("embed"):
        hidden = rng.choice([_log(rng, 64, 8192) // 8 * 8, _log(rng, 64, 8192) | 1])
        tokens = _log(rng, 100, 32768)
        dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
        return _embed(kind, dtype, _log(rng, 1000, 131072 if dtype != "f32" else 65536), hidden, tokens,
                      pad=rng.choice([0, tokens // 50]), grad=rng.choice([dtype, "f32"]) if kind == "embed_grad" else "",
                      wide=rng.random() < 0.5)
    kv = rng.choice([1, 2, 3, 4, 8])
    group = rng.choice([1, 2, 4, 5, 8])
    dim = rng.choice([64, 128, 64, 128, 32, 40, 80, 96])
    most = 16384 * 16 if kind == "attend" else 8192 * 32  # tokens times heads
    tokens = _log(rng, 100, max(200, min(16384 if kind == "attend" else 8192, most // (kv * group))))
    seqs = min(_log(rng, 1, 100), tokens)
    return _attend(kind, rng.choice(["bf16", "f16"]), kv * group, kv, dim, seqs, tokens, mix=rng.randrange(1, 10 ** 6),
                   pad=rng.choice([0, 0, tokens // 40]))


def _lengths(case):
    """The batch's sequence lengths, in order: equal, or of a wide spread.

    The padding at the batch's end belongs to no sequence."""
    n, total = case["seqs"], case["tokens"] - case["pad"]
    if not case["mix"]:
        return [total * (i + 1) // n - total * i // n for i in range(n)]
    share = np.random.default_rng([7, case["mix"]]).lognormal(0.0, 1.2, n)
    ends = np.floor(np.cumsum(share) / share.sum() * (total - n)).astype(np.int64)
    ends[-1] = total - n
    return [int(x) + 1 for x in np.diff(ends, prepend=0)]


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(1000003 * int(seed) + 17)
    dtype, T = TYPES[case["dtype"]], case["tokens"]

    def normal(*shape, dtype=dtype):
        return torch.randn(shape, generator=gen, device=DEVICE, dtype=torch.float32).to(dtype)

    if case["work"].startswith("attend"):
        H, K, d = case["heads"], case["kv_heads"], case["dim"]
        lengths = _lengths(case)
        fused = normal(T, (H + 2 * K) * d)
        ptr = np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32)
        state = dict(case=case, lengths=lengths, q=fused[:, :H * d].view(T, H, d),
                     k=fused[:, H * d:(H + K) * d].view(T, K, d), v=fused[:, (H + K) * d:].view(T, K, d),
                     seq_ptr=torch.from_numpy(ptr).to(DEVICE))
        if case["work"] == "attend_train":
            state["dout"] = normal(T, H, d)
        return state
    V, h = case["vocab"], case["hidden"]
    u = torch.rand(T, generator=gen, device=DEVICE, dtype=torch.float64)
    ids = (torch.exp(u * math.log(V + 1.0)) - 1.0).long().clamp_(0, V - 1)
    ids = ids * 7919 % V if V % 7919 else ids  # frequent words lie anywhere in a table
    if case["pad"]:
        ids[-case["pad"]:] = -1
    ids = ids if case["wide_ids"] else ids.int()
    state = dict(case=case, ids=ids, scale=math.sqrt(h))
    if case["work"] == "embed":
        state["table"] = normal(V, h) * 0.02
    else:
        state["dx"] = normal(T, h)
    return state


# ------------------------------------------------------------------ plain form
def _grouped(x, heads):
    """Rows of one sequence [L, kv heads, d] as [heads, L, d] in 32 bits."""
    L, K, d = x.shape
    return x.float().permute(1, 0, 2).reshape(K, 1, L, d).expand(K, heads // K, L, d).reshape(heads, L, d)


def _scores(q, k, c):
    L = q.shape[1]
    s = torch.matmul(q, k.transpose(1, 2).contiguous()) * c
    later = torch.ones(L, L, dtype=torch.bool, device=q.device).triu_(1)
    return s.masked_fill_(later, -math.inf)


def _plain_attend(s, train):
    q, k, v, ptr = s["q"], s["k"], s["v"], s["lengths"]
    T, H, d = q.shape
    K, c = k.shape[1], 1.0 / math.sqrt(d)
    out, lse = torch.zeros(T, H, d, dtype=q.dtype, device=q.device), torch.full((H, T), -math.inf, device=q.device)
    grads = [torch.zeros(T, n, d, dtype=q.dtype, device=q.device) for n in ((H, K, K) if train else ())]
    at = 0
    for L in ptr:
        rows, at = slice(at, at + L), at + L
        Q, KK, VV = _grouped(q[rows], H), _grouped(k[rows], H), _grouped(v[rows], H)
        x = _scores(Q, KK, c)
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
        grads[0][rows] = dQ.permute(1, 0, 2).to(q.dtype)
        grads[1][rows] = dK.view(K, H // K, L, d).sum(1).permute(1, 0, 2).to(q.dtype)
        grads[2][rows] = dV.view(K, H // K, L, d).sum(1).permute(1, 0, 2).to(q.dtype)
    return dict(out=out, dq=grads[0], dk=grads[1], dv=grads[2]) if train else dict(out=out, lse=lse)


def _plain_embed(s):
    ids, table = s["ids"].long(), s["table"]
    rows = table[ids.clamp(min=0)].float() * s["scale"]
    return (rows * (ids >= 0).unsqueeze(1)).to(table.dtype)


def _plain_embed_grad(s):
    ids, dx, case = s["ids"].long(), s["dx"], s["case"]
    there = ids >= 0
    total = torch.zeros(case["vocab"], dx.shape[1], device=dx.device)
    total.index_add_(0, ids[there], dx[there].float())
    return total.mul_(s["scale"]).to(TYPES[case["grad"]])


def run(state):
    kind = state["case"]["work"]
    if not own:
        if kind.startswith("attend"):
            return _plain_attend(state, kind == "attend_train")
        return _plain_embed(state) if kind == "embed" else _plain_embed_grad(state)
    import paper_2208_00184_amd as cel
    if kind == "embed":
        return cel.embed(state["table"], state["ids"], scale=state["scale"])
    if kind == "embed_grad":
        return cel.embed_grad(state["dx"], state["ids"], state["case"]["vocab"], scale=state["scale"],
                              dtype=TYPES[state["case"]["grad"]])
    q, k, v, ptr = state["q"], state["k"], state["v"], state["seq_ptr"]
    out, lse = cel.attention(q, k, v, ptr)
    if kind == "attend":
        return dict(out=out, lse=lse)
    dq, dk, dv = cel.attention_grad(state["dout"], q, k, v, out, lse, ptr)
    return dict(out=out, dq=dq, dk=dk, dv=dv)


def work(case):
    T = case["tokens"]
    if case["work"].startswith("attend"):
        H, K, d = case["heads"], case["kv_heads"], case["dim"]
        pairs = sum(L * (L + 1) // 2 for L in _lengths(case))
        rows, few = 2 * T * H * d, 2 * T * K * d
        if case["work"] == "attend":  # q, k, v in; out and lse out
            return dict(bytes=2 * rows + 2 * few + 4 * T * H, flops=4 * d * H * pairs)
        # q, k, v, dout in; out, dq, dk, dv out
        return dict(bytes=4 * rows + 4 * few, flops=14 * d * H * pairs)
    size = {"bf16": 2, "f16": 2, "f32": 4}
    V, h, n = case["vocab"], case["hidden"], T - case["pad"]
    wide = 8 if case["wide_ids"] else 4
    if case["work"] == "embed":
        # distinct rows of a Zipf sample: row r is drawn with share log(1 + 1 / r) / log(V + 1)
        r = np.arange(1, V + 1, dtype=np.float64)
        seen = float((1.0 - np.exp(n * np.log1p(-np.log1p(1.0 / r) / math.log(V + 1.0)))).sum())
        return dict(bytes=wide * T + (seen + T) * h * size[case["dtype"]], flops=T * h)
    return dict(bytes=wide * T + n * h * size[case["dtype"]] + V * h * size[case["grad"]], flops=n * h + V * h)


# ------------------------------------------------------- definition in 64 bits
def _attention64(q, k, v, c):
    """Some heads' attention inside one sequence, [n, L, d] each, from the definition."""
    x = (q @ k.transpose(1, 2)) * c
    i = torch.arange(x.shape[1], device=x.device)
    x = torch.where(i[None, :] <= i[:, None], x, torch.full((), -math.inf, dtype=x.dtype, device=x.device))
    lse = torch.logsumexp(x, 2)
    return torch.exp(x - lse[:, :, None]) @ v, lse


def exact(case, seed):
    s = prepare(case, seed)
    if case["work"] == "embed":
        out = torch.zeros(case["tokens"], case["hidden"], dtype=torch.float64, device=DEVICE)
        hit = s["ids"] >= 0
        out[hit] = s["table"].index_select(0, s["ids"][hit].int()).double() * s["scale"]
        return out
    if case["work"] == "embed_grad":
        # sums of runs of the sorted ids, a slice of columns at a time
        V, h = case["vocab"], case["hidden"]
        ids, order = torch.sort(s["ids"].long(), stable=True)
        runs = torch.searchsorted(ids, torch.arange(V + 1, device=DEVICE))
        out = torch.zeros(V, h, dtype=torch.float64, device=DEVICE)
        for a in range(0, h, 512):
            cut = slice(a, min(h, a + 512))
            upto = torch.zeros(len(ids) + 1, cut.stop - a, dtype=torch.float64, device=DEVICE)
            torch.cumsum(s["dx"][:, cut].index_select(0, order).double(), 0, out=upto[1:])
            out[:, cut] = (upto[runs[1:]] - upto[runs[:-1]]) * s["scale"]
        return out
    T, H, K, d = case["tokens"], case["heads"], case["kv_heads"], case["dim"]
    train, c = case["work"] == "attend_train", 1.0 / math.sqrt(d)
    out = torch.zeros(T, H, d, dtype=torch.float64, device=DEVICE)
    lse = torch.full((H, T), -math.inf, dtype=torch.float64, device=DEVICE)
    dq, dk, dv = (torch.zeros(T, n, d, dtype=torch.float64, device=DEVICE) for n in (H, K, K))
    kv_of = torch.arange(H, device=DEVICE) * K // H
    first = 0
    for L in _lengths(case):
        last = first + L
        step = max(1, 2 ** 28 // (L * L))
        for a in range(0, H, step):
            heads = torch.arange(a, min(H, a + step), device=DEVICE)
            q = s["q"][first:last, a:a + step].double().transpose(0, 1).contiguous().requires_grad_(train)
            k = s["k"][first:last][:, kv_of[heads]].double().transpose(0, 1).contiguous().requires_grad_(train)
            v = s["v"][first:last][:, kv_of[heads]].double().transpose(0, 1).contiguous().requires_grad_(train)
            o, z = _attention64(q, k, v, c)
            out[first:last, a:a + step] = o.detach().transpose(0, 1)
            lse[a:a + step, first:last] = z.detach()
            if train:
                do = s["dout"][first:last, a:a + step].double().transpose(0, 1).contiguous()
                gq, gk, gv = torch.autograd.grad(o, (q, k, v), do)
                dq[first:last, a:a + step] = gq.transpose(0, 1)
                dk[first:last].index_add_(1, kv_of[heads], gk.transpose(0, 1).contiguous())
                dv[first:last].index_add_(1, kv_of[heads], gv.transpose(0, 1).contiguous())
        first = last
    return dict(out=out, dq=dq, dk=dk, dv=dv) if train else dict(out=out, lse=lse)
