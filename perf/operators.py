"""Operators of language models around the token-subset backward, as cases to be timed.

Between the linear layers of a language model's block, and below the first of them, a training step with a subset of kept
tokens runs these, and the library has a call for each:

  attention           forward over all tokens: scores capped by a tanh, a bias that falls with the distance, and a mask of causal
                      order, a prefix that everyone sees, and documents packed into one row (tokens of no document are padding)
  attention_backward  its backward on the kept tokens (dropped queries and keys take no part), shared key / value heads included
  norms               the step between two blocks: residual * alpha + gate * norm(block output), and the next block's norm of it
  norms_backward      its backward on the kept rows: the residual gradient of all rows, the compact gradient of the block output,
                      and the gradients of the gate and of both norms' parameters
  embedding           the scaled lookup of a token table and the table's gradient from the kept rows

`own` false computes them in elementary torch operations in 32 bits; `own` true calls the library.
Values: activations and gradients N(0, 1) (queries and keys as well: scores of a fresh model), scales around 1, tokens with
frequencies that fall like 1 / rank.
"""
import math
import random

import torch

own = False

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
EPS = 1e-5


def listed():
    return [
        # Two short sentences in a unit-test-sized fp32 model, a prefix in front: launches and host time are everything.
        dict(name="attention_short_f32", kind="attention", dtype="f32", B=2, n=49, h=3, hk=3, d=64, causal=True, cap=30.0, slopes=False,
             docs=0, prefix=16, pad=0),
        # A batch of packed documents of ordinary length, with a distance bias; the last sample ends in padding.
        dict(name="attention_packed", kind="attention", dtype="bf16", B=4, n=2048, h=12, hk=12, d=64, causal=True, cap=0.0, slopes=True,
             docs=500, prefix=0, pad=300),
        # One long text, 16 query heads that share 2 key / value heads, capped scores: the largest forward.
        dict(name="attention_long", kind="attention", dtype="bf16", B=1, n=8192, h=16, hk=2, d=128, causal=True, cap=50.0, slopes=False,
             docs=0, prefix=0, pad=0),
        # Half the tokens of three rows of 197, one shared key / value head, a prefix of 64 tokens, fp32.
        dict(name="attention_backward_ragged_f32", kind="attention_backward", dtype="f32", B=3, n=197, nk=99, h=3, hk=1, d=64, causal=True,
             cap=30.0, slopes=False, docs=0, prefix=64, pad=0),
        # The packed batch again, in the backward pass of a step that keeps half the tokens.
        dict(name="attention_backward_packed", kind="attention_backward", dtype="bf16", B=4, n=2048, nk=1024, h=12, hk=12, d=64, causal=True,
             cap=0.0, slopes=True, docs=500, prefix=0, pad=300),
        # The long text's backward on 4096 kept tokens: the largest call.
        dict(name="attention_backward_long", kind="attention_backward", dtype="bf16", B=1, n=8192, nk=4096, h=16, hk=2, d=128, causal=True,
             cap=50.0, slopes=False, docs=0, prefix=0, pad=0),
        # The norms between two blocks for 64 tokens: a short request.
        dict(name="norms_short", kind="norms", dtype="bf16", M=64, C=768, layer=True, post=True, pre=True, beta=True, gate=1, alpha=1.0),
        # 16384 tokens of a wide model, root-mean-square norms on both sides of the block, a gate per channel: streaming.
        dict(name="norms_wide", kind="norms", dtype="bf16", M=16384, C=4096, layer=False, post=True, pre=True, beta=False, gate=1, alpha=1.0),
        # Channels that fill no vector, layer norms with shifts, a gate of its own for each of four samples, fp32.
        dict(name="norms_backward_ragged_f32", kind="norms_backward", dtype="f32", M=788, K=396, C=771, layer=True, post=True, pre=True,
             beta=True, gate=4, alpha=0.8),
        # The wide model's backward with half the rows kept.
        dict(name="norms_backward_wide", kind="norms_backward", dtype="bf16", M=16384, K=8192, C=4096, layer=False, post=True, pre=True,
             beta=False, gate=1, alpha=1.0),
        # A small fp32 table, half of 394 tokens kept.
        dict(name="embedding_small_f32", kind="embedding", dtype="f32", M=394, K=198, V=1000, C=200, scale=14.0),
        # 32768 tokens of a table of 50000 words of 2048 channels, half of them kept.
        dict(name="embedding_large", kind="embedding", dtype="bf16", M=32768, K=16384, V=50000, C=2048, scale=45.25),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["attention", "attention_backward", "attention", "attention_backward", "norms", "norms_backward", "embedding"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if kind.startswith("attention"):
        d = rng.choice([16, 32, 64, 64, 128, 128])
        hk = rng.choice([1, 2, 3, 4, 8])
        h = hk * rng.choice([1, 1, 2, 4] if hk <= 4 else [1, 2])
        n = _log(rng, 1, 2048 if dtype == "f32" or d == 16 else 8192)
        most = (1 << 30 if dtype == "bf16" and d > 16 else 1 << 27) // (h * n * n)
        if most < 1:
            n = 2048
            most = max(1, (1 << 27) // (h * n * n))
        B = _log(rng, 1, min(64, most))
        nk = min(n, max(1, int(n * rng.uniform(0.25, 1.0))))
        causal = rng.random() < 0.7
        case = dict(kind=kind, dtype=dtype, B=B, n=n, h=h, hk=hk, d=d, causal=causal, cap=rng.choice([0.0, 20.0, 30.0, 50.0]),
                    slopes=rng.random() < 0.4, docs=rng.choice([0, 0, max(1, n // 5), 300]),
                    prefix=rng.randrange(0, n + 1) if causal and rng.random() < 0.4 else 0, pad=rng.choice([0, n // 4]))
        if kind == "attention_backward":
            case["nk"] = nk
        return case
    if kind.startswith("norms"):
        C = _log(rng, 8, 8192)
        M = _log(rng, 1, min(65536, 67000000 // C))
        gate = rng.choice([0, 1, 1, rng.choice([2, 3, 5])])
        M = max(1, M // max(gate, 1)) * max(gate, 1)
        case = dict(kind=kind, dtype=dtype, M=M, C=C, layer=rng.random() < 0.5, post=rng.random() < 0.7, pre=rng.random() < 0.9,
                    beta=rng.random() < 0.5, gate=gate, alpha=rng.choice([1.0, 1.0, 0.5, 0.8]))
        if kind == "norms_backward":
            per = M // max(gate, 1)
            case["K"] = max(1, int(per * rng.uniform(0.25, 1.0))) * max(gate, 1)
        return case
    C = _log(rng, 8, 4096)
    M = _log(rng, 1, min(65536, 67000000 // C))
    return dict(kind=kind, dtype=dtype, M=M, K=max(1, int(M * rng.uniform(0.25, 1.0))), V=_log(rng, 10, min(128000, 100000000 // C)), C=C,
                scale=round(math.sqrt(C), 3))


def _documents(case):
    """Per sample the lengths of the documents in a row; they follow from the case alone."""
    rng = random.Random(case["n"] * 1000003 + case["docs"] * 1009 + case["B"])
    rows = []
    for b in range(case["B"]):
        left = case["n"] - (case["pad"] if b == case["B"] - 1 else 0)          # the last sample is the padded one
        row = []
        while left > 0:
            row.append(min(left, rng.randint(1, 2 * case["docs"] - 1) if case["docs"] else left))
            left -= row[-1]
        rows.append(row)
    return rows


def _prefixes(case):
    return [case["prefix"] * (b + 1) // case["B"] for b in range(case["B"])]


def _visible_pairs(case):
    total = 0
    for row, p in zip(_documents(case), _prefixes(case)):
        at = 0
        for length in row:
            seen = max(0, min(at + length, p) - at) if case["causal"] else 0
            total += (length * (length + 1) + seen * (seen - 1)) // 2 if case["causal"] else length * length
            at += length
    return total


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    kind, dt = case["kind"], DT[case["dtype"]]

    def randn(*shape, dtype=dt):
        return torch.randn(*shape, generator=g, device="cuda").to(dtype)

    def kept(groups, rows, k):
        """[groups * k] ascending row numbers, k of each group of `rows`, and their inverse map."""
        pick = torch.rand(groups, rows, generator=g, device="cuda").argsort(dim=1)[:, :k].sort(dim=1).values
        idx = (pick + rows * torch.arange(groups, device="cuda")[:, None]).reshape(-1)
        inv = torch.full((groups * rows,), -1, dtype=torch.int32, device="cuda")
        inv[idx] = torch.arange(idx.numel(), dtype=torch.int32, device="cuda")
        return idx.to(torch.int32), inv

    st = dict(case=case)
    if kind.startswith("attention"):
        B, n, h, hk, d = (case[k] for k in ("B", "n", "h", "hk", "d"))
        st["qkv"] = randn(B * n, (h + 2 * hk) * d)
        st["slopes"] = torch.tensor([2.0 ** (-8.0 * (i + 1) / h) for i in range(h)], device="cuda") if case["slopes"] else None
        st["prefix"] = torch.tensor(_prefixes(case), dtype=torch.int32, device="cuda") if case["prefix"] else None
        st["doc"] = None
        if case["docs"] or case["pad"]:
            ids = [[i for i, length in enumerate(row) for _ in range(length)] for row in _documents(case)]
            st["doc"] = torch.tensor([v for row in ids for v in row + [-1] * (n - len(row))], dtype=torch.int32, device="cuda")
        if kind == "attention_backward":
            A, lse = _attention(st)
            idx, _ = kept(B, n, case["nk"])
            rows = idx.long()
            st.update(idx=idx, qkv_k=st["qkv"][rows], A_k=A[rows], lse_k=lse[rows], dA_k=randn(B * case["nk"], h * d))
            del st["qkv"]
    elif kind.startswith("norms"):
        M, C = case["M"], case["C"]
        G = max(case["gate"], 1)

        def vector(wanted, mean, *shape):
            return mean + 0.1 * torch.randn(*shape, C, generator=g, device="cuda") if wanted else None

        st.update(gate=vector(case["gate"], 0.5, G), gamma_post=vector(case["post"], 1.0), gamma_pre=vector(case["pre"], 1.0),
                  beta_post=vector(case["post"] and case["beta"], 0.0), beta_pre=vector(case["pre"] and case["beta"], 0.0))
        if kind == "norms":
            st.update(x=randn(M, C), y=randn(M, C))
        else:
            st["idx"], st["inv"] = kept(G, M // G, case["K"] // G)
            st.update(dx_out=randn(M, C), y_k=randn(case["K"], C), x_out_k=randn(case["K"], C) if case["pre"] else None,
                      dz_k=randn(case["K"], C) if case["pre"] else None)
    else:
        M, K, V, C = (case[k] for k in ("M", "K", "V", "C"))
        rank = torch.rand(M, generator=g, device="cuda", dtype=torch.float64).mul(math.log(V + 1.0)).exp().sub(1.0).long().clamp(0, V - 1)
        names = torch.randperm(V, generator=g, device="cuda")                  # which word has which rank
        st["tokens"] = names[rank]
        st["idx"], _ = kept(1, M, K)
        st.update(table=(0.02 * torch.randn(V, C, generator=g, device="cuda")).to(dt), dE_k=randn(K, C))
    return st


# ---- plain forms: elementary operations, fp32 ----------------------------------------------------------------------

def _groups(B, cells):
    """Runs of samples whose score matrices together stay at 2^30 elements."""
    step = max(1, (1 << 30) // cells)
    return [(b, min(B, b + step)) for b in range(0, B, step)]


def _heads(x, B, rows, h, d, repeat=1):
    return x.float().view(B, rows, h, d).transpose(1, 2).repeat_interleave(repeat, dim=1)


def _scores(case, st, q, k, pos, doc, b0, b1):
    """(scores with the cap and the bias, visible, the cap's slope) for positions [samples, tokens]."""
    s = torch.matmul(q, k.transpose(2, 3).contiguous()) * (case["d"] ** -0.5)
    slope = None
    if case["cap"]:
        t = torch.tanh(s / case["cap"])
        s, slope = case["cap"] * t, 1.0 - t * t
    i, j = pos[:, :, None], pos[:, None, :]
    visible = torch.ones_like(i == j)
    if case["causal"]:
        visible = j <= i
        if st["prefix"] is not None:
            visible = visible | (j < st["prefix"][b0:b1, None, None])
    if doc is not None:
        visible = visible & (doc[:, :, None] == doc[:, None, :]) & (doc[:, None, :] >= 0)
    if st["slopes"] is not None:
        s = s - st["slopes"][None, :, None, None] * (i - j).abs()[:, None].float()
    return s, visible[:, None], slope


def _attention(st):
    c = st["case"]
    B, n, h, hk, d = (c[k] for k in ("B", "n", "h", "hk", "d"))
    A = torch.empty(B * n, h * d, dtype=st["qkv"].dtype, device="cuda")
    lse = torch.empty(B * n, h, device="cuda")
    pos = torch.arange(n, device="cuda")[None]
    for b0, b1 in _groups(B, h * n * n):
        x = st["qkv"][b0 * n:b1 * n]
        q, k, v = x.split([h * d, hk * d, hk * d], dim=1)
        q = _heads(q, b1 - b0, n, h, d)
        k, v = (_heads(t, b1 - b0, n, hk, d, h // hk) for t in (k, v))
        doc = None if st["doc"] is None else st["doc"].view(B, n)[b0:b1]
        s, visible, _ = _scores(c, st, q, k, pos.expand(b1 - b0, n), doc, b0, b1)
        s = torch.where(visible, s, -math.inf)
        m = s.amax(dim=3, keepdim=True)
        e = torch.exp(s - torch.where(m == -math.inf, 0.0, m))
        total = e.sum(dim=3, keepdim=True)
        out = torch.matmul(e, v) / torch.where(total == 0, 1.0, total)
        A[b0 * n:b1 * n] = out.transpose(1, 2).reshape(-1, h * d).to(A.dtype)
        lse[b0 * n:b1 * n] = (m + torch.log(total))[..., 0].transpose(1, 2).reshape(-1, h)
    return A, lse


def _attention_backward(st):
    c = st["case"]
    B, n, nk, h, hk, d = (c[k] for k in ("B", "n", "nk", "h", "hk", "d"))
    out = torch.empty_like(st["qkv_k"])
    rows = st["idx"].long().view(B, nk)
    pos = rows - n * torch.arange(B, device="cuda")[:, None]
    docs = None if st["doc"] is None else st["doc"][rows]
    for b0, b1 in _groups(B, h * nk * nk):
        m, at = b1 - b0, slice(b0 * nk, b1 * nk)
        q, k, v = st["qkv_k"][at].split([h * d, hk * d, hk * d], dim=1)
        q = _heads(q, m, nk, h, d)
        k, v = (_heads(t, m, nk, hk, d, h // hk) for t in (k, v))
        a, g = (_heads(st[t][at], m, nk, h, d) for t in ("A_k", "dA_k"))
        lse = st["lse_k"][at].view(m, nk, h).transpose(1, 2)[..., None]
        s, visible, slope = _scores(c, st, q, k, pos[b0:b1], None if docs is None else docs[b0:b1], b0, b1)
        p = torch.where(visible, torch.exp(torch.where(visible, s - lse, 0.0)), 0.0)
        ds = p * (torch.matmul(g, v.transpose(2, 3).contiguous()) - (g * a).sum(dim=3, keepdim=True)) * (d ** -0.5)
        if slope is not None:
            ds = ds * slope
        dq = torch.matmul(ds, k)
        dk = torch.matmul(ds.transpose(2, 3).contiguous(), q).view(m, hk, h // hk, nk, d).sum(dim=2)
        dv = torch.matmul(p.transpose(2, 3).contiguous(), g).view(m, hk, h // hk, nk, d).sum(dim=2)
        out[at] = torch.cat([t.transpose(1, 2).reshape(m * nk, -1) for t in (dq, dk, dv)], dim=1).to(out.dtype)
    return out


def _normalised(x, layer):
    """(normalised rows, 1 / deviation)."""
    if layer:
        x = x - x.mean(dim=1, keepdim=True)
    r = torch.rsqrt((x * x).mean(dim=1, keepdim=True) + EPS)
    return x * r, r


def _norm(x, gamma, beta, layer):
    out = _normalised(x, layer)[0] * gamma
    return out if beta is None else out + beta


def _norm_backward(g, hat, r, layer):
    """The input gradient for g = output gradient * gamma."""
    out = g - hat * (g * hat).mean(dim=1, keepdim=True)
    if layer:
        out = out - g.mean(dim=1, keepdim=True)
    return out * r


def _spread(gate, rows):
    return gate.repeat_interleave(rows // gate.shape[0], dim=0)


def _norms(st):
    c = st["case"]
    u = st["y"].float()
    if c["post"]:
        u = _norm(u, st["gamma_post"], st["beta_post"], c["layer"])
    if c["gate"]:
        u = u * _spread(st["gate"], c["M"])
    x = c["alpha"] * st["x"].float() + u
    out = [x.to(st["x"].dtype)]
    if c["pre"]:
        out.append(_norm(x, st["gamma_pre"], st["beta_pre"], c["layer"]).to(st["x"].dtype))
    return out


def _norms_backward(st):
    c = st["case"]
    dt, rows = st["y_k"].dtype, st["idx"].long()
    dx = c["alpha"] * st["dx_out"].float()
    t = st["dx_out"][rows].float()
    out = {}
    if c["pre"]:
        dz = st["dz_k"].float()
        hat, r = _normalised(st["x_out_k"].float(), c["layer"])
        t = t + _norm_backward(dz * st["gamma_pre"], hat, r, c["layer"])
        out["dgamma_pre"] = (dz * hat).sum(dim=0)
        if c["beta"]:
            out["dbeta_pre"] = dz.sum(dim=0)
    dx[rows] = c["alpha"] * t
    out["dx"] = dx.to(dt)
    y = st["y_k"].float()
    hat, r = _normalised(y, c["layer"]) if c["post"] else (y, None)
    if c["gate"]:
        u = hat
        if c["post"]:
            u = hat * st["gamma_post"]
            u = u if st["beta_post"] is None else u + st["beta_post"]
        out["dgate"] = (t * u).view(c["gate"], -1, c["C"]).sum(dim=1)
        t = t * _spread(st["gate"], c["K"])
    if c["post"]:
        out["dgamma_post"] = (t * hat).sum(dim=0)
        if c["beta"]:
            out["dbeta_post"] = t.sum(dim=0)
        t = _norm_backward(t * st["gamma_post"], hat, r, c["layer"])
    out["dy_k"] = t.to(dt)
    return {k: out[k] for k in sorted(out)}


def _embedding(st):
    c = st["case"]
    E = (st["table"][st["tokens"]].float() * c["scale"]).to(st["table"].dtype)
    grad = torch.zeros(c["V"], c["C"], device="cuda")
    grad.index_add_(0, st["tokens"][st["idx"].long()], st["dE_k"].float())
    return E, grad.mul_(c["scale"])


PLAIN = {"attention": _attention, "attention_backward": _attention_backward, "norms": _norms, "norms_backward": _norms_backward,
         "embedding": _embedding}


# ---- the library's calls -------------------------------------------------------------------------------------------

def _library(st):
    import paper_2210_00129_amd as sbp
    c = st["case"]
    if c["kind"].startswith("attention"):
        kw = dict(B=c["B"], h=c["h"], d=c["d"], scale=c["d"] ** -0.5, h_kv=c["hk"], cap=c["cap"], causal=c["causal"], slopes=st["slopes"],
                  doc=st["doc"], prefix=st["prefix"])
        if c["kind"] == "attention":
            return sbp.forward_attention_masked(st["qkv"], **kw)
        return sbp.backward_attention_masked(st["qkv_k"], st["A_k"], st["dA_k"], st["lse_k"], n=c["n"], idx=st["idx"], **kw)
    if c["kind"].startswith("norms"):
        kw = dict(gate=st["gate"], alpha=c["alpha"], gamma_post=st["gamma_post"], beta_post=st["beta_post"], gamma_pre=st["gamma_pre"],
                  kind=sbp.NORM_LAYER if c["layer"] else sbp.NORM_RMS, eps=EPS)
        if c["kind"] == "norms":
            x_out, z = sbp.forward_residual_norm(st["x"], st["y"], beta_pre=st["beta_pre"], **kw)
            return [x_out, z] if c["pre"] else [x_out]
        wanted = ["dx", "dy_k"] + ["dgate"] * bool(c["gate"])
        for side in ("post", "pre"):
            wanted += ["dgamma_" + side] * c[side] + ["dbeta_" + side] * (c[side] and c["beta"])
        got = sbp.backward_residual_norm(st["dx_out"], st["dz_k"], st["x_out_k"], st["y_k"], st["idx"], c["M"], inv=st["inv"],
                                         want=wanted, **kw)
        return {k: got[k] for k in sorted(wanted)}
    return (sbp.forward_embedding(st["tokens"], st["table"], c["scale"]),
            sbp.backward_embedding(st["dE_k"], st["tokens"], c["V"], idx=st["idx"], scale=c["scale"], flags=sbp.FLAG_DY_COMPACT))


def run(state):
    if own:
        return _library(state)
    return PLAIN[state["case"]["kind"]](state)


def work(case):
    """Every input read once, every output written once; products of the visible pairs only."""
    size = 4 if case["dtype"] == "f32" else 2
    if case["kind"].startswith("attention"):
        B, n, h, hk, d = (case[k] for k in ("B", "n", "h", "hk", "d"))
        pairs = _visible_pairs(case) * h
        if case["kind"] == "attention":
            return dict(bytes=B * n * ((2 * h + 2 * hk) * d * size + 4 * h), flops=4 * d * pairs)
        share = (case["nk"] / n) ** 2
        return dict(bytes=B * case["nk"] * ((2 * (h + 2 * hk) + 2 * h) * d * size + 4 * h), flops=10 * d * pairs * share)
    if case["kind"] == "norms":
        return dict(bytes=case["M"] * case["C"] * size * (4 if case["pre"] else 3), flops=12 * case["M"] * case["C"])
    if case["kind"] == "norms_backward":
        M, K, C = case["M"], case["K"], case["C"]
        return dict(bytes=(2 * M + (4 if case["pre"] else 2) * K) * C * size, flops=30 * K * C + M * C)
    M, K, V, C = (case[k] for k in ("M", "K", "V", "C"))
    return dict(bytes=(M + min(M, V) + K) * C * size + 4 * V * C + 8 * M + 4 * K, flops=M * C + K * C)


# ---- from the definitions, in 64 bits ------------------------------------------------------------------------------

def _exact_attention(st):
    """Row by row of the definition: weights exp(score) over the visible keys, divided by their sum."""
    c = st["case"]
    B, n, h, hk, d = (c[k] for k in ("B", "n", "h", "hk", "d"))
    back = c["kind"] == "attention_backward"
    rows = st["idx"].long().reshape(B, -1) if back else torch.arange(B * n, device="cuda").reshape(B, n)
    m = rows.shape[1]
    x = st["qkv_k" if back else "qkv"].double().reshape(B, m, h + 2 * hk, d)
    out = torch.zeros_like(x) if back else torch.zeros(B, m, h, d, dtype=torch.float64, device="cuda")
    lse = torch.full((B, m, h), -math.inf, dtype=torch.float64, device="cuda")
    for b in range(B):
        t = rows[b] - b * n
        later = t.reshape(1, m) - t.reshape(m, 1)                 # key position less query position
        hidden = torch.zeros(m, m, dtype=torch.bool, device="cuda")
        if c["causal"]:
            hidden |= (later > 0) & (t.reshape(1, m) >= (0 if st["prefix"] is None else int(st["prefix"][b])))
        if st["doc"] is not None:
            names = st["doc"][rows[b]].long()
            hidden |= (names.reshape(1, m) - names.reshape(m, 1) != 0) | (names < 0).reshape(m, 1)
        for a in range(h):
            q, k, v = x[b, :, a], x[b, :, h + a * hk // h], x[b, :, h + hk + a * hk // h]
            z = q.matmul(k.t().contiguous()) / math.sqrt(d)
            w = c["cap"] * torch.tanh(z / c["cap"]) if c["cap"] else z
            if st["slopes"] is not None:
                w = w - float(st["slopes"][a]) * later.abs()
            w = w.masked_fill(hidden, -math.inf)
            if not back:
                lse[b, :, a] = torch.logsumexp(w, dim=1)
                out[b, :, a] = torch.softmax(w, dim=1).nan_to_num(0.0).matmul(v)
                continue
            own_lse = st["lse_k"].reshape(B, m, h)[b, :, a].double().reshape(m, 1)
            weight = (w - own_lse).exp().masked_fill(hidden, 0.0)
            g, o = (st[name].reshape(B, m, h, d)[b, :, a].double() for name in ("dA_k", "A_k"))
            dz = weight * (g.matmul(v.t().contiguous()) - (g * o).sum(dim=1, keepdim=True))
            if c["cap"]:
                dz = dz / torch.cosh(z / c["cap"]) ** 2
            out[b, :, a] = dz.matmul(k) / math.sqrt(d)
            out[b, :, h + a * hk // h] += dz.t().contiguous().matmul(q) / math.sqrt(d)
            out[b, :, h + hk + a * hk // h] += weight.t().contiguous().matmul(g)
    return out.reshape(B * m, -1) if back else (out.reshape(B * m, -1), lse.reshape(B * m, h))


def _exact_norms(st):
    c = st["case"]
    back = c["kind"] == "norms_backward"
    wide = {k: v.double() for k, v in st.items() if torch.is_tensor(v) and v.is_floating_point()}

    def norm(x, gamma, beta):
        mean = x.mean(dim=1, keepdim=True) if c["layer"] else torch.zeros_like(x[:, :1])
        y = (x - mean) / torch.sqrt(((x - mean) ** 2).mean(dim=1, keepdim=True) + EPS) * gamma
        return y if beta is None else y + beta

    if not back:
        branch = norm(wide["y"], wide["gamma_post"], wide.get("beta_post")) if c["post"] else wide["y"]
        if c["gate"]:
            branch = (branch.reshape(c["gate"], -1, c["C"]) * wide["gate"].reshape(c["gate"], 1, c["C"])).reshape(c["M"], c["C"])
        x = wide["x"] * c["alpha"] + branch
        return [x, norm(x, wide["gamma_pre"], wide.get("beta_pre"))] if c["pre"] else [x]
    # the gradients by differentiation of the forward's definition
    rows = st["idx"].long()
    leaf = {k: wide[k].requires_grad_() for k in ("gate", "gamma_post", "beta_post", "gamma_pre", "beta_pre", "y_k", "x_out_k") if k in wide}
    at_x = wide["dx_out"][rows]
    out = {}
    if c["pre"]:
        names = [k for k in ("x_out_k", "gamma_pre", "beta_pre") if k in leaf]
        got = torch.autograd.grad(norm(leaf["x_out_k"], leaf["gamma_pre"], leaf.get("beta_pre")), [leaf[k] for k in names], wide["dz_k"])
        out.update({"d" + k: v for k, v in zip(names[1:], got[1:])})
        at_x = at_x + got[0]
    branch = norm(leaf["y_k"], leaf["gamma_post"], leaf.get("beta_post")) if c["post"] else leaf["y_k"] * 1.0
    if c["gate"]:
        branch = (branch.reshape(c["gate"], -1, c["C"]) * leaf["gate"].reshape(c["gate"], 1, c["C"])).reshape(c["K"], c["C"])
    names = [k for k in ("gate", "gamma_post", "beta_post", "y_k") if k in leaf and (c["post"] or "post" not in k)]
    out.update({"d" + k: v for k, v in zip(names, torch.autograd.grad(branch, [leaf[k] for k in names], at_x))})
    dx = wide["dx_out"] * c["alpha"]
    dx[rows] = at_x * c["alpha"]
    out["dx"] = dx
    return {k: out[k] for k in sorted(out)}


def _exact_embedding(st):
    c = st["case"]
    words = st["table"].double() * c["scale"]
    order = st["tokens"][st["idx"].long()].sort(stable=True)
    grad = torch.zeros(c["V"], c["C"], dtype=torch.float64, device="cuda")
    grad.index_add_(0, order.values, st["dE_k"].double()[order.indices] * c["scale"])
    return words.index_select(0, st["tokens"]), grad


def exact(case, seed):
    st = prepare(case, seed)
    return (_exact_attention if case["kind"].startswith("attention") else _exact_norms if case["kind"].startswith("norms") else _exact_embedding)(st)
