"""What is measured of the operators on compact targets: verification against given
probabilities, the top logits of target rows, and distillation from them.

``listed()`` names representative calls, ``draw(rng)`` gives more of the same ranges,
``prepare`` makes a call's inputs on the GPU with what a program keeps beside them,
``run`` makes one call: plain torch where ``own`` is false, this package's functions
where it is true.  ``exact`` computes the result from the definitions in 64 bits.
"""
from __future__ import annotations

import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
MOST_ROWS = 16384 * 32000  # entries of the largest listed distillation; drawn cases stay below it


def _verify(name, B, k, V, dtype, draft=True, ragged=False, accept=0.6, minp=0.0, fresh=False):
    return {"name": name, "op": "verify", "B": B, "k": k, "V": V, "dtype": dtype, "draft": draft, "ragged": ragged,
            "accept": accept, "minp": minp, "fresh": fresh}


def _topk(name, G, P, V, dtype, K, active=1.0, rest=True, tau=1.0, fresh=False):
    return {"name": name, "op": "topk", "G": G, "P": P, "V": V, "dtype": dtype, "K": K, "active": active, "rest": rest,
            "tau": tau, "fresh": fresh}


def _distill(name, N, V, dtype, K, kind, beta=0.5, tau=1.0, active=1.0, rest=True, fresh=False):
    return {"name": name, "op": "distill", "N": N, "V": V, "dtype": dtype, "K": K, "kind": kind, "beta": beta, "tau": tau,
            "active": active, "rest": rest, "fresh": fresh}


def listed():
    return [
        # One decoding step of a few sequences, probabilities straight from a softmax: latency.
        _verify("probs_tiny", 4, 4, 32000, "f32", fresh=True),
        # An ordinary serving batch whose sequences carry 0 to 5 drafts, the target's rows filtered by min-p.
        _verify("probs_serving", 32, 5, 32000, "f32", ragged=True, minp=0.02),
        # Drafts looked up in the prompt, which have no distribution; one token added to the vocabulary.
        _verify("probs_lookup", 64, 3, 32001, "bf16", draft=False, accept=0.5),
        # A large batch with a 128k vocabulary.
        _verify("probs_large", 256, 8, 128256, "f32", accept=0.7),
        # The one row a sequence that a serving step rejected, picked by the mismatch mask: latency.
        _topk("topk_step", 32, 5, 32000, "bf16", 64, active=0.2, fresh=True),
        # A stretch of target rows kept for the replay buffer.
        _topk("topk_buffer", 4096, 1, 32000, "bf16", 64),
        # Rows of a 128k vocabulary in fp32, many entries kept, positions strided in [B, k+1, V].
        _topk("topk_wide", 256, 4, 128256, "f32", 256, tau=0.7),
        # Distillation of the few rows of one small step.
        _distill("distill_step", 16, 32000, "f32", 32, "fkl", fresh=True),
        # A buffer flush from kept rows: the bulk of the training side's time.
        _distill("distill_flush", 16384, 32000, "bf16", 64, "rkl"),
        # The same for a buffer of which 40 % of the positions count, at an odd vocabulary.
        _distill("distill_odd", 8192, 32001, "bf16", 100, "jsd", active=0.4),
        # A 128k vocabulary and a teacher cut to its top entries (no mass elsewhere).
        _distill("distill_wide", 2048, 128256, "bf16", 256, "fkl", tau=2.0, rest=False),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _vocab(rng):
    v = _log_int(rng, 4000, 160000)
    how = rng.random()
    if how < 0.6:
        return max(64, v // 64 * 64)  # padded, as most models are
    if how < 0.75:
        return max(4, v // 4 * 4)
    return v


def draw(rng):
    op = rng.choice(["verify", "topk", "distill"])
    V, dtype = _vocab(rng), rng.choice(["bf16", "f32"])
    if op == "verify":
        c = _verify("", _log_int(rng, 1, 256), rng.randint(1, 8), min(V, 128256), dtype, rng.random() < 0.75,
                    rng.random() < 0.4, round(rng.uniform(0.2, 0.95), 2), rng.choice([0.0, 0.0, 0.02]), rng.random() < 0.5)
    elif op == "topk":
        P = rng.choice([1, 1, 3, 5])
        most = max(1, min(8192, MOST_ROWS // 4 // (V * P)))
        c = _topk("", _log_int(rng, 1, most), P, V, dtype, _log_int(rng, 1, 512), rng.choice([1.0, 1.0, 0.3]),
                  rng.random() < 0.85, rng.choice([1.0, 1.0, 0.7, 2.0]), rng.random() < 0.5)
    else:
        # (not TVD, whose gradient jumps where p = q: the side taken there is a matter of rounding)
        kind = rng.choice(["fkl", "rkl", "jsd", "ce"])
        most = max(1, min(16384, MOST_ROWS // V // (2 if dtype == "f32" else 1)))
        c = _distill("", _log_int(rng, 1, most), V, dtype, _log_int(rng, 1, 512), kind, rng.choice([0.1, 0.5, 0.9]),
                     rng.choice([1.0, 1.0, 0.7, 2.0]), rng.choice([1.0, 1.0, 0.4]), kind == "rkl" or rng.random() < 0.7,
                     rng.random() < 0.3)
    c.pop("name", None)
    return c


# ------------------------------------------------------------------ inputs
def _normal(shape, std, g, dtype, base=None):
    """N(0, std^2), plus base, rounded to dtype; made in pieces to bound the fp32 temporaries."""
    out = torch.empty(shape, dtype=dtype, device="cuda")
    flat = out.view(-1, shape[-1])
    rows = max(1, (1 << 27) // shape[-1])
    for r in range(0, flat.shape[0], rows):
        x = torch.empty(flat[r:r + rows].shape, device="cuda").normal_(0.0, std, generator=g)
        if base is not None:
            x.add_(base.view(-1, shape[-1])[r:r + rows].float())
        flat[r:r + rows] = x
    return out


def _mask(n, active, g):
    mask = torch.zeros(n, dtype=torch.uint8, device="cuda")
    mask[torch.randperm(n, generator=g, device="cuda")[:max(1, round(active * n))]] = 1
    return mask


def _prepare_verify(s, g):
    B, k, V, dt = s["B"], s["k"], s["V"], DTYPES[s["dtype"]]
    target = torch.empty(B, k + 1, V, dtype=dt, device="cuda")
    draft = torch.empty(B, k, V, dtype=dt, device="cuda") if s["draft"] else None
    tokens = torch.zeros(B, k, dtype=torch.int32, device="cuda")
    for i in range(k + 1):  # the target agrees with the draft on a share of the mass
        q = torch.softmax(torch.empty(B, V, device="cuda").normal_(0.0, 2.5, generator=g), -1)
        p = torch.softmax(torch.empty(B, V, device="cuda").normal_(0.0, 2.5, generator=g), -1)
        p.mul_(1 - s["accept"])
        if i < k:
            tokens[:, i] = torch.multinomial(q, 1, generator=g)[:, 0].int()
            if draft is not None:
                draft[:, i] = q
        if i < k and draft is None:  # a lookup proposes what the target may well hold likely
            p.scatter_add_(1, tokens[:, i:i + 1].long(), torch.full((B, 1), s["accept"], device="cuda"))
        else:
            p.add_(q, alpha=s["accept"])
        if s["minp"]:
            p = torch.where(p >= s["minp"] * p.amax(-1, keepdim=True), p, 0.0)
            p /= p.sum(-1, keepdim=True)
        target[:, i] = p
    s["draft_probs"], s["target_probs"], s["tokens"], s["lens"] = draft, target, tokens, None
    s["u"] = torch.rand(B, k + 1, generator=g, device="cuda")
    if s["ragged"]:
        s["lens"] = torch.randint(0, k + 1, (B,), generator=g, device="cuda", dtype=torch.int32)
        tokens.masked_fill_(torch.arange(k, device="cuda") >= s["lens"][:, None], -1)
    s["out"] = None
    if not s["fresh"]:  # the server's own buffers
        i32 = {"dtype": torch.int32, "device": "cuda"}
        s["out"] = (torch.zeros(B, **i32), torch.zeros(B, k + 1, **i32), torch.zeros(B, k, dtype=torch.uint8, device="cuda"),
                    None, None)


def _top_of(t, K, tau, rest):
    """The K largest logits of each row, their ids, and the log of the other entries' mass."""
    values, ids = torch.empty(t.shape[0], K, device="cuda"), torch.empty(t.shape[0], K, dtype=torch.int32, device="cuda")
    other = torch.empty(t.shape[0], device="cuda") if rest else None
    step = max(1, (1 << 27) // t.shape[1])
    for r in range(0, t.shape[0], step):
        x = t[r:r + step].float()
        v, i = torch.topk(x, K)
        values[r:r + step], ids[r:r + step] = v, i.int()
        if rest:
            other[r:r + step] = torch.logsumexp(x.scatter_(1, i, -math.inf) / tau, -1)
    return values, ids, other


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    s, V, dt = dict(case), case["V"], DTYPES[case["dtype"]]
    if case["op"] == "verify":
        _prepare_verify(s, g)
    elif case["op"] == "topk":
        G, P, K = case["G"], case["P"], min(case["K"], V)
        # one row a group beyond those taken, as a [B, k+1, V] tensor has, where P > 1
        whole = _normal((G, P + (P > 1), V), 2.5, g, dt)
        s["logits"], s["mask"] = whole[:, :P], None
        if case["active"] < 1.0:
            s["mask"] = _mask(G * P, case["active"], g).view(G, P)
        # the buffer the rows go to: positions that do not count keep what it holds there
        s["out"] = (torch.zeros(G, P, K, device="cuda"), torch.zeros(G, P, K, dtype=torch.int32, device="cuda"),
                    torch.zeros(G, P, device="cuda") if case["rest"] else None)
    else:
        N, K = case["N"], min(case["K"], V)
        s["draft"] = _normal((N, V), 2.0, g, dt)
        s["top"] = _top_of(_normal((N, V), 1.5, g, dt, s["draft"]), K, case["tau"], case["rest"])
        s["mask"] = _mask(N, case["active"], g) if case["active"] < 1.0 else None
        # the trainer's gradient buffer: inactive rows keep the zeros it put there
        s["loss"], s["dlogits"] = None, None
        if not case["fresh"] or s["mask"] is not None:
            s["loss"], s["dlogits"] = torch.zeros(N, device="cuda"), torch.zeros(N, V, device="cuda")
    return s


# ------------------------------------------------------------------ one pass
def _plain_verify(s):
    p, q, y, u = s["target_probs"], s["draft_probs"], s["tokens"].long(), s["u"]
    B, k1, V = p.shape
    k = k1 - 1
    lens = s["lens"].long() if s["lens"] is not None else torch.full((B,), k, device=p.device)
    at = torch.arange(k, device=p.device)
    live = at < lens[:, None]
    yy = torch.where(live, y, 0)
    py = p[:, :k].gather(2, yy[:, :, None])[:, :, 0].double()
    qy = q.gather(2, yy[:, :, None])[:, :, 0].double() if q is not None else torch.ones_like(py)
    fails = live & ~(u[:, :k].double() * qy < py)  # the product of two fp32 numbers is exact in 64 bits
    a = torch.where(fails, at, lens[:, None]).amin(1)
    rows = torch.arange(B, device=p.device)
    w = p[rows, a].double()  # sums of many weights decide a token: 64 bits
    first_p = _first_max(w)
    rejects = a < lens
    ai = a.clamp(max=k - 1)
    if q is not None:
        w = (w - torch.where(rejects[:, None], q[rows, ai].double(), 0.0)).clamp_(min=0.0)
    else:
        less = torch.zeros_like(w).scatter_(1, yy[rows, ai][:, None], rejects[:, None].double())
        w = (w - less).clamp_(min=0.0)
    C = torch.cumsum(w, 1)
    W = C[:, -1:]
    past = C > u[:, k:].double() * W
    last = V - 1 - _first_max((w > 0).flip(1).int())
    token = torch.where(past.any(1), _first_max(past.int()), last)
    token = torch.where(W[:, 0] > 0, token, first_p)
    pos = torch.arange(k1, device=p.device)
    out = torch.where(pos < a[:, None], torch.cat([yy, yy[:, :1]], 1), torch.where(pos == a[:, None], token[:, None], -1))
    return a.int(), out.int(), ((at == a[:, None]) & rejects[:, None]).to(torch.uint8)


def _first_max(x):
    """The lowest index of the maximum of each row."""
    top = x == x.amax(-1, keepdim=True)
    return torch.where(top, torch.arange(x.shape[-1], device=x.device), x.shape[-1]).amin(-1)


def _plain_topk(s):
    x, K = s["logits"], min(s["K"], s["V"])
    G, P, V = x.shape
    flat = x.reshape(G * P, V)
    rows = None
    if s["mask"] is not None:
        rows = s["mask"].view(-1).nonzero()[:, 0]
        flat = flat[rows]
    v, i = torch.sort(flat.float(), dim=1, descending=True, stable=True)
    outs = [v[:, :K], i[:, :K].int()]
    if s["rest"]:
        o = v[:, K:] / s["tau"]
        if K < V:
            m = o[:, :1]
            outs.append(m[:, 0] + torch.log(torch.exp(o - m).sum(1)))
        else:
            outs.append(torch.full((flat.shape[0],), -math.inf, device=x.device))
    full = []
    for o in outs:
        if rows is not None:
            whole = torch.zeros((G * P,) + o.shape[1:], dtype=o.dtype, device=o.device)
            whole[rows] = o
            o = whole
        full.append(o.reshape((G, P) + o.shape[1:]))
    return tuple(full) + ((None,) if not s["rest"] else ())


def _plain_distill(s):
    z, (v, ids, rest), tau, kind, beta = s["draft"], s["top"], s["tau"], s["kind"], s["beta"]
    N, V = z.shape
    rows = None
    if s["mask"] is not None:
        rows = s["mask"].nonzero()[:, 0]
        z, v, ids = z[rows], v[rows], ids[rows]
        rest = rest[rows] if rest is not None else None
    at = ids.long()
    x = z.float() / tau
    m = x.amax(1, keepdim=True)
    e = torch.exp(x - m)
    xc = x.gather(1, at)
    e_rest = e.scatter(1, at, 0.0)  # the draft's mass outside the top entries, summed on its own
    sr = e_rest.sum(1, keepdim=True)
    ec = e.gather(1, at)
    Z = ec.sum(1, keepdim=True) + sr
    lq = torch.cat([xc - m - torch.log(Z), torch.log(sr) - torch.log(Z)], 1)
    q = torch.cat([ec, sr], 1) / Z
    r = rest[:, None] if rest is not None else torch.full_like(sr, -math.inf)
    t = torch.cat([v / tau, r], 1)
    mt = t.amax(1, keepdim=True)
    et = torch.exp(t - mt)
    L = et.sum(1, keepdim=True)
    p = et / L
    lp = t - mt - torch.log(L)
    if kind == "ce":
        p = torch.zeros_like(p)
        p[:, 0] = 1.0  # the top entries are sorted: the first is the label
    if kind in ("fkl", "ce"):
        loss = (-lq[:, 0]) if kind == "ce" else torch.where(p > 0, p * (lp - lq), 0.0).sum(1)
        gq = q - p
        fac = torch.where(sr > 0, gq[:, -1:] / sr, 0.0)
    else:
        if kind == "rkl":
            d = torch.where(q > 0, lq - lp, 0.0)
            loss = (q * d).sum(1)
            g = d - loss[:, None]
        else:
            mix = beta * p + (1 - beta) * q
            lm = torch.log(mix)
            kp = torch.where(p > 0, p * (lp - lm), 0.0).sum(1)
            d = torch.where(q > 0, lq - lm, 0.0)
            kq = (q * d).sum(1)
            loss = beta * kp + (1 - beta) * kq
            g = (1 - beta) * (d - kq[:, None])
        gq = q * g
        fac = g[:, -1:] / Z
    grad = (e_rest * fac).scatter_(1, at, gq[:, :-1]) / tau
    if rows is not None:
        whole_l, whole_g = torch.zeros(N, device=z.device), torch.zeros(N, V, device=z.device)
        whole_l[rows], whole_g[rows] = loss, grad
        return whole_l, whole_g
    return loss, grad


def run(s):
    if not own:
        return {"verify": _plain_verify, "topk": _plain_topk, "distill": _plain_distill}[s["op"]](s)
    import paper_2310_07177_gb300 as osd
    if s["op"] == "verify":
        out = osd.VerifyResult(*s["out"]) if s["out"] is not None else None
        r = osd.osd_verify_probs(s["draft_probs"], s["target_probs"], s["tokens"], s["u"], draft_lens=s["lens"], out=out)
        return tuple(r)[:3]
    if s["op"] == "topk":
        out = osd.TopkResult(*s["out"]) if not s["fresh"] or s["mask"] is not None else None
        return tuple(osd.osd_topk(s["logits"], min(s["K"], s["V"]), s["mask"], temperature=s["tau"], rest=s["rest"], out=out))
    return osd.osd_distill_topk(s["draft"], s["top"], s["mask"], s["kind"], s["beta"], temperature=s["tau"],
                                loss=s["loss"], dlogits=s["dlogits"])


def work(case):
    """Each input read once and each output written once; of verification's rows the pair at the first
    rejection (or the row past the last draft), of masked rows the ones that count."""
    V, es, op = case["V"], DTYPES[case["dtype"]].itemsize, case["op"]
    if op == "verify":
        B, k = case["B"], case["k"]
        lens = range(k + 1) if case["ragged"] else [k]
        passes = sum(case["accept"] ** n for n in lens) / len(lens)  # every draft of a sequence accepted
        rows = 2.0 - passes if case["draft"] else 1.0
        return {"bytes": int(B * (rows * V * es + 2 * k * es + 4 * k + 8 * (k + 1) + k + 4)), "flops": int(B * rows * V * 3)}
    if op == "topk":
        n = case["G"] * case["P"]
        rows = max(1, round(case["active"] * n)) if case["active"] < 1.0 else n
        return {"bytes": rows * (V * es + 8 * min(case["K"], V) + 4), "flops": rows * V * (12 if case["rest"] else 2)}
    rows = max(1, round(case["active"] * case["N"])) if case["active"] < 1.0 else case["N"]
    return {"bytes": rows * (V * (es + 4) + 8 * min(case["K"], V) + 8), "flops": rows * V * 22}


# ------------------------------------------------------------------ 64-bit results
def _exact_verify(s):
    p, q, k = s["target_probs"], s["draft_probs"], s["k"]
    ys, us = s["tokens"].tolist(), s["u"].double().tolist()
    lens = s["lens"].tolist() if s["lens"] is not None else [k] * s["B"]
    acc, toks, masks = [], [], []
    for b in range(s["B"]):
        row, mask, w = [-1] * (k + 1), [0] * k, None
        for i in range(lens[b]):
            y = ys[b][i]
            qy = float(q[b, i, y]) if q is not None else 1.0
            if us[b][i] * qy < float(p[b, i, y]):
                row[i] = y
                continue
            w = p[b, i].double()
            if q is not None:
                w = w - q[b, i].double()
            else:
                w[y] -= 1.0
            w, mask[i] = torch.relu(w), 1
            break
        else:
            i = lens[b]
            w = p[b, i].double()
        C = w.cumsum(0)
        if float(C[-1]) > 0.0:
            over = (C > us[b][k] * C[-1]).nonzero()
            row[i] = int(over[0]) if len(over) else int(w.nonzero()[-1])
        else:
            row[i] = int((p[b, i] == p[b, i].max()).nonzero()[0])
        acc.append(i)
        toks.append(row)
        masks.append(mask)
    return (torch.tensor(acc, dtype=torch.int32), torch.tensor(toks, dtype=torch.int32),
            torch.tensor(masks, dtype=torch.uint8))


def _exact_topk(s):
    x, K = s["logits"], min(s["K"], s["V"])
    G, P, V = x.shape
    values = torch.zeros(G * P, K, dtype=torch.float64, device="cuda")
    ids = torch.zeros(G * P, K, dtype=torch.int32, device="cuda")
    rest = torch.zeros(G * P, dtype=torch.float64, device="cuda") if s["rest"] else None
    on = torch.arange(G * P, device="cuda") if s["mask"] is None else s["mask"].view(-1).nonzero()[:, 0]
    step = max(1, (1 << 26) // V)
    for r in range(0, len(on), step):
        n = on[r:r + step]
        xi = x[n // P, n % P].double()
        # value and index in one integer, so that no two are equal: the values are fp32 numbers
        bits = (xi.float() + 0.0).view(torch.int32).long()
        key = (torch.where(bits < 0, -(bits & 0x7fffffff), bits) << 22) - torch.arange(V, device="cuda")
        i = torch.topk(key, K).indices
        values[n], ids[n] = xi.gather(1, i), i.int()
        if rest is not None:
            rest[n] = torch.logsumexp((xi / s["tau"]).scatter(1, i, -math.inf), 1)
    return values.view(G, P, K), ids.view(G, P, K), rest.view(G, P) if rest is not None else None


def _exact_distill(s):
    z, (v, ids, rest), tau, kind, beta = s["draft"], s["top"], s["tau"], s["kind"], s["beta"]
    N, V = z.shape
    loss = torch.zeros(N, dtype=torch.float64, device="cuda")
    grad = torch.zeros(N, V, dtype=torch.float64, device="cuda")
    on = torch.arange(N, device="cuda") if s["mask"] is None else s["mask"].nonzero()[:, 0]
    step = max(1, (1 << 26) // V)
    for r in range(0, len(on), step):
        n = on[r:r + step]
        lz = torch.log_softmax(z[n].double() / tau, 1)
        i = ids[n].long()
        lqr = torch.logsumexp(lz.scatter(1, i, -math.inf), 1, keepdim=True)
        lq = torch.cat([lz.gather(1, i), lqr], 1)
        t = v[n].double() / tau
        t = torch.cat([t, rest[n, None].double() if rest is not None else torch.full_like(lqr, -math.inf)], 1)
        lp = torch.log_softmax(t, 1)
        p, q = lp.exp(), lq.exp()
        # g: the derivative of the loss by each class's mass, where that mass is not zero
        if kind == "fkl":
            loss[n], g = torch.where(p > 0, p * (lp - lq), 0.0).sum(1), -p / q
        elif kind == "rkl":
            loss[n], g = torch.where(q > 0, q * (lq - lp), 0.0).sum(1), lq - lp
        elif kind == "jsd":
            lm = torch.logaddexp(math.log(beta) + lp, math.log1p(-beta) + lq)
            kl = lambda a, la: torch.where(a > 0, a * (la - lm), 0.0).sum(1)
            loss[n], g = beta * kl(p, lp) + (1 - beta) * kl(q, lq), (1 - beta) * (lq - lm)
        else:
            loss[n], g = -lq[:, 0], torch.zeros_like(q)
            g[:, 0] = -1.0 / q[:, 0]
        g = torch.where(q > 0, g, 0.0)
        g = g - (q * g).sum(1, keepdim=True)
        out = lz.exp() * g[:, -1:]
        grad[n] = out.scatter_(1, i, (q * g)[:, :-1]) / tau
    return loss, grad


def exact(case, seed):
    s = prepare(case, seed)
    s["dlogits"] = None
    return {"verify": _exact_verify, "topk": _exact_topk, "distill": _exact_distill}[case["op"]](s)
