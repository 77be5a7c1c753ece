"""The operators of label-synchronous decoding and training around the package's recurrent layers, as calls of its
public entry points (own = True) and in their plain form (own = False: elementary torch operations).

Kinds:
  attn    qnn.qnn_linear_attention: linear attention with a decay for each head, S = d S + k v^T, y = scale q S, for
          prompts and single frames, with the states of all sequences in and out.
  select  qnn.qnn_beam_select: the n best continuations over beams and classes, score + log softmax, ties to the lowest
          beam and class; finished beams keep their score and continue with the end class only.
  reorder qnn.qnn_beam_reorder: the carried states and label histories of the beams that the selection kept.
  embed   qnn.qnn_embedding: rows of a table by label, scaled; labels below 0 are padding.
  egrad   qnn.qnn_embedding_grad: the table's gradient, the rows of a label added in the order of their positions.

The widths, classes and batches are those of the package's workloads (5 x 500 and 5 x 2048 / 512 stacks, 2000 and 8192
classes, 300 to 1000 frames, batches of 1 to 1024) or generic.
"""
from __future__ import annotations

import math

import torch

own = False
DEV = "cuda"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


# ------------------------------------------------------------------------------------------------
# The cases
# ------------------------------------------------------------------------------------------------

def listed():
    return [
        # one frame of each of 256 streams, states carried: serving
        {"name": "attn_256x1x16x128_bf16", "kind": "attn", "B": 256, "T": 1, "H": 16, "Hq": 16, "Hk": 16, "Hv": 16, "dk": 128,
         "dv": 128, "type": "bf16", "ragged": False, "states": True},
        # one long utterance in full precision: few heads, many frames
        {"name": "attn_1x4000x8x64_f32", "kind": "attn", "B": 1, "T": 4000, "H": 8, "Hq": 8, "Hk": 8, "Hv": 8, "dk": 64,
         "dv": 64, "type": "f32", "ragged": False, "states": True},
        # a padded batch of short utterances: 500 units in five heads, keys and queries shared by all of them
        {"name": "attn_4x300x5x100_f16", "kind": "attn", "B": 4, "T": 300, "H": 5, "Hq": 1, "Hk": 1, "Hv": 5, "dk": 100,
         "dv": 100, "type": "f16", "ragged": True, "states": True},
        # a padded batch of long utterances, 2048 units: the largest
        {"name": "attn_16x1000x16x128_bf16", "kind": "attn", "B": 16, "T": 1000, "H": 16, "Hq": 16, "Hk": 16, "Hv": 16,
         "dk": 128, "dv": 128, "type": "bf16", "ragged": True, "states": False},
        # one utterance, four beams, the 5 x 500 model's classes: latency
        {"name": "select_1x4x2000_f32", "kind": "select", "B": 1, "K": 4, "V": 2000, "n": 4, "type": "f32", "finished": False},
        # 128 utterances of eight beams over 8192 classes, twice as many kept as there are beams
        {"name": "select_128x8x8192_bf16", "kind": "select", "B": 128, "K": 8, "V": 8192, "n": 16, "type": "bf16",
         "finished": True},
        # the states of a 5 x 500 stack for four beams: latency
        {"name": "reorder_1x4_5x500", "kind": "reorder", "B": 1, "K": 4, "L": 5, "H": 500, "P": 0, "S": 64},
        # the states of a 5 x 2048 / 512 stack for 64 utterances of eight beams
        {"name": "reorder_64x8_5x2048p512", "kind": "reorder", "B": 64, "K": 8, "L": 5, "H": 2048, "P": 512, "S": 300},
        # the labels of four beams: latency
        {"name": "embed_4x500_f32", "kind": "embed", "n": 4, "D": 500, "V": 2000, "type": "f32", "padding": False},
        # the labels of a padded batch, 2048 units
        {"name": "embed_16000x2048_bf16", "kind": "embed", "n": 16000, "D": 2048, "V": 8192, "type": "bf16", "padding": True},
        # a padded batch of short label sequences, 500 units
        {"name": "egrad_1200x500_f32", "kind": "egrad", "n": 1200, "D": 500, "V": 2000, "type": "f32", "padding": True},
        # the labels of a training batch, 2048 units
        {"name": "egrad_16000x2048_bf16", "kind": "egrad", "n": 16000, "D": 2048, "V": 8192, "type": "bf16", "padding": True},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    kind = rng.choice(["attn", "attn", "attn", "select", "select", "reorder", "embed", "egrad", "egrad"])
    ty = rng.choice(["f32", "bf16", "f16"])
    if kind == "attn":
        H = rng.choice([1, 2, 4, 5, 8, 12, 16, 32])
        dk = rng.choice([_log(rng, 8, 256), 32, 64, 64, 100, 128, 128, 192, 256])
        dv = dk if rng.random() < 0.7 else rng.choice([_log(rng, 8, 256), 64, 128])
        if rng.random() < 0.35:  # single frames, or a few of them
            T = rng.choice([1, 1, 1, 2, 5])
            B = _log(rng, 1, max(1, min(1024, 256 * 16 * 128 * 128 // (H * dk * dv))))
        else:
            T = _log(rng, 6, 4000)
            B = _log(rng, 1, max(1, min(64, 16 * 16 * 1000 * 1000 // (H * T * T), 16 * 16 * 1000 * 128 // (H * T * max(dk, dv)))))
        few = rng.choice([h for h in (1, 2, 4, H) if H % h == 0])
        Hq, Hk, Hv = rng.choice([(H, H, H), (H, H, H), (few, few, H), (H, few, few)])
        return {"kind": kind, "B": B, "T": T, "H": H, "Hq": Hq, "Hk": Hk, "Hv": Hv, "dk": dk, "dv": dv, "type": ty,
                "ragged": rng.random() < 0.4, "states": rng.random() < 0.7}
    if kind == "select":
        K, V = rng.choice([1, 2, 4, 5, 8, 16, 32]), _log(rng, 29, 65536)
        return {"kind": kind, "B": _log(rng, 1, max(1, min(256, 128 * 8 * 8192 // (K * V)))), "K": K, "V": V,
                "n": rng.choice([K, K, 2 * K]), "type": ty, "finished": rng.random() < 0.5}
    if kind == "reorder":
        K, H = rng.choice([2, 4, 5, 8, 16]), _log(rng, 40, 2048)
        return {"kind": kind, "B": _log(rng, 1, max(1, 512 // K)), "K": K, "L": rng.choice([1, 2, 3, 5]), "H": H,
                "P": rng.choice([0, H // 4]), "S": _log(rng, 1, 300)}
    D, V = _log(rng, 40, 4096), _log(rng, 29, 65536)
    n = _log(rng, 1, max(1, min(65536, 16000 * 2048 // D)))
    return {"kind": kind, "n": n, "D": D, "V": min(V, 16000 * 2048 // D), "type": ty, "padding": rng.random() < 0.5}


def work(case):
    c = dict(case)
    e = TYPES[c["type"]].itemsize if "type" in c else 4
    if c["kind"] == "attn":
        frames = sum(_lengths(c)) if c["ragged"] else c["B"] * c["T"]
        state = c["dk"] * c["dv"]
        return {"bytes": e * frames * ((c["Hq"] + c["Hk"]) * c["dk"] + (c["Hv"] + c["H"]) * c["dv"]) +
                4 * (2 if c["states"] else 1) * c["B"] * c["H"] * state, "flops": 5 * frames * c["H"] * state}
    if c["kind"] == "select":
        n = c["B"] * c["K"] * c["V"]
        return {"bytes": e * n + 4 * c["B"] * c["K"] + 12 * c["B"] * c["n"], "flops": 4 * n}
    if c["kind"] == "reorder":
        values = c["B"] * c["K"] * (c["L"] * (c["H"] + (c["P"] or c["H"])) + c["S"])
        return {"bytes": 8 * values + 4 * c["B"] * c["K"], "flops": values}
    n, D, V = c["n"], c["D"], c["V"]
    if c["kind"] == "embed":
        rows = V * (1.0 - (1.0 - 1.0 / V) ** n)  # no more rows are read than there are, nor than labels
        return {"bytes": e * D * (n + min(n, rows)) + 4 * n, "flops": n * D}
    return {"bytes": e * n * D + 4 * V * D + 4 * n, "flops": n * D}


# ------------------------------------------------------------------------------------------------
# Inputs
# ------------------------------------------------------------------------------------------------

def _lengths(c):
    """Frames of each sequence of a padded batch: from a third of the longest to all of it."""
    B, T = c["B"], c["T"]
    return [T - (b * 7 % 11) * (2 * T // 3) // 10 for b in range(B)]


def prepare(case, seed):
    c = dict(case)
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) + 1)

    def normal(*shape, std=1.0):
        return torch.randn(shape, generator=g, device=DEV) * std

    def uniform(*shape):
        return torch.rand(shape, generator=g, device=DEV)

    if c["kind"] == "attn":
        B, T, H, dk, dv, t = c["B"], c["T"], c["H"], c["dk"], c["dv"], TYPES[c["type"]]
        # decays from 1 - 2^-3 to 1 - 2^-9 a frame over the heads
        rate = 2.0 ** -(3.0 + 6.0 * (torch.arange(H, device=DEV) + uniform(H)) / H)
        return {"case": c, "q": normal(B, T, c["Hq"], dk).to(t), "k": normal(B, T, c["Hk"], dk).to(t),
                "v": normal(B, T, c["Hv"], dv).to(t), "log_decay": torch.log1p(-rate),
                "s_in": normal(B, H, dk, dv, std=2.0) if c["states"] else None,
                "s_out": torch.zeros((B, H, dk, dv), device=DEV), "out": torch.zeros((B, T, H, dv), dtype=t, device=DEV),
                "lengths": torch.tensor(_lengths(c), dtype=torch.int32, device=DEV) if c["ragged"] else None}
    if c["kind"] == "select":
        B, K, V = c["B"], c["K"], c["V"]
        # a few classes of a frame stand out, differently sharp from beam to beam
        logits = normal(B, K, V, std=2.0) * (0.5 + uniform(B, K, 1)) + 6.0 * (uniform(B, K, V) < 4.0 / V)
        scores = torch.sort(-20.0 + normal(B, K, std=2.0), dim=1, descending=True)[0].contiguous()
        return {"case": c, "logits": logits.to(TYPES[c["type"]]), "scores": scores,
                "finished": uniform(B, K) < 0.2 if c["finished"] else None, "eos": 1}
    if c["kind"] == "reorder":
        B, K, L, H, P, S = c["B"], c["K"], c["L"], c["H"], c["P"], c["S"]
        old = [normal(L, B * K, P or H), normal(L, B * K, H),
               (uniform(B * K, S) * 8192).to(torch.int32)]
        return {"case": c, "states": old, "out": [torch.zeros_like(s) for s in old], "dims": [1, 1, 0],
                "parents": (uniform(B, K) ** 2 * K).to(torch.int32).clamp(max=K - 1)}
    n, D, V, t = c["n"], c["D"], c["V"], TYPES[c["type"]]
    # labels by falling frequency, 1 / (rank + 1), scattered over the table
    rank = torch.exp(uniform(n) * math.log(V + 1.0)).to(torch.int64) - 1
    ids = (rank.clamp(0, V - 1) * 7919 + 13) % V if V % 7919 else rank.clamp(0, V - 1)
    if c["padding"]:
        ids = torch.where(uniform(n) < 0.15, torch.full_like(ids, -1), ids)
    ids = ids.to(torch.int32)
    if c["kind"] == "embed":
        return {"case": c, "ids": ids, "table": normal(V, D, std=0.05).to(t), "scale": math.sqrt(D)}
    return {"case": c, "ids": ids, "grad": normal(n, D).to(t), "scale": math.sqrt(D)}


# ------------------------------------------------------------------------------------------------
# One pass: the plain forms
# ------------------------------------------------------------------------------------------------

def _heads(x, H):
    """[B, T, heads, d] -> [B, H, T, d] in 32 bits, each head for those that share it."""
    x = x.float().transpose(1, 2)
    return x.repeat_interleave(H // x.shape[1], 1)


def _plain_attn(s):
    c = s["case"]
    B, T, H = c["B"], c["T"], c["H"]
    scale = c["dk"] ** -0.5
    q, k, v = (_heads(s[n], H) for n in "qkv")
    d = s["log_decay"]
    at = torch.arange(T, device=DEV)
    n = s["lengths"].long() if s["lengths"] is not None else torch.full((B,), T, device=DEV)
    there = at[None, :] < n[:, None]  # [B, T]
    back = (at[:, None] - at[None, :])
    w = torch.where(back >= 0, torch.exp(d[:, None, None] * back.clamp(min=0)), torch.zeros((), device=DEV))  # [H, T, T]
    a = q @ k.transpose(2, 3)
    a *= w
    y = a @ v
    del a
    left = n[:, None] - 1 - at[None, :]
    keep = torch.where(there[:, None, :], torch.exp(d[None, :, None] * left.clamp(min=0)[:, None, :]),
                       torch.zeros((), device=DEV))  # [B, H, T]
    state = (k * keep[..., None]).transpose(2, 3) @ v
    if s["s_in"] is not None:
        y = y + torch.exp(d[:, None] * (at[None, :] + 1))[None, :, :, None] * (q @ s["s_in"])
        state = state + torch.exp(d[None, :] * n[:, None])[..., None, None] * s["s_in"]
    y = torch.where(there[:, None, :, None], y * scale, torch.zeros((), device=DEV))
    return {"y": y.transpose(1, 2).to(s["q"].dtype), "state": state}


def _plain_select(s):
    c = s["case"]
    B, K, V, n = c["B"], c["K"], c["V"], c["n"]
    # in 64 bits: two candidates may lie closer than a rounding to 32 of their scores
    x = s["logits"].double()
    m = x.amax(2, keepdim=True)
    lse = m + torch.log(torch.exp(x - m).sum(2, keepdim=True))
    cand = s["scores"].double()[..., None] + (x - lse)
    none = torch.full((), -math.inf, dtype=torch.float64, device=DEV)
    cand = torch.where(torch.isnan(cand), none, cand)
    if s["finished"] is not None:
        end = torch.arange(V, device=DEV)[None, None, :] == s["eos"]
        kept = torch.where(end, s["scores"].double()[..., None], none)
        cand = torch.where(s["finished"][..., None], kept, cand)
    best, at = torch.sort(cand.view(B, K * V), dim=1, descending=True, stable=True)
    best, at = best[:, :n], at[:, :n]
    lost = best == -math.inf
    zero = torch.zeros_like(at)
    return {"scores": best.float(), "parents": torch.where(lost, zero, at // V).int(),
            "tokens": torch.where(lost, zero + s["eos"], at % V).int()}


def _plain_reorder(s):
    c = s["case"]
    rows = (torch.arange(c["B"], device=DEV)[:, None] * c["K"] + s["parents"].long()).reshape(-1)
    return [x[:, rows] if d == 1 else x[rows] for x, d in zip(s["states"], s["dims"])]


def _plain_embed(s):
    ids, table = s["ids"].long(), s["table"]
    there = (ids >= 0) & (ids < table.shape[0])
    rows = table[torch.where(there, ids, torch.zeros_like(ids))].float() * s["scale"]
    return torch.where(there[:, None], rows, torch.zeros((), device=DEV)).to(table.dtype)


def _plain_egrad(s):
    c = s["case"]
    ids = s["ids"].long()
    out = torch.zeros((c["V"] + 1, c["D"]), device=DEV)
    out.index_add_(0, torch.where(ids >= 0, ids, torch.full_like(ids, c["V"])), s["grad"].float())
    return out[:c["V"]] * s["scale"]


# ------------------------------------------------------------------------------------------------
# One pass
# ------------------------------------------------------------------------------------------------

def run(state):
    s, c = state, state["case"]
    if own:
        from paper_1607_04683_gb300 import qnn
        if c["kind"] == "attn":
            y = qnn.qnn_linear_attention(s["q"], s["k"], s["v"], s["log_decay"], state_in=s["s_in"], state_out=s["s_out"],
                                         lengths=s["lengths"], out=s["out"])
            return {"y": y, "state": s["s_out"]}
        if c["kind"] == "select":
            scores, parents, tokens = qnn.qnn_beam_select(s["logits"], s["scores"], c["n"], finished=s["finished"],
                                                          eos=s["eos"])
            return {"scores": scores, "parents": parents, "tokens": tokens}
        if c["kind"] == "reorder":
            return qnn.qnn_beam_reorder(s["states"], s["parents"], dims=s["dims"], out=s["out"])
        if c["kind"] == "embed":
            return qnn.qnn_embedding(s["ids"], s["table"], scale=s["scale"])
        return qnn.qnn_embedding_grad(s["grad"], s["ids"], c["V"], scale=s["scale"])
    return {"attn": _plain_attn, "select": _plain_select, "reorder": _plain_reorder, "embed": _plain_embed,
            "egrad": _plain_egrad}[c["kind"]](s)


# ------------------------------------------------------------------------------------------------
# The definitions in 64 bits
# ------------------------------------------------------------------------------------------------

def _exact_attn(s):
    c = s["case"]
    B, T, H, dk, dv = c["B"], c["T"], c["H"], c["dk"], c["dv"]
    n = _lengths(c) if c["ragged"] else [T] * B
    n = torch.tensor(n, device=DEV)
    of = {x: torch.arange(H, device=DEV) // (H // c["H" + x]) for x in "qkv"}
    S = torch.zeros((B, H, dk, dv), dtype=torch.float64, device=DEV) if s["s_in"] is None else s["s_in"].double()
    decay = torch.exp(s["log_decay"].double())[None, :, None, None]
    y = torch.zeros((B, T, H, dv), dtype=torch.float64, device=DEV)
    for t in range(T):
        q, k, v = (s[x][:, t].double()[:, of[x]] for x in "qkv")
        new = S * decay
        new += k[..., None] * v[..., None, :]
        on = (t < n)[:, None, None, None]
        S = new if not c["ragged"] else torch.where(on, new, S)
        y[:, t] = torch.where(on[..., 0], (q[..., None, :] @ S)[..., 0, :] / math.sqrt(dk), torch.zeros_like(y[:, t]))
    return {"y": y, "state": S}


def _exact_select(s):
    c = s["case"]
    B, K, V, n = c["B"], c["K"], c["V"], c["n"]
    out = {"scores": torch.full((B, n), -math.inf, dtype=torch.float64), "parents": torch.zeros((B, n), dtype=torch.int32),
           "tokens": torch.full((B, n), s["eos"], dtype=torch.int32)}
    logp = torch.log_softmax(s["logits"].double(), 2)
    # no beam gives more than n: its n best in order, then all beams' against one another
    some = min(n, V)
    order = torch.argsort(logp, dim=2, descending=True, stable=True)[..., :some].cpu()
    logp = torch.gather(logp, 2, order.to(DEV)).cpu()
    scores = s["scores"].double().cpu()
    finished = s["finished"].cpu() if s["finished"] is not None else torch.zeros((B, K), dtype=torch.bool)
    for b in range(B):
        cands = []
        for k in range(K):
            if finished[b, k]:
                cands.append((-float(scores[b, k]), k, s["eos"]))
            else:
                cands += [(-(float(scores[b, k]) + p), k, v) for p, v in zip(logp[b, k].tolist(), order[b, k].tolist())]
        for j, (score, k, v) in enumerate(sorted(cands)[:n]):
            out["scores"][b, j], out["parents"][b, j], out["tokens"][b, j] = -score, k, v
    return {"scores": out["scores"].to(DEV), "parents": out["parents"].to(DEV), "tokens": out["tokens"].to(DEV)}


def _exact_reorder(s):
    c = s["case"]
    out = []
    for x, d in zip(s["states"], s["dims"]):
        x = x.transpose(0, d)
        v = x.reshape(c["B"], c["K"], -1)
        at = s["parents"].long()[..., None].expand(-1, -1, v.shape[2])
        v = torch.gather(v, 1, at).reshape(x.shape).transpose(0, d).contiguous()
        out.append(v.double() if v.is_floating_point() else v)
    return out


def _exact_embed(s):
    one = torch.zeros((s["table"].shape[0] + 1, s["table"].shape[1]), dtype=torch.float64, device=DEV)
    one[1:] = s["table"].double() * s["scale"]
    return torch.index_select(one, 0, s["ids"].long() + 1)


def _exact_egrad(s):
    c = s["case"]
    order = torch.argsort(s["ids"], stable=True)
    ids = s["ids"].long()[order]
    total = torch.zeros((len(ids) + 1, c["D"]), dtype=torch.float64, device=DEV)
    torch.cumsum(s["grad"].double()[order], 0, out=total[1:])
    row = torch.arange(c["V"], device=DEV)
    return (total[torch.searchsorted(ids, row, right=True)] - total[torch.searchsorted(ids, row)]) * s["scale"]


def exact(case, seed):
    s = prepare(case, seed)
    return {"attn": _exact_attn, "select": _exact_select, "reorder": _exact_reorder, "embed": _exact_embed,
            "egrad": _exact_egrad}[s["case"]["kind"]](s)
