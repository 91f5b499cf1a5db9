"""Causal cosine attention with a decay for each head, for prompts, for training and token by token, and trees of
drafted tokens over its states: one pass of each through the public binding (`own`), or from elementary operations.

With qh, kh the L2-normalised rows, g = exp(log_decay[h]) and a scale s[h]:

  prefill  o_i = s qh_i H_i,  H_i = g H_(i-1) + kh_i^T v_i, of B prompts, leaving the state H after the last token;
           with "piece" it starts from a state; with "padded" the prompts have lengths of their own
  train    the same without states, and its gradients dQ, dK, dV, ds
  step     one token: H = g H + kh^T v in place, o = s qh H; with "beams" every sequence goes on from the state of the
           one that the beam search chose as its parent
  tree     T drafted tokens that form a tree: a token's state is its parent's, the roots' is the sequence's, which is
           left as it is;  o_i = s qh_i (g^(depth_i + 1) H + sum over its ancestors j and itself g^(depth_i - depth_j) kh_j^T v_j)
  accept   the state after the accepted path of such a tree, in place

A case is a dict of plain values: kind, B, H (sequences, heads), N (tokens of a sequence; for trees, of a tree), dk, dv (width
of queries and keys, of values), dtype ("bf16", "f16" or "f32": storage of the rows; states are float32) and the words above.

Rows are standard normal, as after the projections of a layer; decays halve a token's weight after 8 to 4096 tokens,
spread over the heads; the scale is drawn around 1.
"""
import math

import numpy as np
import torch

own = False

_TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
_SIZE = {"bf16": 2, "f16": 2, "f32": 4}
_EPS = 1e-6


def listed():
    return [
        # the prompts of a serving batch
        {"name": "prefill_64_prompts", "kind": "prefill", "piece": False, "padded": False, "B": 64, "H": 16, "N": 2048,
         "dk": 128, "dv": 128, "dtype": "bf16"},
        # the next hundred tokens of one user's conversation
        {"name": "prefill_piece", "kind": "prefill", "piece": True, "padded": False, "B": 1, "H": 16, "N": 100,
         "dk": 128, "dv": 128, "dtype": "bf16"},
        # prompts of different lengths in one batch, values wider than keys
        {"name": "prefill_padded", "kind": "prefill", "piece": False, "padded": True, "B": 16, "H": 12, "N": 389,
         "dk": 64, "dv": 128, "dtype": "f16"},
        # a layer of a GPT-shaped training step
        {"name": "train_gpt", "kind": "train", "padded": False, "B": 8, "H": 12, "N": 1024, "dk": 64, "dv": 64,
         "dtype": "bf16"},
        # one long document
        {"name": "train_long", "kind": "train", "padded": False, "B": 1, "H": 16, "N": 65536, "dk": 64, "dv": 64,
         "dtype": "bf16"},
        # an odd length in full precision
        {"name": "train_odd_f32", "kind": "train", "padded": False, "B": 3, "H": 5, "N": 777, "dk": 64, "dv": 64,
         "dtype": "f32"},
        # one user's sequence being generated: nothing but latency
        {"name": "step_one_sequence", "kind": "step", "beams": False, "B": 1, "H": 16, "N": 1, "dk": 128, "dv": 128,
         "dtype": "bf16"},
        # 64 sequences with four beams each
        {"name": "step_256_beams", "kind": "step", "beams": True, "B": 256, "H": 16, "N": 1, "dk": 128, "dv": 128,
         "dtype": "bf16"},
        # a small tree of drafts for one user
        {"name": "tree_one_sequence", "kind": "tree", "B": 1, "H": 16, "N": 13, "dk": 128, "dv": 128, "dtype": "bf16"},
        # full trees for a serving batch
        {"name": "tree_64_sequences", "kind": "tree", "B": 64, "H": 16, "N": 64, "dk": 128, "dv": 128, "dtype": "bf16"},
        # what one user's drafts came to
        {"name": "accept_one_sequence", "kind": "accept", "B": 1, "H": 16, "N": 13, "dk": 128, "dv": 128,
         "dtype": "bf16"},
        # the same for a serving batch
        {"name": "accept_256_sequences", "kind": "accept", "B": 256, "H": 16, "N": 32, "dk": 128, "dv": 128,
         "dtype": "bf16"},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["prefill", "prefill", "train", "train", "step", "tree", "accept"])
    H = rng.choice([5, 8, 12, 16])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    dk = dv = rng.choice([32, 64, 64, 128])
    if rng.random() < 0.25:
        dv = rng.choice([32, 64, 128])
    case = {"kind": kind, "H": H, "dk": dk, "dv": dv, "dtype": dtype}
    if kind in ("prefill", "train"):
        # elements of one row tensor: 1.0e8 at most, 2.5e7 in full precision
        most = 2.5e7 if dtype == "f32" else 1.0e8
        N = _log_int(rng, 2, 16384) if kind == "prefill" else _log_int(rng, 100, 65536)
        if rng.random() < 0.3:
            N = max(64, N // 64 * 64)
        wide = max(dk, dv)
        N = max(2, min(N, int(most / (H * wide))))
        case["N"] = N
        case["B"] = max(1, min(_log_int(rng, 1, 64), int(most / (H * N * wide))))
        case["padded"] = rng.random() < 0.25
        if kind == "prefill":
            case["piece"] = rng.random() < 0.5
        return case
    case["B"] = _log_int(rng, 1, 256)
    case["N"] = 1 if kind == "step" else rng.randint(2, 64)
    if kind == "tree":
        case["B"] = min(case["B"], 64)
    if kind == "step":
        case["beams"] = rng.random() < 0.5
    return case


def _lengths(case):
    """Tokens of each sequence of a padded batch: spread evenly from a quarter of N to N."""
    B, N = case["B"], case["N"]
    return [max(1, round(N * (0.25 + 0.75 * (b + 1) / B))) for b in range(B)]


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    B, H, N, dk, dv = (case[k] for k in ("B", "H", "N", "dk", "dv"))
    kind, dt = case["kind"], _TYPES[case["dtype"]]

    def rows(width):
        shape = (B, H, width) if kind == "step" else (B, H, N, width)
        return torch.randn(shape, generator=gen, device="cuda").to(dt)

    def states():
        return torch.randn((B, H, dk, dv), generator=gen, device="cuda")

    x = {"case": case, "K": rows(dk), "V": rows(dv)}
    half_life = 8.0 * 512.0 ** (torch.arange(H, device="cuda", dtype=torch.float64) / max(1, H - 1))
    x["log_decay"] = (-math.log(2.0) / half_life).float()
    if kind != "accept":
        x["Q"] = rows(dk)
        shape = (B, H) if case.get("padded") else (H,)
        x["s"] = 0.5 + torch.rand(shape, generator=gen, device="cuda")
    if case.get("padded"):
        x["seq_len"] = torch.tensor(_lengths(case), dtype=torch.int32, device="cuda")
    if kind == "train":
        x["dO"] = rows(dv)
    if kind == "prefill":
        x["state"] = torch.empty((B, H, dk, dv), device="cuda")
        if case["piece"]:
            x["state_in"] = states()
    if kind in ("step", "tree", "accept"):
        x["state"] = states()
    if case.get("beams"):
        x["state_in"] = states()
        # beams come in groups of up to four, and a beam's parent is one of its group
        group = torch.arange(B, device="cuda") // 4 * 4
        pick = torch.randint(0, 4, (B,), generator=gen, device="cuda")
        x["parent"] = torch.clamp(group + pick, max=B - 1).to(torch.int32)
    if kind in ("tree", "accept"):
        # token 0 is a root; each further one hangs on an earlier token, mostly on one of the last four
        at = torch.arange(N, device="cuda")
        back = torch.randint(1, 5, (B, N), generator=gen, device="cuda")
        x["parent"] = torch.clamp(at - back, min=-1).to(torch.int32)
        x["parent"][:, 0] = -1
    if kind == "accept":
        # in one sequence of eight nothing was accepted
        last = torch.randint(0, N, (B,), generator=gen, device="cuda")
        none = torch.rand((B,), generator=gen, device="cuda") < 0.125
        x["last"] = torch.where(none, -1, last).to(torch.int32)
    return x


# ---- the framework's calls ----------------------------------------------------------------------

def _run_own(x):
    import paper_2409_18747_amd.binding as cottn
    case = x["case"]
    kind = case["kind"]
    if kind == "prefill":
        O = cottn.cottn_fwd_causal_decay(x["Q"], x["K"], x["V"], x["s"], x["log_decay"], seq_len=x.get("seq_len"),
                                         state_in=x.get("state_in"), state=x["state"])
        return {"O": O, "state": x["state"]}
    if kind == "train":
        code = {"bf16": cottn.COTTN_BF16, "f16": cottn.COTTN_F16, "f32": cottn.COTTN_F32}[case["dtype"]]
        n = cottn.cottn_workspace_bytes_dkdv(cottn.OP_FWD_DECAY, case["B"], case["H"], case["N"], case["dk"], case["dv"],
                                             0, code)
        workspace = torch.empty(n, dtype=torch.uint8, device="cuda") if n else None
        O = cottn.cottn_fwd_causal_decay(x["Q"], x["K"], x["V"], x["s"], x["log_decay"], seq_len=x.get("seq_len"),
                                         workspace=workspace)
        dQ, dK, dV, ds = cottn.cottn_bwd_causal_decay(x["Q"], x["K"], x["V"], x["s"], x["log_decay"], x["dO"],
                                                      seq_len=x.get("seq_len"), fwd_workspace=workspace)
        return {"O": O, "dQ": dQ, "dK": dK, "dV": dV, "ds": ds}
    if kind == "step":
        o = cottn.cottn_step_decay(x["Q"], x["K"], x["V"], x["s"], x["log_decay"], x["state"],
                                   state_in=x.get("state_in"), parent=x.get("parent"))
        return {"o": o, "state": x["state"]}
    if kind == "tree":
        return {"o": cottn.cottn_tree(x["Q"], x["K"], x["V"], x["s"], x["state"], x["parent"], log_decay=x["log_decay"])}
    cottn.cottn_tree_accept(x["K"], x["V"], x["state"], x["parent"], x["last"], log_decay=x["log_decay"])
    return {"state": x["state"]}


# ---- the plain form ------------------------------------------------------------------------------

_CHUNK = 256


def _unit(x):
    """Rows divided by max(norm, eps), and what they were multiplied by."""
    x = x.float()
    r = 1.0 / torch.clamp(torch.sqrt((x * x).sum(-1, keepdim=True)), min=_EPS)
    return x * r, r


def _through_norm(dxh, xh, r):
    return r * (dxh - xh * (xh * dxh).sum(-1, keepdim=True))


def _in_chunks(x, n_chunks, C):
    """[B, H, N, d] as [B, H, chunks, C, d], filled up with zeros."""
    B, H, N, d = x.shape
    full = torch.zeros((B, H, n_chunks * C, d), dtype=x.dtype, device=x.device)
    full[:, :, :N] = x
    return full.view(B, H, n_chunks, C, d)


def _powers(log_decay, exponents):
    """[H, ...]: exp(log_decay[h] * exponent), zero where the exponent is negative."""
    e = exponents.double()
    w = torch.exp(log_decay.double().view((-1,) + (1,) * e.dim()) * torch.clamp(e, min=0.0))
    return torch.where(e < 0, torch.zeros_like(w), w).float()


def _run_rows(x):
    case = x["case"]
    N, dt = case["N"], x["Q"].dtype
    C = min(_CHUNK, N)
    n = -(-N // C)
    dev, ld = x["Q"].device, x["log_decay"]
    at, ci = torch.arange(C, device=dev), torch.arange(n, device=dev)
    (qh, rq), (kh, rk), v = _unit(x["Q"]), _unit(x["K"]), x["V"].float()
    lens = x.get("seq_len")
    s = x["s"].view(-1, case["H"], 1, 1)
    there = None
    if lens is not None:
        there = (torch.arange(N, device=dev) < lens[:, None]).view(-1, 1, N, 1)
        qh, kh, v = (torch.where(there, t, torch.zeros_like(t)) for t in (qh, kh, v))
    q, k, vv = (_in_chunks(t, n, C) for t in (qh, kh, v))
    D = _powers(ld, at[:, None] - at[None, :])[:, None]                 # [H, 1, C, C]
    since = _powers(ld, at + 1)[:, None, :, None]                       # from the state before the chunk to row i
    until = _powers(ld, C - 1 - at)[:, None, :, None]                   # from row j to the chunk's last
    across = _powers(ld, (ci[:, None] - ci[None, :] - 1) * C)           # [H, n, n], zero where not earlier
    totals = torch.matmul((k * until).transpose(-1, -2), vv)            # [B, H, n, dk, dv]
    before = torch.matmul(across, totals.flatten(3)).view(totals.shape)
    if "state_in" in x:
        before = before + _powers(ld, ci * C)[:, :, None, None] * x["state_in"][:, :, None]
    P = torch.matmul(q, k.transpose(-1, -2)) * D
    o = torch.matmul(q * since, before) + torch.matmul(P, vv)
    o = o.view(o.shape[:2] + (n * C, -1))[:, :, :N]
    if case["kind"] == "prefill":
        length = lens.view(-1, 1, 1) if lens is not None else torch.full((1, 1, 1), N, device=dev)
        e = (length - 1 - torch.arange(N, device=dev)).double()         # [B, 1, N]
        w = torch.exp(ld.double().view(1, -1, 1) * torch.clamp(e, min=0.0))
        w = torch.where(e < 0, torch.zeros_like(w), w).float()
        state = torch.matmul(_in_chunks(kh * w[..., None], n, C).transpose(-1, -2), vv).double().sum(2)
        if "state_in" in x:
            state = state + torch.exp(ld.double().view(1, -1, 1) * length.double())[..., None] * x["state_in"].double()
        x["state"].copy_(state)
        return {"O": (s * o).to(dt), "state": x["state"]}
    g = x["dO"].float()
    if there is not None:
        g = torch.where(there, g, torch.zeros_like(g))
    gg = _in_chunks(g, n, C)
    rev = torch.matmul((q * _powers(ld, at)[:, None, :, None]).transpose(-1, -2), gg)
    after = torch.matmul(across.transpose(-1, -2).contiguous(), rev.flatten(3)).view(rev.shape)
    to_end = _powers(ld, C - at)[:, None, :, None]                      # from row j to the first row behind the chunk
    A = torch.matmul(gg, vv.transpose(-1, -2)) * D
    dq = torch.matmul(gg * since, before.transpose(-1, -2)) + torch.matmul(A, k)
    dk = torch.matmul(vv * to_end, after.transpose(-1, -2)) + torch.matmul(A.transpose(-1, -2), q)
    dv = torch.matmul(k * to_end, after) + torch.matmul(P.transpose(-1, -2), gg)
    dq, dk, dv = (t.view(t.shape[:2] + (n * C, -1))[:, :, :N] for t in (dq, dk, dv))
    ds = (g.double() * o).sum((2, 3))
    ds = (ds if there is not None else ds.sum(0)).float()
    return {"O": (s * o).to(dt), "dQ": (s * _through_norm(dq, qh, rq)).to(dt), "dK": (s * _through_norm(dk, kh, rk)).to(dt),
            "dV": (s * dv).to(dt), "ds": ds}


def _ancestors(parent):
    """[B, T, T]: 1 where token j is token i or one of its ancestors."""
    B, T = parent.shape
    up = torch.zeros((B, T, T + 1), device=parent.device)
    up.scatter_(2, parent.long()[..., None] + 1, 1.0)
    up = up[..., 1:] + torch.eye(T, device=parent.device)
    return (torch.linalg.matrix_power(up, 64) > 0.5).float()


def _run_plain(x):
    kind = x["case"]["kind"]
    if kind in ("prefill", "train"):
        return _run_rows(x)
    ld = x["log_decay"]
    kh, v = _unit(x["K"])[0], x["V"].float()
    if kind == "step":
        before = x["state_in"][x["parent"].long()] if "parent" in x else x["state"]
        state = before * torch.exp(ld).view(-1, 1, 1) + kh[..., :, None] * v[..., None, :]
        x["state"].copy_(state)
        o = (_unit(x["Q"])[0][..., :, None] * state).sum(-2)
        return {"o": (x["s"].view(-1, 1) * o).to(x["Q"].dtype), "state": x["state"]}
    anc = _ancestors(x["parent"])                                       # [B, T, T]
    depth = anc.sum(-1) - 1.0
    if kind == "tree":
        apart = torch.clamp(depth[:, :, None] - depth[:, None, :], min=0.0)[:, None]
        w = anc[:, None] * torch.exp(ld.view(-1, 1, 1) * apart)
        since = torch.exp(ld.view(-1, 1, 1) * (depth[:, None, :, None] + 1.0))
        qh = _unit(x["Q"])[0]
        o = torch.matmul(qh * since, x["state"]) + torch.matmul(torch.matmul(qh, kh.transpose(-1, -2)) * w, v)
        return {"o": (x["s"].view(-1, 1, 1) * o).to(x["Q"].dtype)}
    last = x["last"].long()
    row = torch.clamp(last, min=0)
    on_path = torch.gather(anc, 1, row[:, None, None].expand(-1, 1, anc.shape[2]))[:, 0]
    end = torch.gather(depth, 1, row[:, None])
    apart = torch.clamp(end - depth, min=0.0)[:, None]                  # [B, 1, T]
    w = on_path[:, None] * torch.exp(ld.view(-1, 1) * apart) * (last >= 0).view(-1, 1, 1)
    kept = torch.exp(ld * torch.where(last[:, None] >= 0, end + 1.0, torch.zeros_like(end)))
    x["state"].copy_(x["state"] * kept[..., None, None] + torch.matmul((kh * w[..., None]).transpose(-1, -2), v))
    return {"state": x["state"]}


def run(state):
    return _run_own(state) if own else _run_plain(state)


def work(case):
    B, H, N, dk, dv = (case[k] for k in ("B", "H", "N", "dk", "dv"))
    kind, size = case["kind"], _SIZE[case["dtype"]]
    tokens = sum(_lengths(case)) if case.get("padded") else B * N
    units, token_heads, state = B * H, tokens * H, 4 * dk * dv
    if kind == "prefill":
        read = token_heads * size * (2 * dk + dv) + (units * state if case["piece"] else 0)
        written = B * H * N * size * dv + units * state
        return {"bytes": read + written, "flops": token_heads * 4 * dk * dv}
    if kind == "train":
        # the forward reads Q, K, V and the backward those and dO
        read = token_heads * size * (4 * dk + 3 * dv)
        written = B * H * N * size * (2 * dk + 2 * dv)
        return {"bytes": read + written, "flops": token_heads * 14 * dk * dv}
    if kind == "step":
        return {"bytes": units * (2 * state + size * (2 * dk + 2 * dv)), "flops": units * 5 * dk * dv}
    if kind == "tree":
        return {"bytes": units * (state + size * N * (2 * dk + 2 * dv)),
                "flops": units * (2 * N * dk * dv + N * (N + 1) * (dk + dv))}
    # a path has about half as many tokens as the tree at most; three is what four drafts in a row come to
    return {"bytes": units * (2 * state + size * min(3, N) * (dk + dv)), "flops": units * (1 + 2 * min(3, N)) * dk * dv}


# ---- 64 bits, from the definition -----------------------------------------------------------------

def _exact_unit(x):
    x = x.double()
    n = torch.clamp(torch.linalg.vector_norm(x, dim=-1, keepdim=True), min=_EPS)
    return x / n, n


def _exact_rows(x):
    """Blocks of query rows against all keys up to them, head by head of every sequence."""
    case = x["case"]
    B, H, N, dk, dv = (case[k] for k in ("B", "H", "N", "dk", "dv"))
    train = case["kind"] == "train"
    dev = x["Q"].device
    O = torch.zeros((B, H, N, dv), dtype=torch.float64, device=dev)
    dQ, dK, dV = (torch.zeros(t.shape if train else (0,), dtype=torch.float64, device=dev) for t in (x["Q"], x["K"], x["V"]))
    ds = torch.zeros((B, H), dtype=torch.float64, device=dev)
    state = torch.zeros((B, H, dk, dv), dtype=torch.float64, device=dev)
    lens = _lengths(case) if case.get("padded") else [N] * B
    together = B if not case.get("padded") else 1
    for b0 in range(0, B, together):
        n = lens[b0]
        for h in range(H):
            ld = float(x["log_decay"][h])
            part = (slice(b0, b0 + together), h, slice(0, n))
            qh, qn = _exact_unit(x["Q"][part])
            kh, kn = _exact_unit(x["K"][part])
            v = x["V"][part].double()
            at = torch.arange(n, device=dev, dtype=torch.float64)
            sc = x["s"][b0, h].double() if case.get("padded") else x["s"][h].double()
            if train:
                g = x["dO"][part].double()
                gq, gk, gv = torch.zeros_like(qh), torch.zeros_like(kh), torch.zeros_like(v)
            step = max(64, min(n, int(2.0e8 / (together * n))))
            for i0 in range(0, n, step):
                i1 = min(n, i0 + step)
                apart = at[i0:i1, None] - at[None, :i1]
                w = torch.where(apart >= 0, torch.exp(ld * apart.abs()), torch.zeros_like(apart))
                p = torch.matmul(qh[:, i0:i1], kh[:, :i1].transpose(1, 2)) * w
                o = torch.matmul(p, v[:, :i1])
                if "state_in" in x:
                    o = o + torch.exp(ld * (at[i0:i1, None] + 1)) * torch.matmul(qh[:, i0:i1], x["state_in"][b0:b0 + together, h].double())
                O[b0:b0 + together, h, i0:i1] = sc * o
                if train:
                    a = torch.matmul(g[:, i0:i1], v[:, :i1].transpose(1, 2)) * w
                    gq[:, i0:i1] = torch.matmul(a, kh[:, :i1])
                    gk[:, :i1] += torch.matmul(a.transpose(1, 2), qh[:, i0:i1])
                    gv[:, :i1] += torch.matmul(p.transpose(1, 2), g[:, i0:i1])
                    ds[b0:b0 + together, h] += (o * g[:, i0:i1]).sum((1, 2))
            if train:
                dQ[part] = sc * (gq - qh * (qh * gq).sum(-1, keepdim=True)) / qn
                dK[part] = sc * (gk - kh * (kh * gk).sum(-1, keepdim=True)) / kn
                dV[part] = sc * gv
            else:
                w = torch.exp(ld * (n - 1 - at))[:, None]
                state[b0:b0 + together, h] = torch.matmul((kh * w).transpose(1, 2), v)
                if "state_in" in x:
                    state[b0:b0 + together, h] += math.exp(ld * n) * x["state_in"][b0:b0 + together, h].double()
    if train:
        return {"O": O, "dQ": dQ, "dK": dK, "dV": dV, "ds": ds if case.get("padded") else ds.sum(0)}
    return {"O": O, "state": state}


def exact(case, seed):
    x = prepare(case, seed)
    if case["kind"] in ("prefill", "train"):
        return _exact_rows(x)
    decay = torch.exp(x["log_decay"].double())
    kh, v, before = _exact_unit(x["K"])[0], x["V"].double(), x["state"].double()
    if case["kind"] == "step":
        if "parent" in x:
            before = x["state_in"].double()[x["parent"].long()]
        state = decay[:, None, None] * before + torch.einsum("bhk,bhv->bhkv", kh, v)
        o = torch.einsum("bhk,bhkv->bhv", _exact_unit(x["Q"])[0], state)
        return {"o": x["s"].double()[:, None] * o, "state": state}
    parent = x["parent"].cpu().numpy()
    B, T = parent.shape
    weights = np.full((B, T, T), -1, dtype=np.int64)                   # levels between, -1: not an ancestor
    depth = np.zeros((B, T), dtype=np.int64)
    for b in range(B):
        for i in range(T):
            j, up = i, 0
            while j >= 0:
                weights[b, i, j] = up
                j, up = parent[b, j], up + 1
            depth[b, i] = up - 1
    up = torch.from_numpy(weights).to(kh.device)
    levels = torch.from_numpy(depth).to(kh.device)
    if case["kind"] == "tree":
        w = torch.where(up[:, None] >= 0, decay[:, None, None] ** torch.clamp(up, min=0)[:, None].double(), 0.0)
        qh = _exact_unit(x["Q"])[0]
        o = decay[:, None, None] ** (levels[:, None, :, None] + 1.0) * torch.einsum("bhtk,bhkv->bhtv", qh, before)
        o = o + torch.einsum("bhij,bhjv->bhiv", torch.einsum("bhik,bhjk->bhij", qh, kh) * w, v)
        return {"o": x["s"].double()[:, None, None] * o}
    last = x["last"].cpu().tolist()
    state = before.clone()
    for b in range(B):
        if last[b] < 0:
            continue
        u = up[b, last[b]]
        w = torch.where(u >= 0, decay[:, None] ** torch.clamp(u, min=0).double(), 0.0)     # [H, T]
        state[b] = (decay ** (depth[b, last[b]] + 1.0))[:, None, None] * before[b] + torch.matmul(
            (kh[b] * w[..., None]).transpose(1, 2), v[b])
    return {"state": state}
