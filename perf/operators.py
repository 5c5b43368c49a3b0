"""Linear attention with a decay for each head (prompt, gradients, single tokens) and the AdamW step, as cases that can
be timed and compared.

    S_t = lambda S_{t-1} + k_t v_t^T,    o_t = scale S_t^T q_t          lambda = exp(log_decay), one for each state head

Query heads come in groups: `heads` query heads read `kv_heads` states, heads / kv_heads neighbours the same one.
Prompts are [B, T, heads, D], or rows of B sequences of different lengths one after the other (`packed`).

AdamW with bias corrections and decoupled weight decay over a list of tensors, moments in 32 bits or in 8: a block of
256 elements keeps the largest moment as its scale, a first moment is scale * sign(c) * (c / 127)^2 of a whole number
c, a second moment scale * (c / 255)^4 with c >= 1 wherever the moment is not zero.

`run` computes the plain form, or calls the library where `own` is true; `exact` is the definition in 64 bits.
"""
import math
import random

import torch

own = False

DEV = "cuda"
BLOCK = 256                                    # elements that share an 8-bit moment's scale
ADAM = {"lr": 1e-3, "beta1": 0.9, "beta2": 0.999, "eps": 1e-8, "weight_decay": 0.01, "step": 20}
_DT = {"f32": torch.float32, "bf16": torch.bfloat16}


# ---------------------------------------------------------------------------------------------------------------- cases
def listed():
    return [
        # a short prompt to a small model: one sequence, a few chunks a head; launches and latency
        {"name": "prompt_short", "op": "forward", "B": 1, "T": 200, "heads": 8, "kv_heads": 8, "Dk": 64, "Dv": 64,
         "dtype": "bf16", "packed": False, "carry": False},
        # one long document: a single sequence, so that its length has to be split to fill the chip
        {"name": "prompt_long", "op": "forward", "B": 1, "T": 32768, "heads": 32, "kv_heads": 32, "Dk": 128, "Dv": 128,
         "dtype": "bf16", "packed": False, "carry": False},
        # a server's batch of prompts of very different lengths, four query heads to a state, states carried on
        {"name": "prompt_packed_grouped", "op": "forward", "B": 24, "T": 20011, "heads": 32, "kv_heads": 8, "Dk": 128, "Dv": 128,
         "dtype": "bf16", "packed": True, "carry": True},
        # single precision (evaluation, reference runs), head sizes and a length that fill no tile
        {"name": "prompt_f32_odd", "op": "forward", "B": 3, "T": 1777, "heads": 6, "kv_heads": 6, "Dk": 72, "Dv": 100,
         "dtype": "f32", "packed": False, "carry": True},
        # gradients of an ordinary training batch
        {"name": "train_bf16", "op": "backward", "B": 8, "T": 4096, "heads": 16, "kv_heads": 16, "Dk": 128, "Dv": 128,
         "dtype": "bf16", "packed": False, "carry": False},
        # gradients in single precision of packed sequences with shared states, also through the carried state
        {"name": "train_f32_packed", "op": "backward", "B": 9, "T": 3001, "heads": 8, "kv_heads": 4, "Dk": 64, "Dv": 96,
         "dtype": "f32", "packed": True, "carry": True},
        # one new token of one sequence: latency alone
        {"name": "step_single", "op": "step", "B": 1, "slots": 1, "heads": 8, "kv_heads": 8, "Dk": 64, "Dv": 64, "dtype": "bf16"},
        # a token for each sequence of a full server, states at scattered places of a larger pool, some rows empty
        {"name": "step_batch", "op": "step", "B": 250, "slots": 300, "heads": 32, "kv_heads": 8, "Dk": 128, "Dv": 128, "dtype": "bf16"},
        # the recurrent network's own parameters (128 units, one input): three small tensors
        {"name": "adamw_rnn", "op": "adamw", "set": "rnn", "width": 128, "depth": 1, "param": "f32", "grad": "f32", "bits": 32, "copy": False},
        # a masked network of 784 positions and two layers of 2000 units, moments in 8 bits
        {"name": "adamw8_made", "op": "adamw", "set": "made", "width": 2000, "depth": 2, "param": "f32", "grad": "f32", "bits": 8, "copy": False},
        # a stack of layers of 1280 units trained in mixed precision: 32-bit weights and moments, bf16 gradients and copies
        {"name": "adamw_stack", "op": "adamw", "set": "stack", "width": 1280, "depth": 5, "param": "f32", "grad": "bf16", "bits": 32, "copy": True},
        # the same with moments in 8 bits and weights that exist in bf16 only, where memory is short
        {"name": "adamw8_stack", "op": "adamw", "set": "stack", "width": 1280, "depth": 5, "param": "bf16", "grad": "bf16", "bits": 8, "copy": False},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["forward", "forward", "backward", "backward", "step", "adamw"])
    if op == "adamw":
        kind = rng.choice(["rnn", "made", "stack"])
        width = {"rnn": _log_int(rng, 3, 128), "made": _log_int(rng, 100, 2048), "stack": _log_int(rng, 64, 1280)}[kind]
        depth = {"rnn": 1, "made": rng.randint(1, 3), "stack": rng.randint(1, 5)}[kind]
        param = rng.choice(["f32", "f32", "bf16"])
        return {"op": op, "set": kind, "width": width, "depth": depth, "param": param, "grad": rng.choice(["f32", "bf16"]),
                "bits": rng.choice([8, 32]), "copy": param == "f32" and rng.random() < 0.5}
    group = rng.choice([1, 1, 2, 4, 8])
    kv = _log_int(rng, 1, 32 // group)
    dims = [rng.choice([32, 64, 128, 128, rng.randint(1, 128)]) for _ in range(2)]
    c = {"op": op, "heads": kv * group, "kv_heads": kv, "Dk": dims[0], "Dv": dims[1], "dtype": rng.choice(["bf16", "bf16", "f32"])}
    if op == "step":
        c["B"] = _log_int(rng, 1, 250)
        c["slots"] = c["B"] + rng.randint(0, 50)
        return c
    c["packed"], c["carry"] = rng.random() < 0.5, rng.random() < 0.5
    c["B"] = _log_int(rng, 1, 32)
    rows = 32768 if op == "forward" else 24576                 # (with at most 32 heads: no dearer than the largest listed)
    if c["dtype"] == "f32":
        rows //= 4
    c["T"] = _log_int(rng, 1, rows if c["packed"] else rows // c["B"])
    return c


# --------------------------------------------------------------------------------------------------------------- inputs
def _lengths(case):
    """Lengths of the sequences; of packed ones they differ widely (one has no row, one has one), and a few rows are left."""
    B, T = case["B"], case["T"]
    if not case["packed"]:
        return [T] * B
    rng = random.Random(T * 131 + B)
    free = T - min(T // 8, 5)
    share = [rng.expovariate(1.0) for _ in range(B)]
    n = [int(free * s / sum(share)) for s in share]
    if B > 2:
        n[1], n[2] = 0, min(1, free)
    n[0] += free - sum(n) if free > sum(n) else 0
    return n


def _shapes(case):
    w, d = case["width"], case["depth"]
    if case["set"] == "rnn":
        return [(w, w), (w, 1), (w,)]
    if case["set"] == "made":
        dims = [784] + [w] * d + [784]
        return [s for a, b in zip(dims, dims[1:]) for s in ((b, a), (b,))]
    out = [(4001, w)]                                          # (an odd number of symbols)
    for _ in range(d):
        out += [(w, w)] * 4 + [(4 * w, w), (4 * w,), (w, 4 * w), (w,), (w,), (w,)]
    return out + [(w,)]


def _flat(shapes, dtype):
    """One zeroed buffer for tensors of these shapes, each at a multiple of 64 elements, and the tensors in it."""
    sizes = [math.prod(s) for s in shapes]
    at = [0]
    for n in sizes:
        at.append(at[-1] + -(-n // 64) * 64)
    buf = torch.zeros(at[-1], dtype=dtype, device=DEV)
    return buf, [buf[a:a + n].view(s) for a, n, s in zip(at, sizes, shapes)]


def _pad_blocks(x):
    n = x.numel()
    return torch.nn.functional.pad(x.reshape(-1), (0, -n % BLOCK)).reshape(-1, BLOCK)


def _quantise(m, v):
    """8-bit codes and scales of moments given in 64 bits: each element's nearest code."""
    n = m.numel()
    mb, vb = _pad_blocks(m), _pad_blocks(v)
    ms, vs = mb.abs().amax(1).float(), vb.amax(1).float()
    mr = (mb.abs() / ms.double().clamp_min(1e-300).unsqueeze(1)).sqrt() * 127.0
    vr = (vb / vs.double().clamp_min(1e-300).unsqueeze(1)).sqrt().sqrt() * 255.0
    mc = torch.floor(mr + 0.5).clamp_max(127.0) * torch.sign(mb)
    vc = torch.floor(vr + 0.5).clamp_max(255.0)
    vc = torch.where(vb > 0, vc.clamp_min(1.0), vc)
    return (mc.reshape(-1)[:n].to(torch.int8).reshape(m.shape), vc.reshape(-1)[:n].to(torch.uint8).reshape(v.shape), ms, vs)


def _values(mc, vc, ms, vs):
    """The moments that 8-bit codes stand for, in 64 bits."""
    n = mc.numel()
    c = _pad_blocks(mc.double())
    m = c * c.abs() * ms.double().unsqueeze(1) / 127.0 ** 2
    d = _pad_blocks(vc.double())
    v = (d * d) * (d * d) * vs.double().unsqueeze(1) / 255.0 ** 4
    return m.reshape(-1)[:n].reshape(mc.shape), v.reshape(-1)[:n].reshape(vc.shape)


def _inputs(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)

    def normal(*shape, std=1.0, dtype=torch.float32):
        return (torch.randn(*shape, generator=gen, device=DEV) * std).to(dtype)

    st = {"case": case}
    if case["op"] == "adamw":
        shapes = _shapes(case)
        eight = case["bits"] == 8
        st["all"] = {}
        for key, dtype in (("p", _DT[case["param"]]), ("g", _DT[case["grad"]]), ("m", torch.int8 if eight else torch.float32),
                           ("v", torch.uint8 if eight else torch.float32), ("copy", torch.bfloat16), ("mv", torch.float32),
                           ("vv", torch.float32)):
            if (key != "copy" or case["copy"]) and (key not in ("mv", "vv") or eight):
                st["all"][key], st[key] = _flat(shapes, dtype)
        st["ms"], st["vs"] = [], []
        for i, s in enumerate(shapes):
            st["p"][i].copy_(normal(*s, std=0.02))
            st["g"][i].copy_(normal(*s, std=1e-3))
            m = torch.zeros(s, device=DEV)                     # moments as a few steps of such gradients leave them
            v = torch.zeros(s, device=DEV)
            for _ in range(3):
                g = normal(*s, std=1e-3)
                m = 0.9 * m + 0.1 * g
                v = 0.999 * v + 0.001 * g * g
            if eight:
                m, v, ms, vs = _quantise(m.double(), v.double())
                st["ms"].append(ms)
                st["vs"].append(vs)
            st["m"][i].copy_(m)
            st["v"][i].copy_(v)
        return st

    dt, H, Hk, Dk, Dv, n = _DT[case["dtype"]], case["heads"], case["kv_heads"], case["Dk"], case["Dv"], case["B"]
    st["scale"] = Dk ** -0.5
    st["log_decay"] = -torch.exp2(-8.0 * torch.arange(1, Hk + 1, device=DEV, dtype=torch.float32) / Hk)
    if case["op"] == "step":
        for key, heads, D in (("q", H, Dk), ("k", Hk, Dk), ("v", Hk, Dv)):
            st[key] = normal(n, heads, D, dtype=dt)
        st["state"] = normal(case["slots"], Hk, Dk, Dv, std=3.0)
        st["o"] = torch.zeros(n, H, Dv, dtype=dt, device=DEV)
        slots = torch.randperm(case["slots"], generator=gen, device=DEV)[:n].to(torch.int32)
        if n > 8:
            slots[::9] = -1                                    # rows without a sequence
        st["slots"] = slots
        return st

    lead = (case["T"],) if case["packed"] else (n, case["T"])
    st["lengths"] = _lengths(case)
    st["offsets"] = None
    if case["packed"]:
        at = [0]
        for m in st["lengths"]:
            at.append(at[-1] + m)
        st["offsets"] = torch.tensor(at, dtype=torch.int32, device=DEV)
    for key, heads, D in (("q", H, Dk), ("k", Hk, Dk), ("v", Hk, Dv)):
        st[key] = normal(*lead, heads, D, dtype=dt)
    carry = case["carry"]
    st["state"] = normal(n, Hk, Dk, Dv) if carry else None
    if case["op"] == "forward":
        st["o"] = torch.zeros_like(st["q"][..., :1]).expand(*lead, H, Dv).contiguous()
        st["state_out"] = torch.empty(n, Hk, Dk, Dv, device=DEV) if carry else None
    else:
        st["do"] = normal(*lead, H, Dv, dtype=dt)
        st["dq"], st["dk"], st["dv"] = (torch.zeros_like(st[x]) for x in "qkv")
        st["d_state_out"] = normal(n, Hk, Dk, Dv) if carry else None
        st["d_state"] = torch.empty(n, Hk, Dk, Dv, device=DEV) if carry else None
    return st


def prepare(case, seed):
    """The inputs, and what a program of the library's keeps beside them: the marshalled call, or the workspace."""
    st = _inputs(case, seed)
    if not own:
        return st
    from paper_2002_03629_amd import binding as B
    if case["op"] == "adamw":
        eight = case["bits"] == 8
        st["plan"] = B.PreparedAdamW(st["p"], st["g"], st["m"], st["v"], st["ms"] if eight else None, st["vs"] if eight else None,
                                     st.get("copy"))
        return st
    sizes = (case["heads"], case["kv_heads"], case["Dk"], case["Dv"])
    if case["op"] == "step":
        st["plan"] = B.PreparedLinattnStep(st["q"], st["k"], st["v"], st["log_decay"], st["state"], st["slots"], case["B"], *sizes,
                                           st["scale"], st["o"])
        return st
    need = B.linattn_workspace_bytes(case["B"], case["T"], *sizes, _DT[case["dtype"]], packed=case["packed"],
                                     backward=case["op"] == "backward")
    st["workspace"] = torch.empty(need, dtype=torch.uint8, device=DEV)
    return st


# ----------------------------------------------------------------------------------------------------------- plain forms
CHUNK = 128


def _powers(log_decay, n):
    """exp(log_decay * n) for whole n >= 0 (1 for n = 0, also without any memory), one row for each head."""
    return torch.where(n == 0, torch.ones((), device=n.device, dtype=log_decay.dtype), torch.exp(log_decay.unsqueeze(-1) * n))


def _chunked(q, k, v, log_decay, state, late):
    """[B, H, T, D] in 32 bits, one state for each head: outputs without the factor `scale`, and the last state.
    late: a state enters a chunk's first step undecayed (the passes that go back in time)."""
    B, H, T, _ = q.shape
    out = torch.empty(B, H, T, v.shape[3], device=q.device)
    for a in range(0, T, CHUNK):
        n = min(CHUNK, T - a)
        i = torch.arange(n, device=q.device, dtype=torch.float32)
        diff = i.unsqueeze(1) - i.unsqueeze(0)
        mask = torch.where(diff >= 0, _powers(log_decay, diff.clamp_min(0).reshape(-1)).reshape(H, n, n), torch.zeros((), device=q.device))
        qc, kc, vc = q[:, :, a:a + n], k[:, :, a:a + n], v[:, :, a:a + n]
        scores = torch.matmul(qc, kc.transpose(2, 3).contiguous()) * mask
        out[:, :, a:a + n] = torch.matmul(scores, vc) + torch.matmul(qc, state) * _powers(log_decay, i + (1 - late)).unsqueeze(-1)
        kd = kc * _powers(log_decay, n - 1 + late - i).unsqueeze(-1)
        state = state * _powers(log_decay, torch.full((1,), float(n), device=q.device)).unsqueeze(-1) + \
            torch.matmul(kd.transpose(2, 3).contiguous(), vc)
    return out, state


def _sequences(case, lengths):
    """(first row, length, first sequence, number of sequences) of each group that can be computed at once."""
    if not case["packed"]:
        return [(0, case["T"], 0, case["B"])]
    at, out = 0, []
    for b, n in enumerate(lengths):
        out.append((at, n, b, 1))
        at += n
    return out


def _take(x, case, group):
    """[sequences, heads, length, D] in 32 bits of one such group."""
    at, n, _, _ = group
    x = x[at:at + n].unsqueeze(0) if case["packed"] else x
    return x.float().transpose(1, 2).contiguous()


def _put(out, y, case, group):
    at, n, _, _ = group
    y = y.transpose(1, 2).to(out.dtype)
    if case["packed"]:
        out[at:at + n] = y[0]
    else:
        out.copy_(y)


def _plain_forward(st):
    case, G = st["case"], st["case"]["heads"] // st["case"]["kv_heads"]
    ld = st["log_decay"].repeat_interleave(G)
    o = torch.zeros_like(st["o"])
    ends = []
    for group in _sequences(case, st["lengths"]):
        b, nb = group[2], group[3]
        q, k, v = (_take(st[x], case, group) for x in "qkv")
        s0 = st["state"][b:b + nb] if case["carry"] else torch.zeros(nb, case["kv_heads"], case["Dk"], case["Dv"], device=DEV)
        y, end = _chunked(q, k.repeat_interleave(G, 1), v.repeat_interleave(G, 1), ld, s0.repeat_interleave(G, 1), 0)
        _put(o, y * st["scale"], case, group)
        ends.append(end[:, ::G])
    return (o, torch.cat(ends)) if case["carry"] else o


def _plain_backward(st):
    case, G = st["case"], st["case"]["heads"] // st["case"]["kv_heads"]
    Hk, Dk, Dv, sc = case["kv_heads"], case["Dk"], case["Dv"], st["scale"]
    ld = st["log_decay"].repeat_interleave(G)
    grads = [torch.zeros_like(st[x]) for x in "qkv"]
    starts = []
    for group in _sequences(case, st["lengths"]):
        b, nb = group[2], group[3]
        q, k, v, do = (_take(st[x], case, group) for x in ("q", "k", "v", "do"))
        k, v = k.repeat_interleave(G, 1), v.repeat_interleave(G, 1)
        do = do * sc
        zero = torch.zeros(nb, Hk * G, Dk, Dv, device=DEV)
        s0 = st["state"][b:b + nb].repeat_interleave(G, 1) if case["carry"] else zero
        end = zero.clone()
        if case["carry"]:
            end[:, ::G] = st["d_state_out"][b:b + nb]                # (the shared state's gradient enters once)
        dq, _ = _chunked(do, v, k, ld, s0.transpose(2, 3).contiguous(), 0)
        qr, kr, vr, dr = (x.flip(2) for x in (q, k, v, do))
        dk, _ = _chunked(vr, dr, qr, ld, end.transpose(2, 3).contiguous(), 1)
        dv, start = _chunked(kr, qr, dr, ld, end, 1)
        dk, dv, start = (x.reshape(nb, Hk, G, *x.shape[2:]).sum(2) for x in (dk.flip(2), dv.flip(2), start))
        for out, y in zip(grads, (dq, dk, dv)):
            _put(out, y, case, group)
        starts.append(start)
    return tuple(grads) + ((torch.cat(starts),) if case["carry"] else ())


def _plain_step(st):
    case, G = st["case"], st["case"]["heads"] // st["case"]["kv_heads"]
    live = st["slots"] >= 0
    at = st["slots"][live].long()
    q, k, v = (st[x][live].float() for x in "qkv")
    lam = torch.exp(st["log_decay"]).reshape(1, -1, 1, 1)
    s = lam * st["state"][at] + k.unsqueeze(3) * v.unsqueeze(2)
    st["state"][at] = s
    y = (q.reshape(len(at), -1, G, case["Dk"], 1) * s.unsqueeze(2)).sum(3) * st["scale"]
    st["o"][live] = y.reshape(len(at), case["heads"], case["Dv"]).to(st["o"].dtype)
    return st["o"], st["state"]


def _adamw_outputs(st):
    keys = ("p", "m", "v") if st["case"]["bits"] == 32 else ("p", "mv", "vv")
    return [st["all"][x] for x in keys + (("copy",) if st["case"]["copy"] else ())]


def _plain_adamw(st):
    case, a = st["case"], ADAM
    b1, b2 = a["beta1"], a["beta2"]
    c1, c2 = 1.0 / (1.0 - b1 ** a["step"]), 1.0 / (1.0 - b2 ** a["step"])
    for i, p in enumerate(st["p"]):
        g = st["g"][i].float()
        if case["bits"] == 32:
            m = st["m"][i].mul_(b1).add_(g * (1.0 - b1))
            v = st["v"][i].mul_(b2).add_(g * g * (1.0 - b2))
        else:
            # (in 64 bits: a moment next to the border of two codes must fall on its own side)
            m, v = _values(st["m"][i], st["v"][i], st["ms"][i], st["vs"][i])
            g64 = g.double()
            m, v = b1 * m + (1.0 - b1) * g64, b2 * v + (1.0 - b2) * g64 * g64
            for key, x in zip(("m", "v", "ms", "vs"), _quantise(m, v)):
                st[key][i].copy_(x)
            mv, vv = _values(st["m"][i], st["v"][i], st["ms"][i], st["vs"][i])
            st["mv"][i].copy_(mv)
            st["vv"][i].copy_(vv)
            m, v = m.float(), v.float()
        new = p.float() * (1.0 - a["lr"] * a["weight_decay"]) - (a["lr"] * c1) * m / ((v * c2).sqrt() + a["eps"])
        p.copy_(new)
        if case["copy"]:
            st["copy"][i].copy_(new)
    return _adamw_outputs(st)


# ------------------------------------------------------------------------------------------------------------- one pass
def run(state):
    st, case = state, state["case"]
    if not own:
        return {"forward": _plain_forward, "backward": _plain_backward, "step": _plain_step, "adamw": _plain_adamw}[case["op"]](st)
    from paper_2002_03629_amd import binding as B
    if case["op"] == "step":
        st["plan"]()
        return st["o"], st["state"]
    if case["op"] == "adamw":
        a = ADAM
        st["plan"](a["lr"], a["beta1"], a["beta2"], a["eps"], a["weight_decay"], a["step"])
        if case["bits"] == 8:
            B.adamw_unpack(st["m"], st["v"], st["ms"], st["vs"], st["mv"], st["vv"])
        return _adamw_outputs(st)
    sizes = (case["B"], case["T"], case["heads"], case["kv_heads"], case["Dk"], case["Dv"], st["scale"])
    if case["op"] == "forward":
        B.linattn_forward(st["q"], st["k"], st["v"], st["log_decay"], st["state"], st["offsets"], *sizes, st["o"], st["state_out"],
                          workspace=st["workspace"])
        return (st["o"], st["state_out"]) if case["carry"] else st["o"]
    B.linattn_backward(st["q"], st["k"], st["v"], st["log_decay"], st["state"], st["offsets"], st["do"], st["d_state_out"], *sizes,
                       st["dq"], st["dk"], st["dv"], st["d_state"], workspace=st["workspace"])
    return (st["dq"], st["dk"], st["dv"]) + ((st["d_state"],) if case["carry"] else ())


def work(case):
    if case["op"] == "adamw":
        n = [math.prod(s) for s in _shapes(case)]
        p, g = (2 if case[x] == "bf16" else 4 for x in ("param", "grad"))
        each = 2 * p + g + (16 if case["bits"] == 32 else 4) + (2 if case["copy"] else 0)
        blocks = 0 if case["bits"] == 32 else 16 * sum(-(-x // BLOCK) for x in n)
        if case["bits"] == 8:
            each += 8                                          # (the values the new moments stand for are outputs too)
        return {"bytes": sum(n) * each + blocks, "flops": sum(n) * 16}
    e = 2 if case["dtype"] == "bf16" else 4
    H, Hk, Dk, Dv = case["heads"], case["kv_heads"], case["Dk"], case["Dv"]
    state = 4 * Hk * Dk * Dv
    if case["op"] == "step":
        rows = case["B"] - (len(range(0, case["B"], 9)) if case["B"] > 8 else 0)
        return {"bytes": rows * (2 * state + e * (H + Hk) * (Dk + Dv)), "flops": rows * (3 * Hk + 2 * H) * Dk * Dv}
    lengths = _lengths(case)
    rows = sum(lengths)
    # by the recurrence, or by all pairs where a sequence is shorter than its state is wide
    per_row = sum(n * min(2 * (H + Hk) * Dk * Dv, H * (n + 1) * (Dk + Dv)) for n in lengths)
    moved = rows * e * (H * (Dk + Dv) + Hk * (Dk + Dv))
    carried = 2 * state * case["B"] if case["carry"] else 0
    if case["op"] == "forward":
        return {"bytes": moved + carried, "flops": per_row}
    return {"bytes": 2 * moved - rows * e * H * Dv + (carried * 3 // 2 if case["carry"] else 0), "flops": 3 * per_row}


# ---------------------------------------------------------------------------------------------- the definition in 64 bits
def _pairs(ld, rows, cols, n):
    """lambda^(i - j) for j <= i of rows i and columns j, else 0."""
    d = rows.unsqueeze(1) - cols.unsqueeze(0)
    return torch.where(d >= 0, torch.exp(ld * d.clamp_min(0)), torch.zeros((), dtype=torch.float64, device=DEV))


def _exact_sequence(st, rows, b, out):
    """All pairs of steps of one sequence, head by head; rows: its rows in the arrays."""
    case, G, sc = st["case"], st["case"]["heads"] // st["case"]["kv_heads"], st["scale"]
    back = case["op"] == "backward"
    n = rows[1] - rows[0]

    def head(x, h):
        return (x[rows[0]:rows[1], h] if case["packed"] else x[b, :, h]).double()

    def place(y, x, h):
        (y[rows[0]:rows[1]] if case["packed"] else y[b])[:, h] = x

    t = torch.arange(n, device=DEV, dtype=torch.float64)
    for h in range(case["kv_heads"]):
        ld = st["log_decay"][h].double()
        k, v = head(st["k"], h), head(st["v"], h)
        s0 = st["state"][b, h].double() if case["carry"] else torch.zeros(case["Dk"], case["Dv"], dtype=torch.float64, device=DEV)
        into = torch.exp(ld * (t + 1)).unsqueeze(1)            # what is left of s0 at each step
        left = torch.exp(ld * (n - 1 - t)).unsqueeze(1)        # what is left of each step's product at the end
        if not back:
            if case["carry"]:
                out[1][b, h] = torch.exp(ld * n) * s0 + (k * left).t() @ v
        else:
            dk, dv = torch.zeros_like(k), torch.zeros_like(v)
            if case["carry"]:
                ds = st["d_state_out"][b, h].double()
                dk += left * (v @ ds.t())
                dv += left * (k @ ds)
                out[3][b, h] = torch.exp(ld * n) * ds
        for g in range(h * G, (h + 1) * G):
            q = head(st["q"], g)
            do = head(st["do"], g) if back else None
            y = torch.zeros(n, case["Dk"] if back else case["Dv"], dtype=torch.float64, device=DEV)
            for a in range(0, n, 4096):
                r = slice(a, min(a + 4096, n))
                lam = _pairs(ld, t[r], t[:r.stop], n)
                if not back:
                    y[r] = sc * ((q[r] @ k[:r.stop].t() * lam) @ v[:r.stop] + into[r] * (q[r] @ s0))
                else:
                    w = do[r] @ v[:r.stop].t() * lam
                    y[r] = sc * (w @ k[:r.stop] + into[r] * (do[r] @ s0.t()))
                    dk[:r.stop] += sc * (w.t() @ q[r])
                    dv[:r.stop] += sc * ((q[r] @ k[:r.stop].t() * lam).t() @ do[r])
            place(out[0], y, g)
            if back and case["carry"]:
                out[3][b, h] += sc * ((q * into).t() @ do)
        if back:
            place(out[1], dk, h)
            place(out[2], dv, h)


def exact(case, seed):
    st = _inputs(case, seed)

    def zeros(x):
        return torch.zeros(x.shape, dtype=torch.float64, device=DEV)

    if case["op"] in ("forward", "backward"):
        keys = ("o", "state_out") if case["op"] == "forward" else ("dq", "dk", "dv", "d_state")
        out = [zeros(st[x]) for x in keys if st[x] is not None]
        at = 0
        for b, n in enumerate(st["lengths"]):
            _exact_sequence(st, (at, at + n), b, out)
            at += n if case["packed"] else 0
        return tuple(out) if len(out) > 1 else out[0]
    if case["op"] == "step":
        G = case["heads"] // case["kv_heads"]
        o, state = zeros(st["o"]), st["state"].double()
        slots = st["slots"].tolist()
        for h in range(case["heads"]):
            lam = torch.exp(st["log_decay"][h // G].double())
            for r, s in enumerate(slots):
                if s < 0:
                    continue
                if h % G == 0:
                    state[s, h // G] = lam * state[s, h // G] + torch.outer(st["k"][r, h // G].double(), st["v"][r, h // G].double())
                o[r, h] = st["scale"] * (st["q"][r, h].double() @ state[s, h // G])
        return o, state
    a = ADAM
    flat = [_flat(_shapes(case), torch.float64) for _ in range(4 if case["copy"] else 3)]
    for i, p in enumerate(st["p"]):
        g = st["g"][i].double()
        if case["bits"] == 8:
            width = [math.ceil(g.numel() / BLOCK) * BLOCK]

            def spread(s):
                return s.double().repeat_interleave(BLOCK)[:g.numel()].reshape(g.shape)

            c = st["m"][i].double()
            m0 = torch.sign(c) * (c / 127.0) ** 2 * spread(st["ms"][i])
            v0 = (st["v"][i].double() / 255.0) ** 4 * spread(st["vs"][i])
        else:
            m0, v0 = st["m"][i].double(), st["v"][i].double()
        m = a["beta1"] * m0 + (1 - a["beta1"]) * g
        v = a["beta2"] * v0 + (1 - a["beta2"]) * g ** 2
        mh, vh = m / (1 - a["beta1"] ** a["step"]), v / (1 - a["beta2"] ** a["step"])
        p64 = p.double()
        new = p64 - a["lr"] * a["weight_decay"] * p64 - a["lr"] * mh / (vh ** 0.5 + a["eps"])
        if case["bits"] == 8:
            buf = torch.zeros(width, dtype=torch.float64, device=DEV)
            buf[:g.numel()] = m.reshape(-1)
            ms = spread(buf.reshape(-1, BLOCK).abs().max(1).values.float())
            buf[:g.numel()] = v.reshape(-1)
            vs = spread(buf.reshape(-1, BLOCK).max(1).values.float())
            c = torch.floor(127.0 * (m.abs() / ms) ** 0.5 + 0.5).clamp(0, 127)
            m = torch.sign(m) * (c / 127.0) ** 2 * ms
            c = torch.floor(255.0 * (v / vs) ** 0.25 + 0.5).clamp(1, 255)
            v = torch.where(v > 0, (c / 255.0) ** 4 * vs, torch.zeros_like(v))
        for (_, views), y in zip(flat, (new, m, v, new)):
            views[i].copy_(y)
    return [buf for buf, _ in flat]
