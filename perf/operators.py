"""The causal operators of a decoder as measurable cases: linear attention with a decay for each head (whole
prompts, training, single tokens) and the root-mean-square norm with the residual's addition.

A case is a dict of plain values:
  kind       "step"    one new token for each of B sequences, on a cache of states addressed by slots
             "prompt"  attention over whole prompts, with the states that they leave
             "train"   attention over whole sequences, with its gradients
             "norm"    the norm at inference (eight_bit: output in 8 bits with a scale for each row)
             "norm_train"  the norm with its gradients
  dtype      "bf16" or "f32" (storage of the large tensors; states, scales and parameters are float32)
  B H n dk dv           attention: sequences, heads, tokens, widths of queries and keys and of values
  layout     "bhnd": dense (B, H, n, d); "bnhd": heads side by side as a projection leaves them
  packed     prompt: True: B sequences of unequal lengths (n tokens in all) one behind the other in one tensor
  state      prompt, train: True: the sequences go on from a state that they had before
  rows cols residual    norm: size, and whether a residual is added

`own` false: plain forms of torch operations in float32, rounded once at the end; true: the framework's operators.
"""
import math

import numpy as np
import torch

own = False

EPS = 1e-6
# elements of the largest tensor of queries of a drawn prompt or training case, of the largest cache of states
# that a token goes through and of the largest tensor that is normed; the listed cases reach each of them
MOST_TOKENS = 2 * 16 * 65536 * 128
MOST_STATE = 256 * 16 * 128 * 128
MOST_NORM = 131072 * 2048


def _attention(kind, dtype, B, H, n, dk, dv, layout="bnhd", packed=False, state=False):
    return dict(kind=kind, dtype=dtype, B=B, H=H, n=n, dk=dk, dv=dv, layout=layout, packed=packed, state=state)


def _norm(kind, dtype, rows, cols, residual=True, eight_bit=False):
    return dict(kind=kind, dtype=dtype, rows=rows, cols=cols, residual=residual, eight_bit=eight_bit)


def listed():
    return [
        # one user's next token: the smallest call, latency is all
        dict(_attention("step", "bf16", 1, 8, 1, 64, 64), name="step_bf16_one"),
        # a server's next token for 256 users at once, large heads: the states' way through memory
        dict(_attention("step", "bf16", 256, 16, 1, 128, 128), name="step_bf16_256"),
        # two short prompts of no round length
        dict(_attention("prompt", "bf16", 2, 4, 1000, 64, 64), name="prompt_bf16_n1000"),
        # one prompt of 131072 tokens, few heads: the long axis has to be split
        dict(_attention("prompt", "bf16", 1, 8, 131072, 64, 64, layout="bhnd"), name="prompt_bf16_n131072"),
        # a server's batch of prompts of unequal lengths, packed, some of them going on from earlier tokens
        dict(_attention("prompt", "bf16", 24, 16, 65536, 128, 128, packed=True, state=True), name="prompt_bf16_packed"),
        # a training step of an ordinary model
        dict(_attention("train", "bf16", 4, 12, 16384, 64, 64), name="train_bf16_n16384"),
        # a training step of a large model on long sequences, each going on from the part before it
        dict(_attention("train", "bf16", 2, 16, 65536, 128, 128, state=True), name="train_bf16_n65536"),
        # a text classifier's training step in float32, small heads
        dict(_attention("train", "f32", 32, 4, 4000, 32, 32), name="train_f32_n4000"),
        # the norm before a projection in 8 bits, for the next token of eight users
        dict(_norm("norm", "bf16", 8, 512, eight_bit=True), name="norm_bf16_rows8"),
        # the same over the prompts of a large model
        dict(_norm("norm", "bf16", 131072, 2048, eight_bit=True), name="norm_bf16_131072"),
        # the norm between two blocks of a large model in training
        dict(_norm("norm_train", "bf16", 131072, 2048), name="norm_train_bf16"),
        # that of the text classifier, in float32
        dict(_norm("norm_train", "f32", 128000, 128), name="norm_train_f32"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choices(["step", "prompt", "train", "norm", "norm_train"], [3, 4, 4, 2, 2])[0]
    dtype = rng.choices(["bf16", "f32"], [3, 1])[0]
    if kind.startswith("norm"):
        cols = rng.choice([64, 128, 512, 1000, 1024, 2048, 2048, _log_int(rng, 33, 8192)])
        rows = _log_int(rng, 1, min(131072 * 12, MOST_NORM // cols))
        if dtype == "f32":
            rows = max(1, rows // 2)
        return _norm(kind, dtype, rows, cols, residual=rng.random() < 0.75, eight_bit=kind == "norm" and rng.random() < 0.5)
    H = rng.choice([1, 2, 4, 8, 12, 16])
    dk, dv = rng.choice([(64, 64), (64, 64), (128, 128), (128, 128), (64, 128), (32, 32), (16, 16), (48, 80)])
    if kind == "step":
        B = _log_int(rng, 1, max(1, min(512, MOST_STATE // (H * dk * dv))))
        return _attention(kind, dtype, B, H, 1, dk, dv)
    most = MOST_TOKENS // (4 if dtype == "f32" else 1) // (H * max(dk, dv))
    n = _log_int(rng, 1 if kind == "prompt" else 100, min(131072, most))
    packed = kind == "prompt" and n >= 64 and rng.random() < 0.4
    B = _log_int(rng, 2, min(64, n)) if packed else _log_int(rng, 1, max(1, min(64, most // n)))
    return _attention(kind, dtype, B, H, n, dk, dv, layout=rng.choice(["bhnd", "bnhd"]), packed=packed, state=rng.random() < 0.5)


def _dtype(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def _lengths(B, n, seed):
    """B lengths from a long tail, n in all; the first prompt is one token long and, of three or more, the second is empty."""
    rng = np.random.RandomState(seed % (1 << 31))
    w = rng.pareto(1.5, B) + 0.2
    w[0] = 0
    if B > 2:
        w[1] = 0
    cut = np.floor(np.cumsum(w) / w.sum() * (n - 1)).astype(np.int64)
    lengths = np.diff(np.concatenate([[0], cut]))
    lengths[0] = 1
    lengths[-1] += n - lengths.sum()
    return lengths


def prepare(case, seed):
    """Queries, keys and values as projections of normed activations leave them, with what neighbouring tokens have in common; keys of about unit length.
    The heads' decays go from a memory of 32 tokens to one of 4096, as of a fixed geometric schedule."""
    dev = torch.device("cuda")
    g = torch.Generator(device=dev).manual_seed(seed)
    dt = _dtype(case)

    def normal(*shape):
        return torch.randn(shape, generator=g, device=dev, dtype=torch.float32)

    state = dict(case=case)
    if case["kind"].startswith("norm"):
        rows, cols = case["rows"], case["cols"]
        # rows of unequal size and some columns that stand out
        tall = 1 + 7 * (torch.arange(cols, device=dev) % 61 == 5)
        x = normal(rows, cols) * tall
        state.update(x=x.to(dt), weight=1 + 0.2 * normal(cols), residual=None)
        if case["residual"]:
            state["residual"] = (normal(rows, cols) * torch.exp(0.5 * normal(rows, 1))).to(dt)
        if case["kind"] == "norm_train":
            state["dy"] = (0.1 * normal(rows, cols)).to(dt)
            state["dr"] = (0.1 * normal(rows, cols)).to(dt) if case["residual"] else None
            for name in ("x", "weight", "residual"):
                if state[name] is not None:
                    state[name].requires_grad_(True)
        return state

    B, H, n, dk, dv = (case[k] for k in ("B", "H", "n", "dk", "dv"))
    h = torch.arange(H, device=dev, dtype=torch.float32)
    state["log_decay"] = torch.log1p(-torch.exp2(-5 - 7 * h / max(1, H - 1)))
    state["scale"] = dk ** -0.5
    if case["kind"] == "step":
        slots = 2 * B
        q, k, v = normal(B, H, dk), normal(B, H, dk), normal(B, H, dv)
        state.update(q=q.to(dt), k=k.to(dt), v=v.to(dt), cache=2 * normal(slots, H, dk, dv),
                     slots=torch.randperm(slots, generator=g, device=dev)[:B].to(torch.int32))
        return state

    N = 1 if case["packed"] else B

    def tensor(d, gain=1.0):
        x = normal(N, n, H, d)
        x = (gain * (0.8 * x + 0.6 * x.roll(1, 1))).to(dt)
        return x.permute(0, 2, 1, 3) if case["layout"] == "bnhd" else x.permute(0, 2, 1, 3).contiguous()

    state.update(q=tensor(dk), k=tensor(dk), v=tensor(dv), offsets=None, initial=None)
    if case["packed"]:
        state["offsets"] = torch.tensor(np.concatenate([[0], np.cumsum(_lengths(B, n, seed))]), dtype=torch.int32, device=dev)
    if case["state"]:
        state["initial"] = 2 * normal(B, H, dk, dv)
    if case["kind"] == "train":
        state["dout"] = tensor(dv, 0.1)
        for name in ("q", "k", "v", "initial"):
            if state[name] is not None:
                state[name].requires_grad_(True)
        state["dfinal"] = 0.1 * normal(B, H, dk, dv) if case["state"] else None
    return state


# ---- plain forms -------------------------------------------------------------------------------

CHUNK = 256


def _plain_chunks(q, k, v, log_decay, scale, initial, index, same):
    """q, k, v (B, H, chunks, CHUNK, d) in float32: the output.  Within chunks as masked products, between them by one product with the powers of
    the chunks' decay.  index: a chunk's number in its sequence; same: whether two chunks are of one; initial: its sequence's state, for each chunk."""
    B, H, nc, _, dk = q.shape
    ld = log_decay.view(H, 1, 1)
    t = torch.arange(CHUNK, device=q.device)
    rel = t[:, None] - t[None, :]
    D = torch.where(rel >= 0, torch.exp(rel.clamp(min=0) * ld), 0.0)[:, None]
    out = ((q @ k.transpose(3, 4)) * D) @ v
    rel = index[:, None] - 1 - index[None, :]
    M = torch.where((rel >= 0) & same, torch.exp(rel.clamp(min=0) * CHUNK * ld), 0.0)
    left = (k * torch.exp((CHUNK - 1 - t)[:, None] * ld)[:, None]).transpose(3, 4) @ v
    S = (M @ left.reshape(B, H, nc, -1)).reshape(left.shape)
    if initial is not None:
        S = S + torch.exp(index * CHUNK * log_decay.view(H, 1))[..., None, None] * initial
    return scale * (out + torch.exp((t + 1)[:, None] * ld)[:, None] * (q @ S))


def _plain_attention(q, k, v, log_decay, scale, initial):
    """q, k, v (B, H, n, d) in float32: output and final state."""
    B, H, n, _ = q.shape
    nc = -(-n // CHUNK)
    ld = log_decay.view(H, 1)
    final = (k * torch.exp((n - 1 - torch.arange(n, device=q.device)) * ld)[..., None]).transpose(2, 3) @ v
    if initial is not None:
        final = final + torch.exp(n * ld)[..., None] * initial
        initial = initial[:, :, None]
    if n % CHUNK:
        q, k, v = (torch.nn.functional.pad(x, (0, 0, 0, nc * CHUNK - n)) for x in (q, k, v))
    q, k, v = (x.reshape(B, H, nc, CHUNK, x.shape[3]) for x in (q, k, v))
    index = torch.arange(nc, device=q.device)
    out = _plain_chunks(q, k, v, log_decay, scale, initial, index, torch.ones_like(index, dtype=torch.bool))
    return out.reshape(B, H, nc * CHUNK, v.shape[4])[:, :, :n], final


def _plain_packed(q, k, v, log_decay, scale, initial, offsets):
    """q, k, v (1, H, n, d) in float32, sequence b in rows offsets[b] to offsets[b + 1]: each begins a chunk of its own."""
    _, H, n, dk = q.shape
    B, ld, token = offsets.numel() - 1, log_decay.view(H, 1), torch.arange(n, device=q.device)
    lengths = offsets[1:] - offsets[:-1]
    of = torch.searchsorted(offsets, token, right=True) - 1
    chunks = (lengths + CHUNK - 1) // CHUNK
    first = chunks.cumsum(0) - chunks
    seq = torch.repeat_interleave(torch.arange(B, device=q.device), chunks)
    index = torch.arange(seq.numel(), device=q.device) - first[seq]
    row = first[of] * CHUNK + token - offsets[of]

    def spread(x):
        y = x.new_zeros(1, H, seq.numel() * CHUNK, x.shape[3])
        y[:, :, row] = x
        return y.reshape(1, H, seq.numel(), CHUNK, x.shape[3])
    w = torch.exp((offsets[1:][of] - 1 - token) * ld)
    v_chunks = spread(v)
    tails = spread(k * w[..., None]).transpose(3, 4) @ v_chunks
    final = q.new_zeros(B, H, dk, v.shape[3]).index_add(0, seq, tails[0].transpose(0, 1))
    if initial is not None:
        final = final + torch.exp(lengths[:, None] * log_decay)[..., None, None] * initial
        initial = initial[seq].transpose(0, 1)[None]
    out = _plain_chunks(spread(q), spread(k), v_chunks, log_decay, scale, initial, index, seq[:, None] == seq[None, :])
    return out.reshape(1, H, -1, v.shape[3])[:, :, row], final


def _plain(state):
    case = state["case"]
    dt = _dtype(case)
    if case["kind"] == "step":
        q, k, v = (state[n].float() for n in "qkv")
        at = state["slots"].long()
        S = torch.exp(state["log_decay"]).view(-1, 1, 1) * state["cache"][at] + k[..., None] * v[..., None, :]
        state["cache"][at] = S
        return dict(out=(state["scale"] * (q[..., None] * S).sum(2)).to(dt), cache=state["cache"])
    if case["kind"].startswith("norm"):
        train = case["kind"] == "norm_train"
        r = state["x"].detach()
        if case["residual"]:   # the stream is kept in the tensors' type, and the norm reads it as it is kept
            r = (r.float() + state["residual"].detach().float()).to(dt)
        w = state["weight"].detach()
        rf = r.float()
        rstd = torch.rsqrt(rf.square().mean(1, keepdim=True) + EPS)
        hat = rf * rstd
        y = hat * w
        res = dict(r=r) if case["residual"] else {}
        if case["eight_bit"]:
            most = y.abs().amax(1)
            scales = most / 448
            bits = (y * torch.where(most > 0, 448 / most, 1.0)[:, None]).to(torch.float8_e4m3fn)
            return dict(res, y=bits, scales=torch.where(most > 0, scales, 1.0))
        res["y"] = y.to(dt)
        if train:
            dy = state["dy"].float()
            gy = dy * w
            dx = rstd * (gy - hat * (gy * hat).mean(1, keepdim=True))
            if case["residual"]:
                dx = dx + state["dr"].float()
            res.update(dx=dx.to(dt), dweight=(dy * hat).sum(0))
        return res

    train = case["kind"] == "train"
    q, k, v = (state[n].detach().float() for n in "qkv")
    initial = None if state["initial"] is None else state["initial"].detach()
    common = (state["log_decay"], state["scale"])
    if not train:
        out, final = _plain_packed(q, k, v, *common, initial, state["offsets"].long()) if case["packed"] else _plain_attention(q, k, v, *common, initial)
        return dict(out=out.to(dt), final=final)
    leaves = [x.detach().requires_grad_(True) for x in (q, k, v, initial) if x is not None]
    out, final = _plain_attention(*leaves[:3], *common, leaves[3] if case["state"] else None)
    outs, backs = ((out, final), (state["dout"].float(), state["dfinal"])) if case["state"] else ((out,), (state["dout"].float(),))
    grads = torch.autograd.grad(outs, leaves, backs)
    res = dict(out=out.detach().to(dt), dq=grads[0].to(dt), dk=grads[1].to(dt), dv=grads[2].to(dt))
    if case["state"]:
        res.update(final=final.detach(), dinitial=grads[3])
    return res


# ---- the framework's operators -----------------------------------------------------------------

def _own(state):
    from paper_2507_08637_amd import autograd, binding
    case = state["case"]
    if case["kind"] == "step":
        out = binding.wersa_decay_step(state["q"], state["k"], state["v"], state["log_decay"], state["cache"], scale=state["scale"],
                                       slots=state["slots"])
        return dict(out=out, cache=state["cache"])
    if case["kind"] == "norm":
        if case["eight_bit"]:
            y, r, scales = binding.wersa_rms_norm_eight_bit(state["x"], state["weight"], residual=state["residual"], eps=EPS)
            return dict(y=y, scales=scales, **({"r": r} if case["residual"] else {}))
        y, r, _ = binding.wersa_rms_norm_forward(state["x"], state["weight"], residual=state["residual"], eps=EPS)
        return dict(y=y, **({"r": r} if case["residual"] else {}))
    if case["kind"] == "norm_train":
        if not case["residual"]:
            y = autograd.wersa_rms_norm(state["x"], state["weight"], eps=EPS)
            dx, dw = torch.autograd.grad(y, (state["x"], state["weight"]), state["dy"])
            return dict(y=y.detach(), dx=dx, dweight=dw)
        y, r = autograd.wersa_rms_norm(state["x"], state["weight"], residual=state["residual"], eps=EPS)
        dx, dw, _ = torch.autograd.grad((y, r), (state["x"], state["weight"], state["residual"]), (state["dy"], state["dr"]))
        return dict(y=y.detach(), r=r.detach(), dx=dx, dweight=dw)   # (the residual's gradient is the same tensor)
    if case["kind"] == "prompt":
        out, final, _ = binding.wersa_decay_forward(state["q"], state["k"], state["v"], state["log_decay"], scale=state["scale"],
                                                    offsets=state["offsets"], initial_state=state["initial"], want_state=True)
        return dict(out=out, final=final)
    leaves = [state[n] for n in ("q", "k", "v", "initial") if state[n] is not None]
    out, final = autograd.wersa_decay_attention(state["q"], state["k"], state["v"], state["log_decay"], scale=state["scale"],
                                                initial_state=state["initial"])
    outs, backs = ((out, final), (state["dout"], state["dfinal"])) if case["state"] else ((out,), (state["dout"],))
    grads = torch.autograd.grad(outs, leaves, backs)
    res = dict(out=out.detach(), dq=grads[0], dk=grads[1], dv=grads[2])
    if case["state"]:
        res.update(final=final.detach(), dinitial=grads[3])
    return res


def run(state):
    return _own(state) if own else _plain(state)


def work(case):
    """Bytes: every tensor that comes in and goes out, once.  Operations: the norm's per element; attention's in the recurrent form, which has the fewest:
    state update and read per token (2 dk dv each); backward: both again for dq, then the gradient state's update and its reads for dk and dv."""
    e = 4 if case["dtype"] == "f32" else 2
    if case["kind"].startswith("norm"):
        rows, cols = case["rows"], case["cols"]
        inout = 4 if case["residual"] else 2     # x, residual -> r, y
        nbytes = rows * cols * e * inout + 4 * cols
        if case["eight_bit"]:
            nbytes += rows * (cols * (1 - e) + 4)
        if case["kind"] == "norm_train":         # dy (dr) -> dx
            nbytes += rows * cols * e * (3 if case["residual"] else 2) + 4 * cols
        return {"bytes": nbytes, "flops": rows * cols * (14 if case["kind"] == "norm_train" else 5)}
    B, H, n, dk, dv = (case[k] for k in ("B", "H", "n", "dk", "dv"))
    state = 4 * B * H * dk * dv
    if case["kind"] == "step":
        return {"bytes": 2 * state + B * H * (2 * dk + 2 * dv) * e, "flops": 5 * B * H * dk * dv}
    tokens = H * n * (1 if case["packed"] else B)
    if case["kind"] == "prompt":
        return {"bytes": tokens * (2 * dk + 2 * dv) * e + state * (2 if case["state"] else 1), "flops": 4 * tokens * dk * dv}
    return {"bytes": tokens * (4 * dk + 4 * dv) * e + state * (4 if case["state"] else 0), "flops": 14 * tokens * dk * dv}


# ---- from the definitions, in 64 bits ----------------------------------------------------------

def _exact_attention(q, k, v, ld, scale, S0, dout=None, dfinal=None, block=512):
    """One sequence, (H, n, d) in float64: every pair of a row and an earlier one, block by block of rows."""
    H, n, dk = q.shape
    dv = v.shape[2]
    pos = torch.arange(n, device=q.device, dtype=torch.float64)
    out = torch.empty(H, n, dv, device=q.device, dtype=torch.float64)
    tail = torch.exp((n - 1 - pos) * ld[:, None])[..., None]       # of a row in the final state
    final = torch.matmul((k * tail).transpose(1, 2).contiguous(), v)
    if S0 is not None:
        final = final + torch.exp(n * ld)[:, None, None] * S0
    grads = None
    if dout is not None:
        dq, dk_, dv_ = torch.empty_like(q), torch.zeros_like(k), torch.zeros_like(v)
        dS0 = torch.zeros(H, dk, dv, device=q.device, dtype=torch.float64)
        if dfinal is not None:
            dk_ += tail * torch.matmul(v, dfinal.transpose(1, 2).contiguous())
            dv_ += tail * torch.matmul(k, dfinal)
            dS0 += torch.exp(n * ld)[:, None, None] * dfinal
    for i in range(0, n, block):
        j = min(n, i + block)
        rel = pos[i:j, None] - pos[None, :j]
        D = torch.exp(rel.clamp(min=0) * ld[:, None, None]).mul_(scale * (rel >= 0))
        A = torch.matmul(q[:, i:j], k[:, :j].transpose(1, 2)).mul_(D)
        out[:, i:j] = torch.matmul(A, v[:, :j])
        head = scale * torch.exp((pos[i:j] + 1) * ld[:, None])[..., None]
        if S0 is not None:
            out[:, i:j] += head * torch.matmul(q[:, i:j], S0)
        if dout is not None:
            g = dout[:, i:j]
            dv_[:, :j] += torch.matmul(A.transpose(1, 2), g)
            D.mul_(torch.matmul(g, v[:, :j].transpose(1, 2)))
            dq[:, i:j] = torch.matmul(D, k[:, :j])
            dk_[:, :j] += torch.matmul(D.transpose(1, 2), q[:, i:j])
            if S0 is not None:
                dq[:, i:j] += head * torch.matmul(g, S0.transpose(1, 2))
                dS0 += torch.matmul((head * q[:, i:j]).transpose(1, 2), g)
    if dout is not None:
        grads = dq, dk_, dv_, dS0
    return out, final, grads


def exact(case, seed):
    state = prepare(case, seed)
    wide = {n: x.detach().double() if torch.is_tensor(x) and x.is_floating_point() else x for n, x in state.items()}
    if case["kind"].startswith("norm"):
        if case["rows"] * case["cols"] > 1 << 29:
            return None
        r = wide["x"]
        res = {}
        if case["residual"]:
            r = (r + wide["residual"]).to(_dtype(case)).double()   # (the stream as it is kept is part of the definition)
            res["r"] = r
        w = wide["weight"]
        s = torch.sqrt(r.pow(2).sum(1, keepdim=True) / case["cols"] + EPS)
        y = w * r / s
        if case["eight_bit"]:
            most = y.abs().amax(1)
            return dict(res, y=None, scales=torch.where(most > 0, most / 448, 1.0))
        res["y"] = y
        if case["kind"] == "norm_train":
            gy = w * wide["dy"]
            dx = gy / s - r * (gy * r).sum(1, keepdim=True) / (case["cols"] * s.pow(3))
            res.update(dx=dx + wide["dr"] if case["residual"] else dx, dweight=(wide["dy"] * r / s).sum(0))
        return res
    ld, scale = wide["log_decay"], state["scale"]
    if case["kind"] == "step":
        at = state["slots"].long()
        S = torch.exp(ld)[:, None, None] * wide["cache"][at] + wide["k"].unsqueeze(3) * wide["v"].unsqueeze(2)
        wide["cache"][at] = S
        return dict(out=scale * (wide["q"].unsqueeze(3) * S).sum(2), cache=wide["cache"])
    B, H, n = case["B"], case["H"], case["n"]
    lengths = (state["offsets"][1:] - state["offsets"][:-1]).tolist() if case["packed"] else [n] * B
    # pairs of rows, times the products' width and number: about 20 T of them a second
    if sum(x * x for x in lengths) * H * (case["dk"] + case["dv"]) * (3 if case["kind"] == "train" else 1) > 1.5e14:
        return None
    outs, finals, grads = [], [], []
    begin = 0
    for b, length in enumerate(lengths):
        at = (0, slice(None), slice(begin, begin + length)) if case["packed"] else (b,)
        begin += length
        S0 = None if state["initial"] is None else wide["initial"][b]
        back = (wide["dout"][b], wide["dfinal"][b] if case["state"] else None) if case["kind"] == "train" else (None, None)
        o, f, gr = _exact_attention(*(wide[x][at].contiguous() for x in "qkv"), ld, scale, S0, *back)
        outs.append(o)
        finals.append(f)
        grads.append(gr)
    res = dict(out=torch.cat(outs, 1)[None] if case["packed"] else torch.stack(outs))
    if case["kind"] == "prompt" or case["state"]:
        res["final"] = torch.stack(finals)
    if case["kind"] == "train":
        res.update({name: torch.stack([gr[i] for gr in grads]) for i, name in enumerate(("dq", "dk", "dv"))})
        if case["state"]:
            res["dinitial"] = torch.stack([gr[3] for gr in grads])
    return res
