"""Operators of layers whose cost grows linearly with the length of their rows, as cases that can be timed.

A token mixer that looks at all earlier tokens costs the square of the length; two kinds do not, and what either makes joins the residual stream:

  window   causal attention in which a row sees the last `window` tokens up to itself and the first `sinks` tokens of its sequence
  linear   linear attention: one d x d state for each key/value head, S_t = lambda S_(t-1) + k_t v_t^T and o_t = scale S_t^T q_t, lambda = exp(log_decay)
           of the head
  dropout  what joins the residual stream: out = a + dropout(b + bias), its mask from a counter and never stored

`form` says which pass: "train" is forward and backward, "fwd" the forward pass alone, "step" a single token of each of many sequences, which reads and writes a
cache (window: a ring of rows behind the sinks; linear: the state).

`own` says which form run() computes: elementary torch operations, or the library's calls.
"""
import math

import torch

own = False

F32, BF16 = "f32", "bf16"


def _window(form, dtype, batch, seq, nq, nkv, d, window, sinks, rows=0, name=None):
    """form "step": seq is the largest position + 1 of a sequence, rows of its cache hold the sinks and the last rows - sinks tokens."""
    c = {"op": "window", "form": form, "dtype": dtype, "batch": batch, "seq": seq, "nq": nq, "nkv": nkv, "d": d, "window": window, "sinks": sinks, "rows": rows}
    return {**c, "name": name} if name else c


def _linear(form, dtype, batch, seq, nq, nkv, d, state=False, name=None):
    """state: the sequences go on from earlier ones, and the gradient of what they leave comes in (form "step" always goes on)."""
    c = {"op": "linear", "form": form, "dtype": dtype, "batch": batch, "seq": seq, "nq": nq, "nkv": nkv, "d": d, "state": state}
    return {**c, "name": name} if name else c


def _dropout(form, dtype, T, H, p, bias=True, name=None):
    c = {"op": "dropout", "form": form, "dtype": dtype, "T": T, "H": H, "p": p, "bias": bias}
    return {**c, "name": name} if name else c


def listed():
    return [
        # the float32 configuration: two short rows, kernels of a few microseconds
        _window("train", F32, 2, 64, 4, 4, 64, 16, 2, name="window_f32_tiny"),
        # multi-head attention of a small model, ragged length, heads of 64
        _window("train", BF16, 2, 2001, 8, 8, 64, 300, 4, name="window_train_d64"),
        # one long prompt on the few heads of a tensor-parallel shard
        _window("fwd", BF16, 1, 16384, 4, 1, 128, 4096, 4, name="window_fwd_shard"),
        # the heads of a whole 8B model, a training step
        _window("train", BF16, 1, 8192, 32, 8, 128, 1024, 16, name="window_train_whole"),
        # serving: a batch of sequences in bounded caches, some of them behind the ring's first turn
        _window("step", BF16, 64, 12000, 32, 8, 128, 4096, 4, rows=4608, name="window_step_batch"),
        # the float32 configuration
        _linear("train", F32, 2, 64, 4, 4, 64, name="linear_f32_tiny"),
        # a prompt on every head of a model
        _linear("fwd", BF16, 1, 8192, 32, 32, 128, name="linear_fwd_prompt"),
        # two rows in training, four query heads to a state, states passed on between pieces of a row
        _linear("train", BF16, 2, 4096, 32, 8, 128, state=True, name="linear_train_grouped"),
        # ragged rows, heads of 64, few blocks
        _linear("train", BF16, 3, 1999, 8, 8, 64, name="linear_train_d64"),
        # serving: a token of each of many sequences
        _linear("step", BF16, 128, 1000, 32, 32, 128, state=True, name="linear_step_batch"),
        # a short row: latency
        _dropout("train", BF16, 520, 4096, 0.1, name="dropout_small"),
        # the residual stream of a wide model
        _dropout("train", BF16, 16384, 8192, 0.1, name="dropout_wide"),
    ]


MOST_SCORES = 32 * 8192 ** 2  # the plain forms hold heads * batch * seq * seq numbers several times
MOST_FLOPS = 1.2e12           # a drawn case costs no more than the largest listed one
MOST_BYTES = 1.3e9


def _log_uniform(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


def draw(rng):
    op = rng.choice(["window", "window", "linear", "linear", "dropout"])
    while True:
        f32 = rng.random() < 0.2
        dtype, d = (F32, rng.choice([32, 64, 128])) if f32 else (BF16, rng.choice([64, 128, 128]))
        nkv = rng.choice([1, 1, 2, 4, 8])
        nq = nkv * rng.choice([1, 1, 2, 4, 8])
        if op == "dropout":
            c = _dropout(rng.choice(["train", "train", "fwd"]), dtype, int(_log_uniform(rng, 1, 16384)), 8 * int(_log_uniform(rng, 1, 1024)),
                         rng.choice([0.0, 0.05, 0.1, 0.1, 0.3, 0.5]), rng.random() < 0.7)
        elif rng.random() < 0.25:
            batch, seq = int(_log_uniform(rng, 1, 128)), int(_log_uniform(rng, 1, 20000))
            if op == "window":
                window, sinks = int(_log_uniform(rng, 1, 6000)), rng.choice([0, 1, 4, 16, 70])
                c = _window("step", dtype, batch, seq, nq, nkv, d, window, sinks, rows=window + sinks + rng.choice([0, 1, 100, 512]))
            else:
                c = _linear("step", dtype, batch, seq, nq, nkv, d, state=True)
        else:
            batch, seq = rng.choice([1, 1, 2, 3, 5]), int(_log_uniform(rng, 1, 1024 if f32 else 16384))
            form = rng.choice(["train", "train", "fwd"])
            if op == "window":
                c = _window(form, dtype, batch, seq, nq, nkv, d, int(_log_uniform(rng, 1, max(2, 1.2 * seq))), rng.choice([0, 1, 4, 16, 70, 200]))
            else:
                c = _linear(form, dtype, batch, seq, nq, nkv, d, state=rng.random() < 0.5)
            if nq > 32 or batch * nq * seq * seq > MOST_SCORES:
                continue
        if nq <= 32 and work(c)["flops"] <= MOST_FLOPS and work(c)["bytes"] <= MOST_BYTES:
            return c


# ------------------------------------------------------------------------------------------------ what a program has in hand
def _type(c):
    return torch.bfloat16 if c["dtype"] == BF16 else torch.float32


class State:
    pass


def prepare(case, seed):
    c, s = case, State()
    s.case = c
    gen = torch.Generator(device="cuda").manual_seed(seed)
    tt = _type(c)

    def normal(shape, std=1.0, dtype=tt):
        return torch.randn(shape, generator=gen, device="cuda", dtype=dtype).mul_(std)

    def positions():
        """Of each sequence's token: one in eight slots of the batch is not in use (-1), one in eight begins."""
        pos = torch.randint(0, c["seq"], (c["batch"],), generator=gen, device="cuda", dtype=torch.int32)
        kind = torch.rand(c["batch"], generator=gen, device="cuda")
        return torch.where(kind < 0.125, -1, torch.where(kind > 0.875, 0, pos)).to(torch.int32)

    if c["op"] == "dropout":
        T, H = c["T"], c["H"]
        s.a, s.b, s.dout = normal((T, H)), normal((T, H)), normal((T, H), 1e-2)
        s.bias = normal((H,), 0.1) if c["bias"] else None
        s.rng = torch.randint(0, 2 ** 31, (2,), generator=gen, device="cuda", dtype=torch.int64) * torch.tensor([2 ** 31 + 5, 1], device="cuda")  # key and step
        s.site = seed % 97
        s.out, s.dx = torch.zeros_like(s.a), torch.zeros_like(s.a)
        s.dbias = torch.zeros(H, device="cuda") if c["bias"] else None
    else:
        B, n, nq, nkv, d = c["batch"], 1 if c["form"] == "step" else c["seq"], c["nq"], c["nkv"], c["d"]
        s.qkv = normal((B * n, (nq + 2 * nkv) * d))
        s.o = torch.zeros((B * n, nq * d), dtype=tt, device="cuda")
        if c["form"] == "train":
            s.dout, s.dqkv = normal((B * n, nq * d), 1e-2), torch.zeros_like(s.qkv)
        if c["form"] == "step":
            s.pos = positions()
        if c["op"] == "window":
            s.qkv[:, :nq * d].mul_(2.0)  # scores a few units apart, as trained heads have
            if c["form"] == "step":
                s.kv = normal((B, c["rows"], 2 * nkv * d))
            else:
                s.lse, s.delta = torch.zeros((nq, B * n), device="cuda"), torch.zeros((nq, B * n), device="cuda")
        else:
            s.scale = 1.0 / math.sqrt(d)
            # memories of 4 to 1000 tokens, shared out over the heads
            s.log_decay = -torch.exp2(-2.0 - 8.0 * (torch.arange(nkv, device="cuda") + torch.rand(nkv, generator=gen, device="cuda")) / nkv)
            shape = (B, nkv, d, d)
            s.state_in = normal(shape, 1.0, torch.float32) if c["state"] else None
            if c["form"] != "step":
                s.state_out = torch.zeros(shape, device="cuda")
                s.dstate_out = normal(shape, 1e-2, torch.float32) if c["state"] and c["form"] == "train" else None
                s.dstate_in = torch.zeros(shape, device="cuda") if c["state"] and c["form"] == "train" else None
    if own:
        from paper_2411_15871_amd import dhelix as dh
        t, s.ws_bytes = dh.DH_BF16 if c["dtype"] == BF16 else dh.DH_F32, 0
        if c["op"] == "dropout":
            s.ws_bytes = dh.dh_dropout_add_bwd_ws_bytes(c["T"], c["H"])
        elif c["op"] == "window":
            if c["form"] == "step":
                s.ws_bytes = dh.dh_attn_window_step_workspace_bytes(t, B, c["rows"], c["window"], c["sinks"], nq, nkv, d)
            else:
                a = (t, B, n, c["window"], c["sinks"], nq, nkv, d)
                s.ws_bytes = max(dh.dh_attn_window_fwd_workspace_bytes(*a), dh.dh_attn_window_bwd_workspace_bytes(*a))
        elif c["form"] != "step":
            s.ws_bytes = max(dh.dh_linattn_fwd_workspace_bytes(t, B, n, nq, nkv, d), dh.dh_linattn_bwd_workspace_bytes(t, B, n, nq, nkv, d))
        s.ws = torch.zeros(max(16, s.ws_bytes), dtype=torch.uint8, device="cuda")
    return s


# ------------------------------------------------------------------------------------------------ the library's calls
def _own_window(c, s):
    from paper_2411_15871_amd import dhelix as dh
    t, st = dh.DH_BF16 if c["dtype"] == BF16 else dh.DH_F32, torch.cuda.current_stream()
    if c["form"] == "step":
        dh.dh_attn_window_step(t, c["batch"], c["rows"], c["window"], c["sinks"], c["nq"], c["nkv"], c["d"], s.pos, s.qkv, s.kv, s.o, s.ws, s.ws_bytes, st)
        return {"o": s.o, "kv": s.kv}
    a = (t, c["batch"], c["seq"], c["window"], c["sinks"], c["nq"], c["nkv"], c["d"])
    dh.dh_attn_window_fwd(*a, s.qkv, s.o, s.lse, s.ws, s.ws_bytes, st)
    if c["form"] == "fwd":
        return {"o": s.o, "lse": s.lse}
    dh.dh_attn_window_bwd(*a, s.qkv, s.o, s.dout, s.lse, s.dqkv, s.delta, s.ws, s.ws_bytes, st)
    return {"o": s.o, "lse": s.lse, "dqkv": s.dqkv}


def _own_linear(c, s):
    from paper_2411_15871_amd import dhelix as dh
    t, st = dh.DH_BF16 if c["dtype"] == BF16 else dh.DH_F32, torch.cuda.current_stream()
    if c["form"] == "step":
        dh.dh_linattn_step(t, c["batch"], c["nq"], c["nkv"], c["d"], s.scale, s.log_decay, s.pos, s.qkv, s.state_in, s.state_in, s.o, st)
        return {"o": s.o, "state": s.state_in}
    a = (t, c["batch"], c["seq"], c["nq"], c["nkv"], c["d"], s.scale, s.log_decay)
    dh.dh_linattn_fwd(*a, s.qkv, s.state_in, s.o, s.state_out, s.ws, s.ws_bytes, st)
    if c["form"] == "fwd":
        return {"o": s.o, "state": s.state_out}
    dh.dh_linattn_bwd(*a, s.qkv, s.state_in, s.dout, s.dstate_out, s.dqkv, s.dstate_in, s.ws, s.ws_bytes, st)
    r = {"o": s.o, "state": s.state_out, "dqkv": s.dqkv}
    return {**r, "dstate": s.dstate_in} if c["state"] else r


def _own_dropout(c, s):
    from paper_2411_15871_amd import dhelix as dh
    t, st = dh.DH_BF16 if c["dtype"] == BF16 else dh.DH_F32, torch.cuda.current_stream()
    dh.dh_dropout_add_fwd(t, c["T"], c["H"], s.a, s.b, s.bias, c["p"], s.rng, s.site, s.out, st)
    if c["form"] == "fwd":
        return {"out": s.out}
    dh.dh_dropout_add_bwd(t, c["T"], c["H"], s.dout, c["p"], s.rng, s.site, s.dx, s.dbias, False, s.ws, s.ws_bytes, st)
    r = {"out": s.out, "dx": s.dx}
    return {**r, "dbias": s.dbias} if c["bias"] else r


# ------------------------------------------------------------------------------------------------ the plain forms
def _t(x):
    return x.transpose(1, 2).contiguous()


def _rows_of(t, B, n):
    """[B * heads, n, d] -> [B * n, heads * d]"""
    return t.view(B, -1, n, t.shape[2]).transpose(1, 2).reshape(B * n, -1)


def _heads_of(t, B, heads, d):
    return t.float().view(B, -1, heads, d).transpose(1, 2).reshape(-1, t.shape[0] // B, d)


def _split(c, qkv, B):
    """q, k, v in float32 as [B * nq, n, d], keys and values repeated for the query heads of their group."""
    nq, nkv, d = c["nq"], c["nkv"], c["d"]
    q = _heads_of(qkv[:, :nq * d], B, nq, d)
    k, v = (_heads_of(t, B, nkv, d).repeat_interleave(nq // nkv, 0) for t in (qkv[:, nq * d:(nq + nkv) * d], qkv[:, (nq + nkv) * d:]))
    return q, k, v


def _grouped(c, t):
    """Sums over the query heads of a group."""
    return t.view(-1, c["nq"] // c["nkv"], *t.shape[1:]).sum(1)


def _plain_window(c, s):
    B, n, nq, d = c["batch"], c["seq"], c["nq"], c["d"]
    q, k, v = _split(c, s.qkv, B)
    at = torch.arange(n, device="cuda")
    seen = (at[None, :] <= at[:, None]) & ((at[None, :] > at[:, None] - c["window"]) | (at[None, :] < c["sinks"]))
    y = torch.matmul(q, _t(k)).mul_(1.0 / math.sqrt(d)).masked_fill_(~seen, -math.inf)
    top = y.amax(2, keepdim=True)
    p = y.sub_(top).exp_()
    total = p.sum(2, keepdim=True)
    p.div_(total)
    lse = (top + total.log()).view(B, nq, n).transpose(0, 1).reshape(nq, B * n)
    o = torch.matmul(p, v)
    r = {"o": _rows_of(o, B, n).to(_type(c)), "lse": lse}
    if c["form"] == "fwd":
        return r
    do = _heads_of(s.dout, B, nq, d)
    delta = (do * _heads_of(r["o"], B, nq, d)).sum(2, keepdim=True)  # of the outputs as they are kept
    dv = torch.matmul(_t(p), do)
    ds = torch.matmul(do, _t(v)).sub_(delta).mul_(p).mul_(1.0 / math.sqrt(d))
    dq, dk = torch.matmul(ds, k), torch.matmul(_t(ds), q)
    r["dqkv"] = torch.cat([_rows_of(dq, B, n), _rows_of(_grouped(c, dk), B, n), _rows_of(_grouped(c, dv), B, n)], 1).to(_type(c))
    return r


def _row_of(c, pos):
    """The cache's row of a position."""
    return torch.where(pos < c["rows"], pos, c["sinks"] + (pos - c["sinks"]) % max(1, c["rows"] - c["sinks"]))


def _plain_window_step(c, s):
    B, nq, nkv, d, w, n = c["batch"], c["nq"], c["nkv"], c["d"], c["window"], c["sinks"]
    pos, each = s.pos.long(), torch.arange(B, device="cuda")
    on = pos >= 0
    row = _row_of(c, pos.clamp(min=0))
    s.kv[each, row] = torch.where(on[:, None], s.qkv[:, nq * d:], s.kv[each, row])
    col = torch.arange(n + w, device="cuda")
    j = torch.where(col < n, col, pos[:, None] - w + 1 + col - n)
    seen = (j <= pos[:, None]) & ((col < n) | (j >= n))
    kv = s.kv[each[:, None], _row_of(c, j.clamp(min=0)).clamp(max=c["rows"] - 1)].float().view(B, n + w, 2, nkv, d)
    k, v = (kv[:, :, i].transpose(1, 2).reshape(B * nkv, n + w, d) for i in (0, 1))
    q = s.qkv[:, :nq * d].float().reshape(B * nkv, nq // nkv, d)
    y = torch.matmul(q, _t(k)).mul_(1.0 / math.sqrt(d)).view(B, nq, n + w).masked_fill_(~seen[:, None, :], -math.inf)
    p = (y - y.amax(2, keepdim=True).clamp(min=-1e30)).exp()
    p = (p / p.sum(2, keepdim=True).clamp(min=1e-30)).view(B * nkv, nq // nkv, n + w)
    o = torch.matmul(p, v).view(B, nq * d).to(_type(c))
    return {"o": torch.where(on[:, None], o, s.o), "kv": s.kv}


def _powers(c, s, B, n):
    """lambda^0 .. lambda^n of each query head of the batch, [B * nq, n + 1]."""
    p = torch.exp(s.log_decay.double()[:, None] * torch.arange(n + 1, device="cuda")).float()
    return p.repeat_interleave(c["nq"] // c["nkv"], 0).repeat(B, 1)


def _plain_linear(c, s):
    B, n, nq, nkv, d = c["batch"], c["seq"], c["nq"], c["nkv"], c["d"]
    q, k, v = _split(c, s.qkv, B)
    first = slice(None, None, nq // nkv)  # a query head of each group: its keys and values
    power = _powers(c, s, B, n)
    at = torch.arange(n, device="cuda")
    apart = at[:, None] - at[None, :]
    weight = power[:nq, :n][:, apart.clamp(min=0)].masked_fill_(apart < 0, 0.0).mul_(s.scale).repeat(B, 1, 1)  # scale lambda^(t - j)
    up, down = power[:, 1:, None], power[:, :n].flip(1)[:, :, None]  # lambda^(t + 1), lambda^(n - 1 - t)
    scores = torch.matmul(q, _t(k)).mul_(weight)
    o = torch.matmul(scores, v)
    state = torch.matmul(_t(k[first]), v[first] * down[first])
    if c["state"]:
        before = s.state_in.view(B * nkv, d, d).repeat_interleave(nq // nkv, 0)
        o += torch.matmul(q * (up * s.scale), before)
        state += power[first, n, None, None] * s.state_in.view(B * nkv, d, d)
    r = {"o": _rows_of(o, B, n).to(_type(c)), "state": state.view(B, nkv, d, d)}
    if c["form"] == "fwd":
        return r
    do = _heads_of(s.dout, B, nq, d)
    dv = _grouped(c, torch.matmul(_t(scores), do))
    g = torch.matmul(do, _t(v)).mul_(weight)
    dq, dk = torch.matmul(g, k), _grouped(c, torch.matmul(_t(g), q))
    if c["state"]:
        behind = s.dstate_out.view(B * nkv, d, d)
        dq += torch.matmul(do * (up * s.scale), _t(before))
        dk += torch.matmul(v[first] * down[first], _t(behind))
        dv += torch.matmul(k[first] * down[first], behind)
        ds = _grouped(c, torch.matmul(_t(q * (up * s.scale)), do)) + power[first, n, None, None] * behind
        r["dstate"] = ds.view(B, nkv, d, d)
    r["dqkv"] = torch.cat([_rows_of(dq, B, n), _rows_of(dk, B, n), _rows_of(dv, B, n)], 1).to(_type(c))
    return r


def _plain_linear_step(c, s):
    B, nq, nkv, d = c["batch"], c["nq"], c["nkv"], c["d"]
    x = s.qkv.float()
    q, k, v = x[:, :nq * d].view(B, nkv, nq // nkv, d), x[:, nq * d:(nq + nkv) * d].view(B, nkv, d, 1), x[:, (nq + nkv) * d:].view(B, nkv, 1, d)
    old = torch.where((s.pos == 0)[:, None, None, None], 0.0, s.state_in)
    new = old * s.log_decay.double().exp().float()[:, None, None] + k * v
    on = s.pos >= 0
    o = (torch.matmul(q, new) * s.scale).reshape(B, nq * d).to(_type(c))
    s.state_in.copy_(torch.where(on[:, None, None, None], new, s.state_in))
    return {"o": torch.where(on[:, None], o, s.o), "state": s.state_in}


def _plain_philox(key, step, site, vectors):
    """Philox4x32-10 of the counters (vector low, vector high, step, site): [vectors, 4], 32 bits each, in int64 (whose products keep the low 64 bits)."""
    low = 0xFFFFFFFF
    v = torch.arange(vectors, device="cuda")
    x0, x1, x2, x3 = v & low, v >> 32, torch.full_like(v, 0) + (step & low), torch.full_like(v, site)
    k0, k1 = key & low, (key >> 32) & low
    for _ in range(10):
        p, r = x0 * 0xD2511F53, x2 * 0xCD9E8D57
        x0, x1, x2, x3 = ((r >> 32) & low) ^ x1 ^ k0, r & low, ((p >> 32) & low) ^ x3 ^ k1, p & low
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    return torch.stack([x0, x1, x2, x3], 1)


def _plain_dropout(c, s):
    T, H, tt = c["T"], c["H"], _type(c)
    drop = round(c["p"] * 65536)  # of 65536 values of an element's 16 bits
    words = _plain_philox(s.rng[0], s.rng[1], s.site, T * H // 8)
    keep = (torch.stack([words & 0xFFFF, words >> 16], 2) >= drop).view(T, H)
    factor = 65536.0 / (65536 - drop)
    x = s.b.float()
    if c["bias"]:
        x += s.bias.float()
    r = {"out": torch.where(keep, x.mul_(factor), 0.0).add_(s.a).to(tt)}
    if c["form"] == "fwd":
        return r
    g = torch.where(keep, s.dout.float() * factor, 0.0)
    r["dx"] = g.to(tt)
    return {**r, "dbias": g.sum(0, dtype=torch.float64).float()} if c["bias"] else r


def run(state):
    c = state.case
    if own:
        return {"window": _own_window, "linear": _own_linear, "dropout": _own_dropout}[c["op"]](c, state)
    if c["op"] == "dropout":
        return _plain_dropout(c, state)
    if c["op"] == "window":
        return (_plain_window_step if c["form"] == "step" else _plain_window)(c, state)
    return (_plain_linear_step if c["form"] == "step" else _plain_linear)(c, state)


# ------------------------------------------------------------------------------------------------ what a pass cannot do without
def _pairs(n, window, sinks):
    """(row, key) pairs that the mask leaves in a sequence of n rows: of the window, and of the sinks before it."""
    full = max(0, n - window)
    of_window = n * (n + 1) // 2 - full * (full + 1) // 2
    m = min(sinks, full)  # rows window .. n - 1 have 1, 2, ... tokens before their window
    return of_window + m * (m + 1) // 2 + (full - m) * m


def work(case):
    c = case
    size = 2 if c["dtype"] == BF16 else 4
    train = c["form"] == "train"
    if c["op"] == "dropout":
        n = c["T"] * c["H"]
        return {"bytes": (5 if train else 3) * n * size + (c["H"] * (size + 4 * train) if c["bias"] else 0), "flops": (5 if train else 3) * n}
    B, n, nq, nkv, d = c["batch"], c["seq"], c["nq"], c["nkv"], c["d"]
    if c["form"] == "step":
        rows = B * (2 * nq + 2 * nkv) * d * size + 4 * B
        if c["op"] == "window":  # a sequence sees as many rows as fit, on the average over its positions
            seen = _pairs(n, c["window"], c["sinks"]) / n
            return {"bytes": rows + B * (seen + 1) * 2 * nkv * d * size, "flops": B * seen * 4 * nq * d}
        return {"bytes": rows + 2 * 4 * B * nkv * d * d, "flops": B * (3 * nkv + 2 * nq) * d * d}
    T = B * n
    qkv, o = T * (nq + 2 * nkv) * d * size, T * nq * d * size
    if c["op"] == "window":
        return {"bytes": qkv + o + 4 * T * nq + (qkv + o if train else 0), "flops": (14 if train else 4) * B * nq * d * _pairs(n, c["window"], c["sinks"])}
    state = 4 * B * nkv * d * d
    # a token: the state's update and what each query head reads of it, and as much twice more behind
    return {"bytes": qkv + o + state * (2 if c["state"] else 1) + (2 * qkv + o + (2 * state if c["state"] else 0) if train else 0),
            "flops": 2 * T * d * d * ((nq + nkv) + (3 * nq + 2 * nkv if train else 0))}


# ------------------------------------------------------------------------------------------------ in 64 bits
def _exact_window(c, s):
    B, n, nq, nkv, d = c["batch"], c["seq"], c["nq"], c["nkv"], c["d"]
    x = s.qkv.double().view(B, n, nq + 2 * nkv, d)
    o, lse = torch.zeros((B, n, nq, d), dtype=torch.float64, device="cuda"), torch.zeros((nq, B, n), dtype=torch.float64, device="cuda")
    grads = torch.zeros_like(x)
    ahead = torch.ones((n, n), dtype=torch.bool, device="cuda").triu(1)
    behind = torch.ones((n, n), dtype=torch.bool, device="cuda").tril(-c["window"])
    behind[:, :c["sinks"]] = False
    hidden = ahead | behind
    for b in range(B):
        for h in range(nq):
            hk = nq + h // (nq // nkv)
            q, k, v = x[b, :, h], x[b, :, hk], x[b, :, hk + nkv]
            z = (q @ k.T / math.sqrt(d)).masked_fill(hidden, -math.inf)
            lse[h, b] = torch.logsumexp(z, 1)
            p = torch.softmax(z, 1)
            o[b, :, h] = p @ v
            if c["form"] == "train":
                g = s.dout.double().view(B, n, nq, d)[b, :, h]
                dz = p * (g @ v.T - (g * o[b, :, h]).sum(1, keepdim=True)) / math.sqrt(d)
                grads[b, :, h] = dz @ k
                grads[b, :, hk] += dz.T @ q
                grads[b, :, hk + nkv] += p.T @ g
    r = {"o": o.view(B * n, -1), "lse": lse.view(nq, B * n)}
    return {**r, "dqkv": grads.view(B * n, -1)} if c["form"] == "train" else r


def _exact_window_step(c, s):
    B, nq, nkv, d, w, n = c["batch"], c["nq"], c["nkv"], c["d"], c["window"], c["sinks"]
    o = torch.zeros((B, nq, d), dtype=torch.float64, device="cuda")
    kv = s.kv.double()
    for b, p in enumerate(s.pos.tolist()):
        if p < 0:
            continue
        seen = torch.tensor([j for j in range(p + 1) if j < n or j > p - w], device="cuda")
        turn = c["rows"] - n
        rows = seen if p < c["rows"] else torch.where(seen < c["rows"], seen, seen % turn if n == 0 else n + (seen - n) % turn)
        at = int(rows[-1])
        kv[b, at] = s.qkv[b, nq * d:].double()
        k, v = kv[b, rows].view(len(rows), 2, nkv, d).unbind(1)
        q = s.qkv[b, :nq * d].double().view(nkv, nq // nkv, d)
        weights = torch.softmax(torch.matmul(q, k.permute(1, 2, 0).contiguous()) / math.sqrt(d), 2)
        o[b] = torch.matmul(weights, v.permute(1, 0, 2).contiguous()).view(nq, d)
    return {"o": o.view(B, -1), "kv": kv}


def _exact_linear(c, s):
    """The recurrence itself, token by token."""
    B, n, nq, nkv, d = c["batch"], c["seq"], c["nq"], c["nkv"], c["d"]
    grp = nq // nkv
    x = s.qkv.double().view(B, n, -1).transpose(0, 1).contiguous()
    q, k, v = x[..., :nq * d].reshape(n, B * nkv, grp, d), x[..., nq * d:(nq + nkv) * d].reshape(n, B * nkv, d, 1), x[..., (nq + nkv) * d:].reshape(n, B * nkv, d, 1)
    lam = torch.exp(s.log_decay.double()).repeat(B)[:, None, None]
    zero = torch.zeros((B * nkv, d, d), dtype=torch.float64, device="cuda")
    S = s.state_in.double().view(-1, d, d) if c["state"] else zero
    o, dq, dk, dv = torch.zeros_like(q), torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    g = s.dout.double().view(B, n, -1).transpose(0, 1).reshape(n, B * nkv, grp, d) if c["form"] == "train" else None
    for t in range(n):
        S = lam * S + k[t] * v[t].transpose(1, 2)
        o[t] = torch.matmul(q[t], S)
        if g is not None:
            dq[t] = torch.matmul(g[t], S.transpose(1, 2).contiguous())

    def rows(t, heads):
        return t.reshape(n, B, heads * d).transpose(0, 1).reshape(B * n, heads * d)

    r = {"o": s.scale * rows(o, nq), "state": S.view(B, nkv, d, d)}
    if g is None:
        return r
    R = s.dstate_out.double().view(-1, d, d) if c["state"] else zero
    for t in reversed(range(n)):
        R = R + s.scale * torch.matmul(q[t].transpose(1, 2).contiguous(), g[t])
        dk[t], dv[t] = torch.matmul(R, v[t]), torch.matmul(R.transpose(1, 2).contiguous(), k[t])
        R = lam * R
    r["dqkv"] = torch.cat([s.scale * rows(dq, nq), rows(dk, nkv), rows(dv, nkv)], 1)
    return {**r, "dstate": R.view(B, nkv, d, d)} if c["state"] else r


def _exact_linear_step(c, s):
    B, nq, nkv, d = c["batch"], c["nq"], c["nkv"], c["d"]
    S, o = s.state_in.double(), torch.zeros((B, nq, d), dtype=torch.float64, device="cuda")
    x = s.qkv.double().view(B, nq + 2 * nkv, d)
    for b, p in enumerate(s.pos.tolist()):
        if p >= 0:
            kv = x[b, nq:nq + nkv, :, None] * x[b, nq + nkv:, None, :]
            S[b] = kv + (S[b] * torch.exp(s.log_decay.double())[:, None, None] if p > 0 else 0.0)
            o[b] = s.scale * torch.matmul(x[b, :nq].view(nkv, -1, d), S[b]).view(nq, d)
    return {"o": o.view(B, -1), "state": S}


def _exact_keep(c, s):
    """The mask, with products of 32 bits made of 16-bit halves."""
    def product(x, m):
        a, b, e, f = x >> 16, x & 0xFFFF, m >> 16, m & 0xFFFF
        low = b * f
        mid = a * f + (low >> 16)
        up = b * e + (mid & 0xFFFF)
        return a * e + (mid >> 16) + (up >> 16), (up & 0xFFFF) * 65536 + (low & 0xFFFF)

    key, step = (int(v) % 2 ** 64 for v in s.rng.tolist())
    n = c["T"] * c["H"] // 8
    words = []
    for first in range(0, n, 1 << 22):
        c0 = torch.arange(first, min(n, first + (1 << 22)), device="cuda")
        c1, c2, c3 = torch.zeros_like(c0), torch.full_like(c0, step % 2 ** 32), torch.full_like(c0, s.site)
        for i in range(10):
            k0, k1 = ((key % 2 ** 32) + i * 0x9E3779B9) % 2 ** 32, ((key >> 32) + i * 0xBB67AE85) % 2 ** 32
            (h0, l0), (h1, l1) = product(c0, 0xD2511F53), product(c2, 0xCD9E8D57)
            c0, c1, c2, c3 = h1 ^ c1 ^ k0, l1, h0 ^ c3 ^ k1, l0
        words += [torch.stack([w for x in (c0, c1, c2, c3) for w in (x % 65536, x // 65536)], 1).to(torch.int32)]
    return torch.cat(words).view(c["T"], c["H"]) >= int(65536 * c["p"] + 0.5)


def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["op"] == "window":
        return (_exact_window_step if c["form"] == "step" else _exact_window)(c, s)
    if c["op"] == "linear":
        return (_exact_linear_step if c["form"] == "step" else _exact_linear)(c, s)
    mask = _exact_keep(c, s).double() / (1.0 - int(65536 * c["p"] + 0.5) / 65536.0)
    x = s.b.double() if s.bias is None else s.b.double() + s.bias.double()
    r = {"out": s.a.double() + mask * x}
    if c["form"] == "fwd":
        return r
    r["dx"] = mask * s.dout.double()
    return r if s.bias is None else {**r, "dbias": r["dx"].sum(0)}
