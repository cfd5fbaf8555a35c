"""The layers that stand between the MoBA layers of a hybrid model, as measurable cases.

The paper's models alternate: every other layer attends to a sliding window of the last keys and turns
its queries and keys by rotary positions, the rest are dense or MoBA.  Two operators make such a layer:

  rope      rotary positions of queries and keys: forward, or its gradient (the turn backwards)
  forward   attention of every position to the last `window` keys up to itself (0: to all of them),
            as prefill, or for the last `q_len` positions against a cache
  train     the same followed by its backward pass, which recomputes the probabilities

Both forms are here: the plain one in elementary torch operations in 32 bits, and the calls of the
library's own operators.  Sizes are those of the configurations in ``workloads.py`` and of the sweep,
decode and packed-batch modes of ``bench.py``, the paper's window of 256, and odd relatives of them.
"""
import math

import torch

own = False

ROPE_KEYS = ("rot_dim", "interleaved", "theta", "scale_factor", "orig_len", "band_low", "band_high", "amplitude",
             "position0")


def _rope(batch, heads, kv_heads, N, d, *, name=None, dtype="bf16", rot_dim=0, interleaved=False, theta=10000.0,
          scale_factor=1.0, orig_len=0, band_low=1.0, band_high=32.0, amplitude=1.0, position0=0, given=False,
          back=False):
    c = {"kind": "rope", "batch": batch, "heads": heads, "kv_heads": kv_heads, "N": N, "d": d, "dtype": dtype,
         "rot_dim": rot_dim or d, "interleaved": interleaved, "theta": theta, "scale_factor": scale_factor,
         "orig_len": orig_len, "band_low": band_low, "band_high": band_high, "amplitude": amplitude,
         "position0": position0, "given": given, "back": back}
    if name:
        c["name"] = name
    return c


def _window(kind, batch, heads, kv_heads, N, d, window, *, name=None, dtype="bf16", q_len=0, rows=0, lens=""):
    c = {"kind": kind, "batch": batch, "heads": heads, "kv_heads": kv_heads, "N": N, "d": d, "window": window,
         "dtype": dtype, "q_len": q_len or N, "rows": rows or N, "lens": lens}
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # one token of each sequence of a small serving batch, each at a position of its own: latency
        _rope(8, 16, 4, 1, 128, name="rope_tokens", given=True),
        # queries and keys of a training step of the headline length
        _rope(1, 16, 16, 32768, 64, name="rope_32k"),
        # a long document: part of the head turned, interleaved pairs, slow channels stretched eightfold,
        # gradients on their way back; the largest
        _rope(1, 16, 4, 131072, 128, name="rope_back_131k_partial", rot_dim=96, interleaved=True, theta=500000.0,
              scale_factor=8.0, orig_len=16384, amplitude=1.2079, back=True),
        # a serving step of a sliding-window layer against a cache with room to grow: latency
        _window("forward", 2, 16, 16, 32805, 64, 256, name="window_token", q_len=1, rows=33024),
        # a serving step of a dense layer with shared heads against a long cache, a few tokens at once
        _window("forward", 1, 16, 4, 131109, 128, 0, name="dense_4_tokens_131k", q_len=4, rows=131328),
        # prefill of a sliding-window layer
        _window("forward", 1, 16, 16, 8192, 64, 256, name="window_8k"),
        # prefill of a dense layer with shared heads
        _window("forward", 1, 16, 4, 16384, 128, 0, name="dense_16k_gqa_d128"),
        # a model's gradients checked at full precision
        _window("train", 1, 2, 2, 2048, 64, 256, name="window_train_f32_2k", dtype="f32"),
        # a packed batch of documents of very different lengths, odd sizes throughout
        _window("train", 1, 6, 6, 10081, 64, 1000, name="window_train_packed_10k",
                lens="3001,1300,17,1,4762,1000"),
        # a training step of the headline length with the paper's window
        _window("train", 1, 16, 16, 32768, 64, 256, name="window_train_32k"),
        # a training step of a dense layer
        _window("train", 2, 16, 16, 8192, 64, 0, name="dense_train_8k"),
        # long context, shared heads, a wide window: the largest
        _window("train", 1, 16, 4, 32768, 128, 2048, name="window_train_32k_wide_gqa_d128"),
    ]


def _spread(rng, lo, hi):
    """Log-uniform between lo and hi."""
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


def _pairs(c):
    """(query, key) pairs of one head and batch entry."""
    W = c["window"] or c["N"]
    if c["lens"]:
        seqs = [(n, n) for n in map(int, c["lens"].split(","))]
    else:
        seqs = [(c["N"], c["q_len"])]
    total = 0
    for n, q in seqs:
        first = n - q                                      # position of the first query
        ramp = max(0, min(W, n) - first)                   # queries that see fewer than W keys, and the first that sees W
        total += sum((first + 1, first + ramp)) * ramp // 2 + (q - ramp) * W
    return total


def draw(rng):
    while True:
        kind = rng.choice(["rope", "rope", "token", "forward", "train", "train"])
        d = rng.choice([64, 64, 128])
        kv = rng.choice([1, 2, 3, 4, 6, 8, 16])
        heads = kv * rng.choice([g for g in (1, 1, 2, 3, 4, 8) if kv * g <= 32])
        dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
        if kind == "rope":
            N = int(_spread(rng, 1, 131072.9))
            batch = int(_spread(rng, 1, 8.9))
            if batch * (heads + kv) * N * d * (2 if dtype == "bf16" else 4) > 20 * 131072 * 128 * 2:
                continue
            s = rng.choice([1.0, 1.0, 2.0, 8.0, 32.0])
            return _rope(batch, heads, kv, N, d, dtype=dtype, rot_dim=rng.choice([d, d, d // 2, 3 * d // 4, 32, 20, 2]),
                         interleaved=rng.random() < 0.5, theta=rng.choice([10000.0, 500000.0, 1000000.0]),
                         scale_factor=s, orig_len=rng.choice([0, 8192, 16384]),
                         amplitude=rng.choice([1.0, 1.0 + 0.1 * math.log(s)]),
                         position0=rng.choice([0, 0, int(_spread(rng, 1, 1e6))]), given=rng.random() < 0.3,
                         back=rng.random() < 0.5)
        if kind == "token":
            N = int(_spread(rng, 1, 131072.9))
            batch = int(_spread(rng, 1, 16.9))
            q_len = min(N, rng.choice([1, 1, 1, 2, 4, 7, 16]))
            c = _window("forward", batch, heads, kv, N, d, rng.choice([0, 256, int(_spread(rng, 1, 20000))]), dtype=dtype,
                        q_len=q_len, rows=N + rng.choice([0, 1, 27, 512]))
            if batch * kv * c["rows"] * d * (2 if dtype == "bf16" else 4) > 2e9:
                continue
        else:
            N = int(_spread(rng, 1, 65536.9))
            window = rng.choice([0, 256, int(_spread(rng, 1, 8192)), int(_spread(rng, 1, 8192))])
            lens = ""
            batch = int(_spread(rng, 1, 4.9))
            if rng.random() < 0.25:
                lens = ",".join(str(int(_spread(rng, 1, 8000))) for _ in range(rng.randint(1, 9)))
                N, batch = sum(map(int, lens.split(","))), 1
            q_len = N if lens or rng.random() < 0.8 else rng.randint(1, N)
            c = _window(kind, batch, heads, kv, N, d, window, dtype=dtype, q_len=q_len, lens=lens)
        bits = 2 if dtype == "bf16" else 4
        if batch * heads * _pairs(c) * d * bits > 16 * 32768 * 2048 * 128 * 2:
            continue
        return c


def _normal(g, shape, dtype):
    return torch.randn(shape, generator=g, dtype=torch.float32, device="cuda").to(dtype)


def _inputs(c, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = torch.bfloat16 if c["dtype"] == "bf16" else torch.float32
    b, h, hkv, N, d = c["batch"], c["heads"], c["kv_heads"], c["N"], c["d"]
    x = {}
    if c["kind"] == "rope":
        x["Q"], x["K"] = _normal(g, (b, h, N, d), dt), _normal(g, (b, hkv, N, d), dt)
        x["positions"] = None
        if c["given"]:                                     # every sequence of the batch goes on from a place of its own
            start = torch.randint(0, 131072, (b, 1), generator=g, device="cuda")
            x["positions"] = (start + torch.arange(N, device="cuda")).to(torch.int32)
        return x
    # normalised queries and keys, a few keys of which stand out, as attention's own do
    x["Q"] = _normal(g, (b, h, c["q_len"], d), dt)
    K = torch.randn((b, hkv, c["rows"], d), generator=g, device="cuda")
    K *= 1.0 + 1.5 * (torch.rand((b, hkv, c["rows"], 1), generator=g, device="cuda") < 0.02)
    x["K"], x["V"] = K.to(dt), _normal(g, (b, hkv, c["rows"], d), dt)
    if c["kind"] == "train":
        x["dO"] = _normal(g, (b, h, c["q_len"], d), dt)
    x["first"] = None
    if c["lens"]:                                          # a query sees keys of its own document only
        first, at = [], 0
        for n in map(int, c["lens"].split(",")):
            first += [at] * n
            at += n
        x["first"] = torch.tensor([first] * b, dtype=torch.int32, device="cuda")
    return x


def prepare(case, seed):
    st = _inputs(case, seed)
    st["case"] = c = dict(case)
    if own:
        import paper_2511_11571_amd as moba
        from paper_2511_11571_amd import binding
        code = binding.BF16 if c["dtype"] == "bf16" else binding.F32
        st["moba"] = moba
        if c["kind"] == "rope":
            st["shape"] = moba.RopeShape(c["batch"], c["heads"], c["N"], c["d"], kv_heads=c["kv_heads"], dtype=code,
                                         **{k: c[k] for k in ROPE_KEYS})
        else:
            st["shape"] = sh = moba.WindowShape(c["batch"], c["heads"], c["q_len"], c["N"], c["d"], window=c["window"],
                                                dtype=code, kv_heads=c["kv_heads"], kv_rows=c["rows"])
            fwd, bwd = moba.window_workspace_bytes(sh)
            need = max(fwd, bwd) if c["kind"] == "train" else fwd
            st["ws"] = torch.empty(max(need, 256), dtype=torch.uint8, device="cuda")
    return st


# ---- the plain forms ------------------------------------------------------------------------------------
def _frequencies(c):
    """Radians per position of every pair of channels, 64 bits, on the host."""
    freq = []
    for i in range(c["rot_dim"] // 2):
        f = c["theta"] ** (-2.0 * i / c["rot_dim"])
        if c["scale_factor"] != 1.0:
            keep = 0.0                                     # share of the pair's own speed
            if c["orig_len"] > 0:
                turns = c["orig_len"] * f / (2.0 * math.pi)
                keep = min(1.0, max(0.0, (turns - c["band_low"]) / (c["band_high"] - c["band_low"])))
            f *= keep + (1.0 - keep) / c["scale_factor"]
        freq.append(f)
    return freq


def _plain_rope(st):
    c = st["case"]
    freq = torch.tensor(_frequencies(c), dtype=torch.float64, device="cuda")
    if st["positions"] is not None:
        pos = st["positions"].double()[:, None, :, None]
    else:
        pos = (torch.arange(c["N"], device="cuda") + c["position0"]).double()[None, None, :, None]
    angle = pos * freq
    cos = (torch.cos(angle) * c["amplitude"]).float()
    sin = (torch.sin(angle) * (-c["amplitude"] if c["back"] else c["amplitude"])).float()
    r, out = c["rot_dim"], {}
    for name in ("Q", "K"):
        x = st[name].float()
        y = x.clone()
        if c["interleaved"]:
            a, b = x[..., 0:r:2], x[..., 1:r:2]
            y[..., 0:r:2] = a * cos - b * sin
            y[..., 1:r:2] = b * cos + a * sin
        else:
            a, b = x[..., :r // 2], x[..., r // 2:r]
            y[..., :r // 2] = a * cos - b * sin
            y[..., r // 2:r] = b * cos + a * sin
        out[name] = y.to(st[name].dtype)
    return out


def _plain_window(st):
    c = st["case"]
    b, h, hkv, N, d, q = c["batch"], c["heads"], c["kv_heads"], c["N"], c["d"], c["q_len"]
    G, W, scale, dt = h // hkv, c["window"] or N, 1.0 / math.sqrt(d), st["Q"].dtype
    train = c["kind"] == "train"
    Q = st["Q"].view(b, hkv, G, q, d)
    K, V = st["K"][:, :, :N].float(), st["V"][:, :, :N].float()
    O = torch.empty((b, hkv, G, q, d), dtype=dt, device="cuda")
    lse = torch.empty((b, hkv, G, q), dtype=torch.float32, device="cuda")
    if train:
        dO = st["dO"].view(b, hkv, G, q, d)
        dQ, dK, dV = torch.empty_like(O), torch.zeros_like(K), torch.zeros_like(V)
    step = max(1, min(max(256, min(W, 2048)), (1 << 28) // (b * h * min(N, W + 2048))))
    for r0 in range(0, q, step):                           # a slice of the queries and the keys that it can see
        r1 = min(q, r0 + step)
        lo, hi = max(0, N - q + r0 - W + 1), N - q + r1
        t = torch.arange(N - q + r0, hi, device="cuda")[:, None]
        u = torch.arange(lo, hi, device="cuda")[None, :]
        seen = (u <= t) & (u > t - W)
        if st["first"] is not None:
            seen = (seen & (u >= st["first"][:, r0:r1, None]))[:, None, None]
        Qc = Q[:, :, :, r0:r1].reshape(b, hkv, -1, d).float()
        Kc, Vc = K[:, :, lo:hi], V[:, :, lo:hi]
        S = torch.matmul(Qc, Kc.transpose(-1, -2)).view(b, hkv, G, r1 - r0, hi - lo) * scale
        S = torch.where(seen, S, -math.inf)
        m = S.amax(-1, keepdim=True)
        P = torch.exp(S - m)
        l = P.sum(-1, keepdim=True)
        P /= l
        lse[:, :, :, r0:r1] = (m + torch.log(l))[..., 0]
        P = P.view(b, hkv, -1, hi - lo)
        O[:, :, :, r0:r1] = torch.matmul(P, Vc).view(b, hkv, G, r1 - r0, d).to(dt)
        if train:
            g = dO[:, :, :, r0:r1].reshape(b, hkv, -1, d).float()
            dP = torch.matmul(g, Vc.transpose(-1, -2))
            dS = P * (dP - (P * dP).sum(-1, keepdim=True)) * scale
            dQ[:, :, :, r0:r1] = torch.matmul(dS, Kc).view(b, hkv, G, r1 - r0, d).to(dt)
            dK[:, :, lo:hi] += torch.matmul(dS.transpose(-1, -2), Qc)
            dV[:, :, lo:hi] += torch.matmul(P.transpose(-1, -2), g)
    out = {"O": O.view(b, h, q, d), "lse": lse.view(b, h, q)}
    if train:
        out.update(dQ=dQ.view(b, h, q, d), dK=dK.to(dt), dV=dV.to(dt))
    return out


def run(state):
    st = state
    if not own:
        return _plain_rope(st) if st["case"]["kind"] == "rope" else _plain_window(st)
    moba, sh = st["moba"], st["shape"]
    if st["case"]["kind"] == "rope":
        turn = moba.rope_backward if st["case"]["back"] else moba.rope
        Q, K = turn(sh, st["Q"], st["K"], st["positions"])
        return {"Q": Q, "K": K}
    O, lse = moba.window_forward(sh, st["Q"], st["K"], st["V"], first_key=st["first"], ws=st["ws"])
    out = {"O": O, "lse": lse}
    if st["case"]["kind"] == "train":
        out["dQ"], out["dK"], out["dV"] = moba.window_backward(sh, st["Q"], st["K"], st["V"], O, lse, st["dO"],
                                                               first_key=st["first"], ws=st["ws"])
    return out


def work(case):
    c = case
    es = 2 if c["dtype"] == "bf16" else 4
    b, h, hkv, N, d = c["batch"], c["heads"], c["kv_heads"], c["N"], c["d"]
    if c["kind"] == "rope":
        rows = b * (h + hkv) * N
        return {"bytes": 2 * rows * d * es + (4 * b * N if c["given"] else 0), "flops": 3 * rows * c["rot_dim"]}
    pairs = b * h * _pairs(c)
    keys = min(N, c["q_len"] + (c["window"] or N) - 1)     # that some query sees
    q_rows, kv_rows = b * h * c["q_len"], b * hkv * keys
    bytes_ = (2 * q_rows + 2 * kv_rows) * d * es + 4 * q_rows + (4 * b * c["q_len"] if c["lens"] else 0)
    flops = 4 * d * pairs
    if c["kind"] == "train":
        bytes_ += 2 * (q_rows * d * es) + 2 * b * hkv * N * d * es           # dO read; dQ, dK, dV written
        flops += 10 * d * pairs
    return {"bytes": bytes_, "flops": flops}


# ---- the definitions in 64 bits -------------------------------------------------------------------------
def _exact_rope(c, x):
    # a pair of channels is a complex number, which the position turns
    N, r = c["N"], c["rot_dim"]
    pos = x["positions"].double() if x["positions"] is not None else \
        torch.arange(c["position0"], c["position0"] + N, dtype=torch.float64, device="cuda").expand(c["batch"], N)
    i = torch.arange(r // 2, dtype=torch.float64, device="cuda")
    speed = torch.exp(i * (-2.0 / r * math.log(c["theta"])))
    if c["orig_len"] > 0:
        keep = ((speed * c["orig_len"] / (2 * math.pi) - c["band_low"]) / (c["band_high"] - c["band_low"])).clamp(0, 1)
    else:
        keep = torch.zeros_like(speed)
    if c["scale_factor"] != 1.0:
        speed = speed * keep + speed / c["scale_factor"] * (1 - keep)
    turn = torch.polar(torch.full((c["batch"], N, r // 2), c["amplitude"], dtype=torch.float64, device="cuda"),
                       pos[..., None] * speed)
    if c["back"]:
        turn = turn.conj()
    out = {}
    for name in ("Q", "K"):
        y = x[name].double()
        for head in range(y.shape[1]):                     # one head at a time: 64 bits of the longest are large
            z = y[:, head, :, :r]
            z = z.reshape(z.shape[:-1] + (r // 2, 2)) if c["interleaved"] else \
                torch.stack((z[..., :r // 2], z[..., r // 2:]), -1)
            z = torch.view_as_real(torch.view_as_complex(z.contiguous()) * turn)
            y[:, head, :, :r] = z.flatten(-2) if c["interleaved"] else torch.cat((z[..., 0], z[..., 1]), -1)
        out[name] = y
    return out


def exact(case, seed):
    c = case
    x = _inputs(c, seed)
    if c["kind"] == "rope":
        return _exact_rope(c, x)
    b, h, N, d, q = c["batch"], c["heads"], c["N"], c["d"], c["q_len"]
    G, W, s0 = h // c["kv_heads"], c["window"] or N, N - q
    train = c["kind"] == "train"
    f64 = {"dtype": torch.float64, "device": "cuda"}
    out = {"O": torch.zeros((b, h, q, d), **f64), "lse": torch.zeros((b, h, q), **f64)}
    if train:
        out.update(dQ=torch.zeros((b, h, q, d), **f64), dK=torch.zeros((b, h // G, c["rows"], d), **f64),
                   dV=torch.zeros((b, h // G, c["rows"], d), **f64))
    rows = 1024
    for i in range(b):
        for j in range(h):
            Kj, Vj = x["K"][i, j // G].double(), x["V"][i, j // G].double()
            Qj = x["Q"][i, j].double() / math.sqrt(d)
            for a in range(0, q, rows):
                e = min(q, a + rows)
                first = max(0, s0 + a + 1 - W)
                keys = slice(first, s0 + e)
                logits = Qj[a:e] @ Kj[keys].T
                back = torch.arange(s0 + a, s0 + e, device="cuda")[:, None] - torch.arange(first, s0 + e, device="cuda")
                out_of = (back < 0) | (back >= W)
                if x["first"] is not None:
                    out_of |= torch.arange(first, s0 + e, device="cuda") < x["first"][i, a:e, None]
                logits.masked_fill_(out_of, -math.inf)
                z = torch.logsumexp(logits, -1)
                p = torch.exp(logits - z[:, None])
                o = p @ Vj[keys]
                out["O"][i, j, a:e], out["lse"][i, j, a:e] = o, z
                if train:
                    do = x["dO"][i, j, a:e].double()
                    ds = p * (do @ Vj[keys].T - (do * o).sum(-1, keepdim=True))
                    out["dQ"][i, j, a:e] = ds @ Kj[keys] / math.sqrt(d)
                    out["dK"][i, j // G, keys] += ds.T @ Qj[a:e]
                    out["dV"][i, j // G, keys] += p.T @ do
    return out
