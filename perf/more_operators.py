"""Cases of three more operators of a policy learner: sizes, inputs, one pass, what the pass cannot do without, and its
value in 64 bits.

Kinds of case
  delta_step     the gated delta rule for single tokens, on a table of matrix states (marl_delta_step)
  delta_scan     the delta rule over whole sequences, forward (marl_delta_scan)
  delta_train    forward and backward (marl_delta_scan, marl_delta_scan_grad)
  distill        divergence of a student's logits from a teacher's kept alternatives (marl_distill)
  distill_train  the same with the gradient of the logits (marl_distill, marl_distill_grad)
  penalize       penalties for repeated tokens, biases and a grammar's mask on logits (marl_penalize)

`own` chooses between elementary torch operations (False) and the framework's entry points (True); both start from
what prepare() gives.
"""
import math

import torch

own = False

DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
CHUNK = 64                                    # steps that the plain form of the delta rule takes at once


def listed():
    return [
        # The smallest call: a worker's eight environments of three agents, two heads of 32; latency alone counts.
        dict(name="step_worker", kind="delta_step", slots=24, n=24, Hk=2, Hv=2, Dk=32, Dv=32, dtype="fp32", reset=True),
        # Serving: the listed 201 of 512 running sequences get one token; two value heads share a key.
        dict(name="step_serve", kind="delta_step", slots=512, n=201, Hk=8, Hv=16, Dk=128, Dv=128, dtype="bf16", reset=False),
        # A few short sequences with head sizes that fit no tile.
        dict(name="scan_odd_heads", kind="delta_scan", B=7, T=333, Hk=3, Hv=3, Dk=40, Dv=72, dtype="fp16", filled=False, reset=True, fused=False),
        # One long sequence read before an answer: sixteen heads are all that runs side by side. Odd length.
        dict(name="scan_prefill", kind="delta_scan", B=1, T=20011, Hk=8, Hv=16, Dk=128, Dv=128, dtype="bf16", filled=False, reset=False, fused=True),
        # A learner batch of the 2s3z scenario (64 episodes of five agents, 120 slots, 64 units as four heads): episodes end early, some are empty.
        dict(name="train_2s3z", kind="delta_train", B=320, T=120, Hk=4, Hv=4, Dk=16, Dv=16, dtype="fp32", filled=True, reset=False, fused=False),
        # The largest recurrence: four long rows of packed documents, q, k and v as column blocks of one projection's result.
        dict(name="train_long", kind="delta_train", B=4, T=8192, Hk=8, Hv=16, Dk=128, Dv=128, dtype="bf16", filled=False, reset=True, fused=True),
        # How far a small server's answers are from the teacher's fifty alternatives: few rows, a large vocabulary.
        dict(name="distill_eval", kind="distill", R=16, V=131072, K=50, dtype="bf16", avail="none", tail=True),
        # The scale-up learner batch (64 episodes, 200 slots, 32 agents, 40 actions) with its availability mask, five kept actions.
        dict(name="distill_actions", kind="distill_train", R=409600, V=40, K=5, dtype="fp32", avail="rows", tail=True),
        # Answers of a teacher over an odd vocabulary whose rows start at any alignment.
        dict(name="distill_tokens", kind="distill_train", R=8191, V=50021, K=20, dtype="fp16", avail="none", tail=False),
        # A worker's agents that have an action each: the smallest edit.
        dict(name="penalize_actions", kind="penalize", R=24, V=40, L=120, M=4, dtype="fp32", allowed="rows"),
        # Sampling step of a small server: few rows, a large vocabulary, a grammar.
        dict(name="penalize_decode", kind="penalize", R=16, V=131072, L=4096, M=16, dtype="bf16", allowed="rows"),
        # Sampling step of a full server: many rows of an odd vocabulary, long histories, biases.
        dict(name="penalize_serve", kind="penalize", R=777, V=50021, L=8192, M=64, dtype="fp16", allowed="shared"),
    ]


def _log_int(rng, low, high):
    return max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))


def draw(rng):
    kind = rng.choice(["delta_step", "delta_scan", "delta_train", "distill", "distill_train", "penalize"])
    dtype = rng.choice(["fp32", "bf16", "fp16"])
    if kind.startswith("delta"):
        Hk = _log_int(rng, 1, 8)
        Hv = Hk * rng.choice([1, 1, 2, 4])
        Dk, Dv = _log_int(rng, 8, 128), _log_int(rng, 8, 256)
        heads = dict(Hk=Hk, Hv=Hv, Dk=Dk, Dv=Dv, dtype=dtype)
        state = Hv * Dk * Dv
        if kind == "delta_step":
            slots = _log_int(rng, 1, max(1, min(1024, 130_000_000 // state)))
            return dict(kind=kind, slots=slots, n=rng.randint(1, min(slots, max(1, 52_000_000 // state))), **heads, reset=rng.random() < 0.5)
        most = 8_000_000_000 if kind == "delta_train" else 5_000_000_000          # entries of states, over all steps
        T = _log_int(rng, 1, max(1, min(20011 if kind == "delta_scan" else 8192, most // state)))
        B = _log_int(rng, 1, max(1, min(320, most // (T * state), 40_000_000 // (T * Hv * max(Dk, Dv)))))
        return dict(kind=kind, B=B, T=T, **heads, filled=rng.random() < 0.5, reset=rng.random() < 0.5, fused=rng.random() < 0.5)
    V = _log_int(rng, 2, 150000)
    if kind == "penalize":
        R = _log_int(rng, 1, max(1, min(4096, 38_000_000 // V)))
        return dict(kind=kind, R=R, V=V, L=_log_int(rng, 1, max(1, min(8192, 6_000_000 // R))), M=rng.choice([0, 1, 4, 16, 64]), dtype=dtype,
                    allowed=rng.choice(["none", "rows", "shared"]))
    R = _log_int(rng, 1, max(1, min(409600, (400_000_000 if dtype != "fp32" else 200_000_000) // V)))
    return dict(kind=kind, R=R, V=V, K=rng.choice([k for k in (1, 5, 20, 50) if k <= V]), dtype=dtype, avail=rng.choice(["none", "rows", "shared"]),
                tail=rng.random() < 0.5)


# ------------------------------------------------------------------------------------------------ inputs
def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _inputs(case, seed):
    """The tensors of a case; the same for both forms and for exact()."""
    g = _generator(seed)
    dt = DTYPES[case["dtype"]]
    randn = lambda *s: torch.randn(*s, generator=g, device="cuda")
    rand = lambda *s: torch.rand(*s, generator=g, device="cuda")
    unit = lambda t: t / torch.sqrt((t * t).sum(-1, keepdim=True) + 1e-6)
    kind, s = case["kind"], {}
    if kind.startswith("delta"):
        Hk, Hv, Dk, Dv = (case[k] for k in ("Hk", "Hv", "Dk", "Dv"))
        lead = (case["n"],) if kind == "delta_step" else (case["B"], case["T"])
        q, k, v = unit(randn(*lead, Hk, Dk)), unit(randn(*lead, Hk, Dk)), randn(*lead, Hv, Dv)
        if case.get("fused"):
            proj = torch.cat([q.flatten(-2), k.flatten(-2), v.flatten(-2)], -1).to(dt)
            q, k, v = (p.unflatten(-1, d) for p, d in zip(proj.split([Hk * Dk, Hk * Dk, Hv * Dv], -1), ((Hk, Dk), (Hk, Dk), (Hv, Dv))))
        s.update(q=q.to(dt), k=k.to(dt), v=v.to(dt), scale=Dk ** -0.5)
        # heads that keep between 0.8 and 0.999 of their state a step, half to twice that rate by the token
        rate = -torch.log(0.8 + 0.199 * rand(Hv))
        s["log_decay"] = -rate * (0.5 + 1.5 * rand(*lead, Hv))
        s["beta"] = torch.sigmoid(randn(*lead, Hv))
        if kind == "delta_step":
            s["s_in"] = randn(case["slots"], Hv, Dk, Dv) * 0.3
            s["slot"] = torch.randperm(case["slots"], generator=g, device="cuda")[:case["n"]].to(torch.int32)
            s["reset"] = (rand(case["n"]) < 0.1).to(torch.uint8) if case["reset"] else None
            return s
        B, T = lead
        s.update(s_first=randn(B, Hv, Dk, Dv) * 0.3, reset=None, filled=None)
        if case["reset"]:                       # documents of about 500 steps
            s["reset"] = (rand(B, T) < 1.0 / 500).to(torch.uint8)
        if case["filled"]:                      # episodes that end early, one in sixteen without a step
            length = (rand(B) * 1.2 * T).clamp(max=T) * (rand(B) > 1.0 / 16)
            s["filled"] = (torch.arange(T, device="cuda")[None] < length[:, None]).to(torch.uint8)
        if kind == "delta_train":
            s["grad_o"] = randn(B, T, Hv, Dv).to(dt)
            s["grad_s_last"] = randn(B, Hv, Dk, Dv) * 0.3
        return s
    R, V = case["R"], case["V"]
    s["logits"] = torch.randn(R, V, generator=g, device="cuda", dtype=dt).mul_(2.5)
    if kind.startswith("distill"):
        K = case["K"]
        s["avail"] = None
        if case["avail"] == "rows":             # agents that are out have no action
            s["avail"] = (rand(R, V) < 0.7).to(torch.uint8)
            s["avail"][rand(R) < 0.05] = 0
        elif case["avail"] == "shared":
            s["avail"] = (rand(V) < 0.9).to(torch.uint8)
            s["avail"][0] = 1
        s["scale"], s["tail"] = (1.0 if kind == "distill_train" else 0.8), case["tail"]
        # the teacher's alternatives: distinct places of the row, 0.97 of its probability in descending order, the last ones missing now and then
        start, stride = torch.randint(0, V, (R, 1), generator=g, device="cuda"), _coprime(V)
        s["top_id"] = ((start + stride * torch.arange(K, device="cuda")) % V).to(torch.int32)
        p = torch.sort(torch.softmax(2.0 * randn(R, K), 1), 1, descending=True).values
        s["top_value"] = torch.log(0.97 * p)
        if K > 1:
            s["top_id"][rand(R) < 0.1, K - 1] = -1
        s["top_value"][s["top_id"] < 0] = -math.inf
        if kind == "distill_train":
            # a mean over the rows; in fp16 under a loss scale, without which the small ones would be lost
            s["grad_loss"] = torch.full((R,), 4096.0 if case["dtype"] == "fp16" else 1.0 / R, device="cuda") * (0.5 + rand(R))
        return s
    L, M = case["L"], case["M"]
    # tokens come back: most are of the few that the row favours
    own_few = torch.randint(0, V, (R, max(1, L // 8)), generator=g, device="cuda")
    again = own_few.gather(1, torch.randint(0, own_few.shape[1], (R, L), generator=g, device="cuda"))
    s["history"] = torch.where(rand(R, L) < 0.7, again, torch.randint(0, V, (R, L), generator=g, device="cuda")).to(torch.int32)
    s["length"] = (rand(R) * (L + 1)).to(torch.int32).clamp(max=L)
    s["prompt"] = (rand(R) * s["length"]).to(torch.int32)
    s["repetition"], s["presence"], s["frequency"] = 1.0 + 0.3 * rand(R), 0.5 * rand(R), 0.2 * rand(R)
    s["bias_id"] = s["bias_value"] = s["allowed"] = None
    if M:
        s["bias_id"] = torch.randint(-1, V, (R, M), generator=g, device="cuda").to(torch.int32)
        s["bias_value"] = 3.0 * randn(R, M)
    words = (V + 31) // 32
    if case["allowed"] != "none":
        shape = (R, words) if case["allowed"] == "rows" else (words,)
        s["allowed"] = torch.randint(-2 ** 31, 2 ** 31, shape, generator=g, device="cuda").to(torch.int32)
    return s


def _coprime(V):
    """A stride that visits V places before it comes back."""
    stride = max(1, int(V * 0.381966))
    while math.gcd(stride, V) != 1:
        stride += 1
    return stride


def prepare(case, seed):
    s = dict(case=case, **_inputs(case, seed))
    dt = DTYPES[case["dtype"]]
    kind = case["kind"]
    new = lambda *shape, dtype=torch.float32: torch.zeros(*shape, dtype=dtype, device="cuda")
    size = lambda entry, *args: 0
    if own:
        from paper_2205_05248_amd import binding
        size = lambda entry, *args: getattr(binding, entry)(*args)
    bytes_ = 0
    if kind.startswith("delta"):
        s["o"] = new(*s["v"].shape, dtype=dt)
        if kind == "delta_step":
            s["s_out"] = torch.zeros_like(s["s_in"])
            return s
        B, T, Hk, Hv, Dk, Dv = (case[k] for k in ("B", "T", "Hk", "Hv", "Dk", "Dv"))
        s["s_last"] = new(B, Hv, Dk, Dv)
        if kind == "delta_train":
            s.update(grad_q=new(B, T, Hk, Dk, dtype=dt), grad_k=new(B, T, Hk, Dk, dtype=dt), grad_v=new(B, T, Hv, Dv, dtype=dt),
                     grad_log_decay=new(B, T, Hv), grad_beta=new(B, T, Hv), grad_s_first=new(B, Hv, Dk, Dv))
        bytes_ = size("marl_delta_scan_workspace_bytes", case["dtype"], B, T, Hk, Hv, Dk, Dv, kind == "delta_train")
    elif kind.startswith("distill"):
        R = case["R"]
        s.update(loss=new(R), log_sum=new(R), log_rest=new(R) if case["tail"] else None)
        if kind == "distill_train":
            s["grad_logits"] = new(R, case["V"], dtype=dt)
        bytes_ = size("marl_distill_workspace_bytes", R, case["V"], case["K"])
    else:
        s["out"] = new(case["R"], case["V"], dtype=dt)
    s["workspace"] = torch.empty(bytes_, dtype=torch.uint8, device="cuda")
    return s


# ------------------------------------------------------------------------------------------------ one pass
def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_own(s):
    from paper_2205_05248_amd import binding
    kind = s["case"]["kind"]
    if kind == "delta_step":
        binding.marl_delta_step(s["q"], s["k"], s["v"], s["log_decay"], s["beta"], s["scale"], s["slot"], s["reset"], s["s_in"], s["s_out"], s["o"])
        return s["o"], s["s_out"]
    if kind.startswith("delta"):
        train = kind == "delta_train"
        binding.marl_delta_scan(s["q"], s["k"], s["v"], s["log_decay"], s["beta"], s["scale"], s["reset"], s["filled"], s["s_first"], s["o"],
                                s["s_last"], s["workspace"], keep=train)
        if not train:
            return s["o"], s["s_last"]
        binding.marl_delta_scan_grad(s["q"], s["k"], s["v"], s["log_decay"], s["beta"], s["scale"], s["reset"], s["filled"], s["grad_o"],
                                     s["grad_s_last"], s["workspace"], s["grad_q"], s["grad_k"], s["grad_v"], s["grad_log_decay"], s["grad_beta"],
                                     s["grad_s_first"])
        return [s[k] for k in ("o", "s_last", "grad_q", "grad_k", "grad_v", "grad_log_decay", "grad_beta", "grad_s_first")]
    if kind.startswith("distill"):
        binding.marl_distill(s["logits"], s["top_id"], s["top_value"], s["avail"], s["scale"], s["tail"], s["loss"], s["log_sum"], s["log_rest"],
                             s["workspace"])
        out = [s["loss"], s["log_sum"]] + ([s["log_rest"]] if s["tail"] else [])
        if kind == "distill_train":
            binding.marl_distill_grad(s["logits"], s["top_id"], s["top_value"], s["avail"], s["scale"], s["tail"], s["log_sum"], s["log_rest"],
                                      s["grad_loss"], s["grad_logits"])
            out.append(s["grad_logits"])
        return out
    binding.marl_penalize(s["logits"], s["history"], s["length"], s["prompt"], s["repetition"], s["presence"], s["frequency"], s["bias_id"],
                          s["bias_value"], s["allowed"], s["out"])
    return s["out"]


def _run_plain(s):
    kind, dt = s["case"]["kind"], DTYPES[s["case"]["dtype"]]
    if kind == "delta_step":
        return _plain_step(s, dt)
    if kind.startswith("delta"):
        return _plain_scan(s, kind == "delta_train", dt)
    if kind.startswith("distill"):
        return _plain_distill(s, kind == "distill_train", dt)
    return _plain_penalize(s, dt)


def _plain_step(s, dt):
    group = s["v"].shape[1] // s["q"].shape[1]
    q, k = (s[n].float().repeat_interleave(group, 1) for n in "qk")
    slot = s["slot"].long()
    a = torch.exp(s["log_decay"])
    if s["reset"] is not None:
        a = a.masked_fill((s["reset"] != 0)[:, None], 0.0)
    S = a[..., None, None] * s["s_in"][slot]
    u = s["beta"][..., None] * (s["v"].float() - (S * k[..., None]).sum(2))
    S = S + k[..., None] * u[..., None, :]
    s_out = torch.zeros_like(s["s_in"])
    s_out[slot] = S
    return (s["scale"] * (S * q[..., None]).sum(2)).to(dt), s_out


def _chunks(t, n):
    """[B,T,H,...] to [B H, n, CHUNK, ...], the end filled up with zeros."""
    B, T, H = t.shape[:3]
    t = torch.cat([t, t.new_zeros(B, n * CHUNK - T, *t.shape[2:])], 1) if n * CHUNK > T else t
    return t.unflatten(1, (n, CHUNK)).movedim(3, 1).flatten(0, 1).contiguous()


def _steps(t, B, T):
    """The other way: [B H, n, CHUNK, ...] to [B,T,H,...]."""
    return t.unflatten(0, (B, -1)).movedim(1, 3).flatten(1, 2)[:, :T]


def _unit_lower_inverse(A):
    """(I + A)^-1 of strictly lower [..., CHUNK, CHUNK]: blocks of 16 by substitution, all at once, then two rounds of joins."""
    size, N = 16, A.shape[:-2]
    blocks = torch.stack([A[..., i:i + size, i:i + size] for i in range(0, CHUNK, size)], -3)
    X = torch.eye(size, device=A.device).expand(blocks.shape).contiguous()
    for i in range(1, size):
        X[..., i, :] -= (blocks[..., i, :i, None] * X[..., :i, :]).sum(-2)
    while size < CHUNK:
        first, second = X[..., 0::2, :, :], X[..., 1::2, :, :]
        low = torch.stack([A[..., i + size:i + 2 * size, i:i + size] for i in range(0, CHUNK, 2 * size)], -3)
        low = -torch.matmul(torch.matmul(second, low), first)
        X = torch.cat([torch.cat([first, torch.zeros_like(first)], -1), torch.cat([low, second], -1)], -2)
        size *= 2
    return X.reshape(*N, CHUNK, CHUNK)


def _plain_scan(s, train, dt):
    B, T, Hv, Dv = s["v"].shape
    Hk, Dk = s["q"].shape[2:]
    n, group, scale = -(-T // CHUNK), Hv // Hk, s["scale"]
    live = torch.ones(B, T, dtype=torch.bool, device="cuda") if s["filled"] is None else s["filled"] != 0
    new = torch.zeros_like(live) if s["reset"] is None else (s["reset"] != 0) & live
    wide = lambda t: _chunks(t.float().repeat_interleave(Hv // t.shape[2], 2) * live[..., None, None], n)
    q, k, v = wide(s["q"]), wide(s["k"]), wide(s["v"])
    beta = _chunks(s["beta"] * live[..., None], n)[..., None]
    g = _chunks(s["log_decay"] * (live & ~new)[..., None], n)
    part = torch.cumsum(_chunks(new[..., None].expand(B, T, Hv).to(torch.int32), n), -1)          # which sequence of its chunk a step belongs to
    G = torch.cumsum(g.double(), -1)
    end = G[..., -1:]
    causal = torch.ones(CHUNK, CHUNK, dtype=torch.bool, device="cuda").tril()
    same = (part[..., :, None] == part[..., None, :]) & causal
    E = torch.exp((G[..., :, None] - G[..., None, :]).masked_fill(~same, -math.inf)).float()
    from_start = (torch.exp(G) * (part == 0)).float()[..., None]
    to_end = (torch.exp(end - G) * (part == part[..., -1:])).float()[..., None]
    whole = from_start[..., -1:, :]
    Ah = (E * torch.matmul(k, k.transpose(-1, -2))).tril(-1)
    inv = _unit_lower_inverse(beta * Ah)
    P = E * torch.matmul(q, k.transpose(-1, -2))
    W = torch.matmul(inv, beta * from_start * k)
    U0 = torch.matmul(inv, beta * v)
    k_end = (to_end * k).transpose(-1, -2).contiguous()
    S = torch.empty(B * Hv, n + 1, Dk, Dv, device="cuda")
    S[:, 0] = s["s_first"].flatten(0, 1)
    for c in range(n):                          # each chunk's state from the one before
        U0[:, c] -= torch.matmul(W[:, c], S[:, c])
        S[:, c + 1] = torch.baddbmm(whole[:, c] * S[:, c], k_end[:, c], U0[:, c])
    U, last, S = U0, S[:, n].unflatten(0, (B, Hv)).clone(), S[:, :n]
    o = scale * (from_start * torch.matmul(q, S) + torch.matmul(P, U))
    o = _steps(o, B, T).to(dt)
    if not train:
        return o, last
    do = scale * wide(s["grad_o"])
    dU = torch.matmul(P.transpose(-1, -2).contiguous(), do)
    k_end = k_end.transpose(-1, -2).contiguous()
    dS = torch.empty(B * Hv, n + 1, Dk, Dv, device="cuda")
    dS[:, :n] = torch.matmul((from_start * q).transpose(-1, -2).contiguous(), do)
    dS[:, n] = s["grad_s_last"].flatten(0, 1)
    W = W.transpose(-1, -2).contiguous()
    for c in range(n - 1, -1, -1):
        dU[:, c] += torch.matmul(k_end[:, c], dS[:, c + 1])
        dS[:, c] += whole[:, c] * dS[:, c + 1] - torch.matmul(W[:, c], dU[:, c])
    grad_s_first, dS = dS[:, 0].unflatten(0, (B, Hv)).clone(), dS[:, 1:]
    dR = torch.matmul(inv.transpose(-1, -2).contiguous(), dU)
    turned = S.transpose(-1, -2).contiguous()
    dA = -torch.matmul(dR, U.transpose(-1, -2).contiguous()).tril(-1)
    R = v - from_start * torch.matmul(k, S)
    dbeta = (dR * R).sum(-1) + (dA * Ah).sum(-1)
    dR = beta * dR
    dA = beta * dA
    dP = torch.matmul(do, U.transpose(-1, -2).contiguous())
    dq_far = from_start * torch.matmul(do, turned)
    dk_far = -from_start * torch.matmul(dR, turned)
    dk_end = to_end * torch.matmul(U, dS.transpose(-1, -2).contiguous())
    flow = (dA * Ah + dP * P).double()
    to_later = (k * dk_end).double().sum(-1)
    dG = flow.sum(-1) - flow.sum(-2) + (q * dq_far + k * dk_far).double().sum(-1) - to_later
    dG[..., -1] += to_later.sum(-1) + (whole[..., 0, 0] * (dS * S).sum((-1, -2))).double()
    dg = dG.flip(-1).cumsum(-1).flip(-1).float()
    dN, dM = dP * E, dA * E
    dq = dq_far + torch.matmul(dN, k)
    dk = dk_far + dk_end + torch.matmul(dN.transpose(-1, -2).contiguous(), q) + torch.matmul(dM + dM.transpose(-1, -2), k)
    shared = lambda t: (_steps(t, B, T) * live[..., None, None]).unflatten(2, (Hk, group)).sum(3).to(dt)
    dv = _steps(dR, B, T) * live[..., None, None]
    return (o, last, shared(dq), shared(dk), dv.to(dt), _steps(dg[..., None], B, T)[..., 0] * (live & ~new)[..., None],
            _steps(dbeta[..., None], B, T)[..., 0] * live[..., None], grad_s_first)


def _plain_distill(s, train, dt):
    z = s["scale"] * s["logits"].float()
    if s["avail"] is not None:
        z = z.masked_fill(s["avail"] == 0, -math.inf)
    top = z.max(1, keepdim=True).values
    some = top > -math.inf
    z = z - torch.where(some, top, torch.zeros_like(top))
    e = torch.exp(z)
    total = e.sum(1, keepdim=True)
    place = s["top_id"].long().clamp(min=0)
    kept = (s["top_id"] >= 0) & (z.gather(1, place) > -math.inf)
    value = s["top_value"].masked_fill(~kept, -math.inf)
    if not s["tail"]:
        best = value.max(1, keepdim=True).values
        best = torch.where(best > -math.inf, best, torch.zeros_like(best))
        value = value - best
        value = value - torch.log(torch.exp(value).sum(1, keepdim=True).clamp(min=1e-30))
    p = torch.exp(value)
    log_q = z.gather(1, place) - torch.log(total)
    loss = torch.where(p > 0, p * (value - log_q), torch.zeros_like(p)).sum(1)
    log_sum = torch.where(some, top + torch.log(total), torch.full_like(top, -math.inf))[:, 0]
    out = [loss, log_sum]
    weight = p.sum(1, keepdim=True)
    if s["tail"]:
        # one minus a sum next to one, and the sum of the places that are left: zeros at the kept ones
        p_rest = (1 - torch.exp(value.double()).sum(1, keepdim=True)).clamp(min=0).float()
        listed_ = torch.zeros_like(e).scatter_reduce_(1, place, kept.float(), "amax")
        taken, rest = (e * listed_).sum(1, keepdim=True), (e * (1 - listed_)).sum(1, keepdim=True)
        p_rest = torch.where(rest > 0, p_rest, torch.zeros_like(p_rest))
        log_rest = torch.where(taken < rest, torch.log1p(-taken / total), torch.log(rest / total))
        log_rest = torch.where(rest > 0, log_rest, torch.full_like(rest, -math.inf))
        out[0] = loss + torch.where(p_rest > 0, p_rest * (torch.log(p_rest) - log_rest), torch.zeros_like(p_rest))[:, 0]
        out.append(log_rest[:, 0])
        weight = weight + p_rest
    if train:
        q = e / total
        g = q * weight
        if s["tail"]:
            ratio = torch.where(p_rest > 0, p_rest * torch.exp(-log_rest), torch.zeros_like(p_rest))
            g = g - q * (1 - listed_) * ratio
        g.scatter_add_(1, place, -p * kept)
        g = g * (s["scale"] * s["grad_loss"])[:, None]
        out.append(torch.where(some & (e > 0), g, torch.zeros_like(g)).to(dt))
    return out


def _plain_penalize(s, dt):
    z = s["logits"].float()
    R, V = z.shape
    L = s["history"].shape[1]
    at = torch.arange(L, device="cuda")[None]
    token = s["history"].long()
    seen = torch.zeros(R, V, device="cuda").scatter_add_(1, token, (at < s["length"][:, None]).float())
    count = torch.zeros(R, V, device="cuda").scatter_add_(1, token, ((at >= s["prompt"][:, None]) & (at < s["length"][:, None])).float())
    rho = s["repetition"][:, None]
    z = torch.where(seen > 0, torch.where(z > 0, z / rho, z * rho), z)
    z = z - s["presence"][:, None] * (count > 0) - s["frequency"][:, None] * count
    if s["bias_id"] is not None:
        z = z.scatter_add(1, s["bias_id"].long().clamp(min=0), s["bias_value"].masked_fill(s["bias_id"] < 0, 0.0))
    if s["allowed"] is not None:
        bits = (s["allowed"][..., None] >> torch.arange(32, device="cuda", dtype=torch.int32)) & 1
        z = z.masked_fill(bits.flatten(-2)[..., :V] == 0, -math.inf)
    return z.to(dt)


# ------------------------------------------------------------------------------------------------ accounting
def work(case):
    size = 4 if case["dtype"] == "fp32" else 2
    kind = case["kind"]
    if kind.startswith("delta"):
        Hk, Hv, Dk, Dv = (case[k] for k in ("Hk", "Hv", "Dk", "Dv"))
        token = (2 * Hk * Dk + 2 * Hv * Dv) * size + 8 * Hv
        if kind == "delta_step":
            return {"bytes": case["n"] * (token + 8 * Hv * Dk * Dv + 5), "flops": 7 * case["n"] * Hv * Dk * Dv}
        B, T = case["B"], case["T"]
        masks = B * T * (int(case["reset"]) + int(case["filled"]))
        out = {"bytes": B * T * token + masks + 8 * B * Hv * Dk * Dv, "flops": 7 * B * T * Hv * Dk * Dv}
        if kind == "delta_train":
            out["bytes"] += B * T * ((4 * Hk * Dk + 3 * Hv * Dv) * size + 16 * Hv) + masks + 8 * B * Hv * Dk * Dv
            out["flops"] += 16 * B * T * Hv * Dk * Dv
        return out
    R, V = case["R"], case["V"]
    if kind.startswith("distill"):
        mask = {"none": 0, "rows": R * V, "shared": V}[case["avail"]]
        out = {"bytes": R * V * size + mask + R * (8 * case["K"] + 12), "flops": 4 * R * V}
        if kind == "distill_train":
            out["bytes"] += 2 * R * V * size + mask + R * (8 * case["K"] + 12)
            out["flops"] += 4 * R * V
        return out
    words = (V + 31) // 32
    bits = {"none": 0, "rows": R * words, "shared": words}[case["allowed"]] * 4
    return {"bytes": 2 * R * V * size + bits + R * (2 * case["L"] + 8 * case["M"] + 20), "flops": 6 * R * V}


# ------------------------------------------------------------------------------------------------ in 64 bits
def exact(case, seed):
    s = _inputs(case, seed)
    kind = case["kind"]
    if kind == "delta_step":
        return _exact_step(case, s)
    if kind.startswith("delta"):
        return _exact_scan(case, s)
    if kind.startswith("distill"):
        return _exact_distill(case, s)
    return _exact_penalize(case, s)


def _by_value_head(t, Hv):
    t = t.double()
    return t[..., torch.arange(Hv, device="cuda") // (Hv // t.shape[-2]), :]


def _exact_step(case, s):
    Hv = case["Hv"]
    q, k, v = (_by_value_head(s[n], Hv) for n in "qkv")
    keep = torch.exp(s["log_decay"].double())
    if s["reset"] is not None:
        keep = torch.where(s["reset"][:, None] != 0, torch.zeros_like(keep), keep)
    slot = s["slot"].long()
    old = keep[..., None, None] * s["s_in"][slot].double()
    delta = s["beta"].double()[..., None] * (v - torch.matmul(k[..., None, :], old)[..., 0, :])
    state = old + k[..., :, None] * delta[..., None, :]
    table = torch.zeros(s["s_in"].shape, dtype=torch.float64, device="cuda")
    table[slot] = state
    return s["scale"] * torch.matmul(q[..., None, :], state)[..., 0, :], table


def _exact_scan(case, s):
    """Step by step; the backward pass forms the states of a stretch again from the one kept at its start."""
    Hv, Hk, B, T = case["Hv"], case["Hk"], case["B"], case["T"]
    q, k, v = (_by_value_head(s[n], Hv) for n in "qkv")
    keep, beta = torch.exp(s["log_decay"].double()), s["beta"].double()
    own_decay = torch.ones(B, T, 1, dtype=torch.float64, device="cuda")
    if s["reset"] is not None:
        own_decay = own_decay * (s["reset"] == 0)[..., None]
    keep = keep * own_decay
    if s["filled"] is not None:
        pad = (s["filled"] == 0)[..., None]
        keep, beta = keep.masked_fill(pad, 1.0), beta.masked_fill(pad, 0.0)
        own_decay = own_decay.masked_fill(pad, 0.0)
        q, k, v = (t.masked_fill(pad[..., None], 0.0) for t in (q, k, v))
    stretch = 64

    def ahead(t, state):
        old = keep[:, t, :, None, None] * state
        miss = v[:, t] - torch.matmul(k[:, t, :, None], old)[..., 0, :]
        return old, miss, old + k[:, t, :, :, None] * (beta[:, t, :, None] * miss)[..., None, :]

    state, starts = s["s_first"].double(), []
    o = torch.empty(v.shape, dtype=torch.float64, device="cuda")
    for t in range(T):
        if t % stretch == 0:
            starts.append(state)
        _, _, state = ahead(t, state)
        o[:, t] = s["scale"] * torch.matmul(q[:, t, :, None], state)[..., 0, :]
    if case["kind"] == "delta_scan":
        return o, state
    do = s["grad_o"].double() * s["scale"]
    if s["filled"] is not None:
        do = do.masked_fill(pad[..., None], 0.0)
    dq, dk, dv = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    dg, db = torch.zeros_like(keep), torch.zeros_like(beta)
    adj = s["grad_s_last"].double()
    for c in range(len(starts) - 1, -1, -1):
        trail, at = [], starts[c]
        steps = range(c * stretch, min(T, (c + 1) * stretch))
        for t in steps:
            trail.append(at)
            at = ahead(t, at)[2]
        for t in reversed(steps):
            before = trail.pop()
            old, miss, after = ahead(t, before)
            dq[:, t] = torch.matmul(after, do[:, t, :, :, None])[..., 0]
            adj = adj + q[:, t, :, :, None] * do[:, t, :, None, :]
            d_delta = torch.matmul(k[:, t, :, None], adj)[..., 0, :]
            db[:, t] = (d_delta * miss).sum(-1)
            d_miss = beta[:, t, :, None] * d_delta
            dv[:, t] = d_miss
            dk[:, t] = torch.matmul(adj, (beta[:, t, :, None] * miss)[..., None])[..., 0] - torch.matmul(old, d_miss[..., None])[..., 0]
            d_old = adj - k[:, t, :, :, None] * d_miss[..., None, :]
            dg[:, t] = (d_old * old).sum((-1, -2)) * own_decay[:, t]
            adj = keep[:, t, :, None, None] * d_old
    together = lambda t: t.reshape(B, T, Hk, Hv // Hk, -1).sum(3)
    if s["filled"] is not None:
        dq, dk, dv = (t.masked_fill(pad[..., None], 0.0) for t in (dq, dk, dv))
        db = db.masked_fill(pad, 0.0)
    return o, state, together(dq), together(dk), dv, dg, db, adj


def _exact_distill(case, s):
    """Row blocks of at most 2^26 values at a time."""
    R, V = case["R"], case["V"]
    block = max(1, (1 << 26) // V)
    parts = []
    for lo in range(0, R, block):
        rows = slice(lo, min(R, lo + block))
        z = s["logits"][rows].double() * s["scale"]
        if s["avail"] is not None:
            ok = s["avail"] if s["avail"].dim() == 1 else s["avail"][rows]
            z = torch.where(ok != 0, z, torch.full_like(z, -math.inf))
        norm = torch.logsumexp(z, 1, keepdim=True)
        empty = torch.isinf(norm)
        log_q = torch.where(empty, z, z - norm)
        ids, value = s["top_id"][rows].long(), s["top_value"][rows].double()
        mine = torch.where(ids >= 0, log_q.gather(1, ids.clamp(min=0)), torch.full_like(value, -math.inf))
        use = mine > -math.inf
        value = torch.where(use, value, torch.full_like(value, -math.inf))
        if not case["tail"]:
            mass = torch.logsumexp(value, 1, keepdim=True)
            value = torch.where(use, value - mass, value)
        p = torch.exp(value)
        loss = torch.where(p > 0, p * (value - torch.where(use, mine, torch.zeros_like(mine))), torch.zeros_like(p)).sum(1)
        out, target = [loss, norm[:, 0]], torch.zeros_like(z)
        target.scatter_add_(1, ids.clamp(min=0), torch.where(use, p, torch.zeros_like(p)))
        if case["tail"]:
            beside = torch.cat([log_q, torch.full_like(log_q[:, :1], -math.inf)], 1)               # a place for what is not kept
            others = beside.scatter_(1, torch.where(use, ids, torch.full_like(ids, V)), -math.inf)[:, :V]
            rest = torch.logsumexp(others, 1, keepdim=True)
            left = torch.where(torch.isinf(rest), torch.zeros_like(rest), (1 - p.sum(1, keepdim=True)).clamp(min=0))
            out[0] = loss + torch.where(left > 0, left * (torch.log(left) - rest), torch.zeros_like(left))[:, 0]
            out.append(rest[:, 0])
            share = torch.exp(torch.where(torch.isinf(rest), others, others - rest))
            target = target + left * share
        if case["kind"] == "distill_train":
            grad = torch.exp(log_q) * target.sum(1, keepdim=True) - target
            out.append(torch.where(log_q > -math.inf, grad, torch.zeros_like(grad)) * (s["scale"] * s["grad_loss"][rows].double())[:, None])
        parts.append(out)
    return [torch.cat(p) for p in zip(*parts)]


def _exact_penalize(case, s):
    R, V, L = case["R"], case["V"], case["L"]
    block = max(1, (1 << 26) // V)
    parts = []
    for lo in range(0, R, block):
        rows = slice(lo, min(R, lo + block))
        z = s["logits"][rows].double()
        n = z.shape[0]
        where = torch.arange(L, device="cuda")[None]
        length, prompt = s["length"][rows, None], s["prompt"][rows, None]
        base = torch.arange(n, device="cuda")[:, None] * V + s["history"][rows].long()
        tally = lambda pick: torch.bincount(base[pick], minlength=n * V).reshape(n, V).double()
        generated, any_ = tally((where >= prompt) & (where < length)), tally(where < length)
        rho = s["repetition"][rows, None].double()
        z = torch.where(any_ == 0, z, torch.where(z > 0, z / rho, z * rho))
        z -= s["presence"][rows, None].double() * (generated != 0) + s["frequency"][rows, None].double() * generated
        if s["bias_id"] is not None:
            ids = s["bias_id"][rows].long()
            pick = ids >= 0
            at = (torch.arange(n, device="cuda")[:, None] * V + ids)[pick]
            z += torch.bincount(at, weights=s["bias_value"][rows].double()[pick], minlength=n * V).reshape(n, V)
        if s["allowed"] is not None:
            word = s["allowed"] if s["allowed"].dim() == 1 else s["allowed"][rows]
            place = torch.arange(V, device="cuda")
            ok = (word[..., place // 32].long() >> (place % 32)) & 1
            z = torch.where(ok != 0, z, torch.full_like(z, -math.inf))
        parts.append(z)
    return torch.cat(parts)
