"""What a neighbor node's training step needs around the stack calls, as cases that can be timed and compared.

  head_fwd    log-probabilities of given tokens under the LM head: log softmax(c U W^T)[row, label] and the log-sum-exp
  head_bwd    their gradient: dU and dW from the gradient of every row's log-probability
  preference  loss over pairs of sequences from their summed (or mean) log ratios, and the gradient of every token's
              log-probability
  policy      clipped policy loss with a KL term over sequences, with the same gradient
  ckpt        a tensor kept as an 8-bit checkpoint and read back: groups of 32 columns of a row share a power of two
  ckpt_bwd    the neighbor-mode backward of a block whose stored tensor H (and, where kept, G and Z) is such a checkpoint

`run` computes them in plain torch operations, or, where `own` is true, through paper_2510_16415_amd.binding.
Inputs are made on the GPU from the seed alone.  Activations N(0, 1), weights N(0, 0.02^2), log-probabilities as a
vocabulary of some ten thousand tokens gives them, sequences of uneven length whose first part (the prompt) is not counted.
"""
import math

import torch

own = False

EPS = 1e-6
VOCAB = 32000
GROUP = 32       # columns that share a power of two


def listed():
    return [
        # a handful of answers of one or two sentences: the launches are all it takes
        dict(name="pref_small", path="preference", pairs=4, mean_len=40, ref=True, mean=False),
        # a batch of long answers, without a reference model, mean log-probability and a margin
        dict(name="pref_long", path="preference", pairs=64, mean_len=4096, ref=False, mean=True),
        # rollouts of one step, an advantage per answer
        dict(name="policy_answers", path="policy", seqs=64, mean_len=300, ref=True, per_token=False, by_seq=True),
        # the largest rollout batch: long answers, an advantage per token
        dict(name="policy_long", path="policy", seqs=512, mean_len=2048, ref=True, per_token=True, by_seq=False),
        # one answer of odd length is scored
        dict(name="head_fwd_answer", path="head_fwd", dtype="bf16", tokens=77, d=1024, vocab=VOCAB),
        # a micro-batch of the 7B shape
        dict(name="head_fwd_7b", path="head_fwd", dtype="bf16", tokens=8192, d=4096, vocab=VOCAB),
        # reference precision, smallest model, a vocabulary of odd size
        dict(name="head_bwd_f32", path="head_bwd", dtype="f32", tokens=256, d=256, vocab=8191),
        # a micro-batch of the 1B shape, and one of the 7B shape
        dict(name="head_bwd_1b", path="head_bwd", dtype="bf16", tokens=2048, d=2048, vocab=VOCAB),
        dict(name="head_bwd_7b", path="head_bwd", dtype="bf16", tokens=8192, d=4096, vocab=VOCAB),
        # the stored tensor of one layer of the 7B shape
        dict(name="ckpt_7b", path="ckpt", dtype="bf16", rows=8192, cols=4096),
        # the reference-precision block from its checkpoint
        dict(name="ckpt_bwd_f32", path="ckpt_bwd", dtype="f32", tokens=256, d=256, f=688, rank=32, saved=False),
        # a layer of the 350M shape from checkpoints of H, G and Z, exact weight gradients
        dict(name="ckpt_bwd_350m", path="ckpt_bwd", dtype="bf16", tokens=4096, d=1024, f=2736, rank=0, saved=True),
    ]


def _log(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


def draw(rng):
    path = rng.choice(["preference", "policy", "head_fwd", "head_bwd", "ckpt", "ckpt_bwd"])
    if path == "preference":
        pairs = int(_log(rng, 1, 256))
        return dict(path=path, pairs=pairs, mean_len=int(_log(rng, 1, min(8192, 500000 // pairs))), ref=rng.random() < 0.7,
                    mean=rng.random() < 0.4)
    if path == "policy":
        seqs = int(_log(rng, 1, 1024))
        return dict(path=path, seqs=seqs, mean_len=int(_log(rng, 1, min(8192, 1000000 // seqs))), ref=rng.random() < 0.8,
                    per_token=rng.random() < 0.5, by_seq=rng.random() < 0.5)
    if path in ("head_fwd", "head_bwd"):
        if rng.random() < 0.2:
            return dict(path=path, dtype="f32", tokens=int(_log(rng, 1, 512)), d=int(_log(rng, 32, 512)),
                        vocab=int(_log(rng, 1000, 32000)))
        return dict(path=path, dtype="bf16", tokens=int(_log(rng, 1, 8192)), d=8 * int(_log(rng, 16, 512)),
                    vocab=int(_log(rng, 1000, 32000)))
    if path == "ckpt":
        rows = int(_log(rng, 1, 8192))
        return dict(path=path, dtype=rng.choice(["bf16", "bf16", "f32"]), rows=rows, cols=int(_log(rng, 8, min(11008, 3.3e7 / rows))))
    half = rng.random() < 0.5
    d = 8 * int(_log(rng, 16, 128 if half else 64))
    return dict(path=path, dtype="bf16" if half else "f32", tokens=int(_log(rng, 1, 4096 if half else 512)), d=d,
                f=int(d * rng.uniform(2.4, 3.0)), rank=0 if half else max(8, d // 8), saved=half and rng.random() < 0.5)


# ---- inputs ---------------------------------------------------------------------------------------
def _type(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _up(x, n=8):
    return (x + n - 1) // n * n


def _power(e):
    """2 ** (e - 127) of bytes 1 to 254, exact; 255 stands for NaN."""
    p = (e.int() << 23).view(torch.float32)
    return torch.where(e == 255, torch.full_like(p, math.nan), p)


def _groups(x):
    """[rows x cols] -> [rows x groups x GROUP], padded with zeros."""
    rows, cols = x.shape
    n = _up(cols, GROUP)
    y = torch.zeros(rows, n, dtype=torch.float32, device=x.device)
    y[:, :cols] = x
    return y.view(rows, n // GROUP, GROUP)


def _quantise(x):
    """q int8 [rows x groups x GROUP] and e uint8 [rows x groups] of a matrix."""
    y = _groups(x)
    most = y.abs().amax(2)
    fine = torch.isfinite(y).all(2)
    high = (torch.where(fine, most, torch.zeros_like(most)).view(torch.int32) >> 23)      # biased exponent of the largest
    e = torch.clamp(high, min=7) - 6
    inv = ((254 - e) << 23).view(torch.float32)
    q = torch.round(torch.where(fine[:, :, None], y, torch.zeros_like(y)) * inv[:, :, None]).clamp_(-127, 127)
    return q.to(torch.int8), torch.where(fine, e, torch.full_like(e, 255)).to(torch.uint8)


def _values(q, e, rows, cols):
    return (q.float() * _power(e)[:, :, None]).reshape(rows, -1)[:, :cols]


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(20251016 + int(seed))
    return _PREPARE[case["path"]](case, g, dict(case=case))


def _normal(g, shape, std, dtype):
    return (torch.randn(shape, generator=g, device="cuda") * std).to(dtype)


def _sequences(g, n, mean_len):
    """Offsets of n sequences, n * mean_len tokens in all, whose lengths spread by a factor of two, and which tokens count."""
    tokens = n * mean_len
    spread = torch.cumsum(torch.exp(0.5 * torch.randn(n, generator=g, device="cuda", dtype=torch.float64)), 0)
    off = torch.zeros(n + 1, dtype=torch.int64, device="cuda")
    off[1:] = torch.round(spread / spread[-1] * tokens).long()
    seq = torch.repeat_interleave(torch.arange(n, device="cuda"), off[1:] - off[:-1])
    prompt = (0.25 * (off[1:] - off[:-1])).long()
    mask = (torch.arange(tokens, device="cuda") - off[seq] >= prompt[seq]).to(torch.uint8)
    return off, mask, tokens


def _logps(g, mask):
    x = torch.randn(mask.shape, generator=g, device="cuda")
    return torch.where(mask > 0, -torch.log1p(torch.exp(1.5 * x - 0.5)) * 1.5, torch.zeros_like(x))


def _single(x):
    """A number as 32 bits hold it: which side of a border a value falls on goes by it."""
    return torch.tensor(x, dtype=torch.float32).item()


def _near(g, x, mask, std):
    return torch.where(mask > 0, x + std * torch.randn(x.shape, generator=g, device="cuda"), torch.zeros_like(x))


def _prepare_preference(case, g, s):
    off, mask, tokens = _sequences(g, 2 * case["pairs"], case["mean_len"])
    logp = _logps(g, mask)
    s.update(off=off, mask=mask, tokens=tokens, logp=logp, ref=_near(g, logp, mask, 0.1) if case["ref"] else None)
    s.update(beta=0.1 if case["ref"] else 2.0, smooth=0.1 if case["mean"] else 0.0, margin=0.5 if case["mean"] else 0.0)
    return s


def _prepare_policy(case, g, s):
    off, mask, tokens = _sequences(g, case["seqs"], case["mean_len"])
    logp = _logps(g, mask)
    old = _near(g, logp, mask, 0.15)
    adv = torch.randn(tokens if case["per_token"] else case["seqs"], generator=g, device="cuda")
    s.update(off=off, mask=mask, tokens=tokens, logp=logp, old=old, ref=_near(g, logp, mask, 0.2) if case["ref"] else None,
             adv=adv, low=_single(0.2), high=_single(0.28), kl=0.04 if case["ref"] else 0.0)
    return s


def _prepare_head(case, g, s):
    b, d, v, t = case["tokens"], case["d"], case["vocab"], _type(case)
    s.update(U=_normal(g, (b, d), 1.0, t), W=_normal(g, (v, d), 0.02, t))
    labels = torch.randint(0, v, (b,), generator=g, device="cuda")
    skipped = torch.rand(b, generator=g, device="cuda") < 0.1      # tokens that are not scored
    skipped[0] = False
    s["labels"] = torch.where(skipped, torch.full_like(labels, -1), labels)
    if case["path"] == "head_bwd":
        # what the forward pass kept, and what the loss hands back
        lse = torch.logsumexp(torch.matmul(s["U"].float(), s["W"].float().t()), 1)
        s.update(lse=lse, dlogp=-torch.rand(b, generator=g, device="cuda") / b)
    return s


def _kept(x):
    """x in rows of a multiple of eight elements, as the library's 16-bit tensors have them."""
    y = torch.zeros(x.shape[0], _up(x.shape[1]), dtype=x.dtype, device="cuda")[:, :x.shape[1]]
    return y.copy_(x)


def _prepare_ckpt(case, g, s):
    x = torch.randn(case["rows"], case["cols"], generator=g, device="cuda")
    loud = torch.rand(case["cols"], generator=g, device="cuda") < 0.01      # a residual stream has a few loud columns
    s["X"] = _kept(torch.where(loud[None, :], 20 * x, x).to(_type(case)))
    return s


def _prepare_ckpt_bwd(case, g, s):
    b, d, f, r, t = case["tokens"], case["d"], case["f"], case["rank"], _type(case)
    H = _normal(g, (b, d), 1.0, t)
    s.update(dOut=_normal(g, (b, d), 1.0, t), gamma=(1 + _normal(g, (d,), 0.1, torch.float32)).to(t))
    s.update({k: _normal(g, (f, d), 0.02, t) for k in ("Wg", "Wu")}, Wd=_kept(_normal(g, (d, f), 0.02, t)))
    s["H"] = _quantise(H)
    if case["saved"]:
        h = _values(*s["H"], b, d)
        u = h * torch.rsqrt(h.square().mean(1, keepdim=True) + EPS) * s["gamma"].float()
        s["G"], s["Z"] = (_quantise(torch.matmul(u, s[k].float().t())) for k in ("Wg", "Wu"))
    if r:
        s.update(Pg=_normal(g, (d, r), d ** -0.5, t), Pu=_normal(g, (d, r), d ** -0.5, t), Pd=_normal(g, (f, r), f ** -0.5, t))
    return s


_PREPARE = dict(preference=_prepare_preference, policy=_prepare_policy, head_fwd=_prepare_head, head_bwd=_prepare_head,
                ckpt=_prepare_ckpt, ckpt_bwd=_prepare_ckpt_bwd)


# ---- one pass -------------------------------------------------------------------------------------
def run(s):
    path = s["case"]["path"]
    return (_OWN if own else _PLAIN)[path](s)


def _segments(s, x, n):
    """Sums of a token array over its sequences, and every token's sequence, in 64 bits."""
    ids = torch.searchsorted(s["off"], torch.arange(x.shape[0], device="cuda"), right=True) - 1
    return torch.zeros(n, dtype=torch.float64, device="cuda").index_add_(0, ids, x), ids


def _plain_preference(s):
    case, n = s["case"], s["case"]["pairs"]
    m = s["mask"].double()
    x = torch.where(s["mask"] > 0, s["logp"].double() - (s["ref"].double() if case["ref"] else 0.0), 0.0)
    r, ids = _segments(s, x, 2 * n)
    per = torch.full((2 * n,), s["beta"], dtype=torch.float64, device="cuda")
    if case["mean"]:
        count, _ = _segments(s, m, 2 * n)
        per = per / torch.clamp(count, min=1)
    r = r * per
    h = r[0::2] - r[1::2] - s["margin"]
    e = s["smooth"]
    soft = lambda t: torch.clamp(t, min=0) + torch.log1p(torch.exp(-t.abs()))      # noqa: E731
    loss = ((1 - e) * soft(-h) + e * soft(h)).mean()
    dh = (-(1 - e) / (1 + torch.exp(h)) + e / (1 + torch.exp(-h))) / n
    ds = torch.stack((dh, -dh), 1).reshape(-1) * per
    return dict(loss=loss.float().reshape(1), margins=h.float(), rewards=r.float(), dlogp=(ds[ids] * m).float())


def _plain_policy(s):
    case, n = s["case"], s["case"]["seqs"]
    on = s["mask"] > 0
    m = s["mask"].double()
    zero = torch.zeros_like(m)
    diff = torch.where(on, s["logp"].double() - s["old"].double(), zero)
    q = torch.where(on, s["ref"].double() - s["logp"].double(), zero) if case["ref"] else zero
    count, ids = _segments(s, m, n)
    if case["by_seq"]:
        w = m / (torch.clamp(count, min=1) * torch.clamp((count > 0).sum(), min=1))[ids]
    else:
        w = m / torch.clamp(m.sum(), min=1)
    A = s["adv"].double() if case["per_token"] else s["adv"].double()[ids]
    rho = torch.exp(diff)
    over = ((A > 0) & (diff > math.log1p(s["high"]))) | ((A < 0) & (diff < math.log1p(-s["low"])))
    kept = torch.clamp(rho, 1 - s["low"], 1 + s["high"])
    kl = torch.expm1(q) - q
    loss = (w * (s["kl"] * kl - torch.where(over, kept, rho) * A)).sum()
    d = w * (torch.where(over, zero, -rho * A) - s["kl"] * torch.expm1(q))
    return dict(loss=loss.float().reshape(1), kl=(w * kl).sum().float().reshape(1),
                clipped=(w * over).sum().float().reshape(1), dlogp=d.float())


def _plain_head_fwd(s):
    z = torch.matmul(s["U"].float(), s["W"].float().t())
    lse = torch.logsumexp(z, 1)
    at = torch.gather(z, 1, torch.clamp(s["labels"], min=0)[:, None])[:, 0]
    return dict(logp=torch.where(s["labels"] >= 0, at - lse, torch.zeros_like(lse)), lse=lse)


def _plain_head_bwd(s):
    U, W = s["U"].float(), s["W"].float()
    dz = torch.matmul(U, W.t()).sub_(s["lse"][:, None]).exp_()
    c = torch.where(s["labels"] >= 0, s["dlogp"], torch.zeros_like(s["dlogp"]))
    dz.mul_(-c[:, None])
    dz.scatter_add_(1, torch.clamp(s["labels"], min=0)[:, None], c[:, None])
    return dict(dU=torch.matmul(dz, W).to(s["U"].dtype), dW=torch.matmul(dz.t(), U).to(s["W"].dtype))


def _plain_ckpt(s):
    x = s["X"]
    return _values(*_quantise(x), *x.shape).to(x.dtype)


def _plain_ckpt_bwd(s):
    case = s["case"]
    b, d, f, t = case["tokens"], case["d"], case["f"], _type(case)
    w = {k: s[k].float() for k in ("Wg", "Wu", "Wd", "dOut", "gamma")}
    H = _values(*s["H"], b, d)
    rs = torch.rsqrt(H.square().mean(1, keepdim=True) + EPS)
    N = H * rs
    U = N * w["gamma"]
    G, Z = (_values(*s[k], b, f) if case["saved"] else torch.matmul(U, w[m].t()) for k, m in (("G", "Wg"), ("Z", "Wu")))
    sg = torch.sigmoid(G)
    A = G * sg * Z
    dA = torch.matmul(w["dOut"], w["Wd"])
    dZ = dA * G * sg
    dG = dA * Z * (sg * (1 + G * (1 - sg)))
    dU = torch.matmul(dG, w["Wg"]) + torch.matmul(dZ, w["Wu"])
    dN = dU * w["gamma"]
    out = dict(dX=w["dOut"] + rs * (dN - N * (dN * N).mean(1, keepdim=True)), dgamma=(dU * N).sum(0))
    if case["rank"]:
        P = {k: s[k].float() for k in ("Pg", "Pu", "Pd")}
        part = lambda gy, x, p: torch.matmul(torch.matmul(gy.t(), torch.matmul(x, p)), p.t())      # noqa: E731
        out.update(dWg=part(dG, U, P["Pg"]), dWu=part(dZ, U, P["Pu"]), dWd=part(w["dOut"], A, P["Pd"]))
    else:
        out.update(dWg=torch.matmul(dG.t(), U), dWu=torch.matmul(dZ.t(), U), dWd=torch.matmul(w["dOut"].t(), A))
    return {k: v.to(t) for k, v in out.items()}


_PLAIN = dict(preference=_plain_preference, policy=_plain_policy, head_fwd=_plain_head_fwd, head_bwd=_plain_head_bwd,
              ckpt=_plain_ckpt, ckpt_bwd=_plain_ckpt_bwd)


# ---- the framework's calls --------------------------------------------------------------------------
def _bytes(n):
    return torch.empty(max(1, n), dtype=torch.uint8, device="cuda")


def _f32(*shape):
    return torch.empty(shape, dtype=torch.float32, device="cuda")


def _code(B, case):
    return B.BF16 if case["dtype"] == "bf16" else B.F32


def _own_preference(s):
    from paper_2510_16415_amd import binding as B
    n = s["case"]["pairs"]
    if "ws" not in s:
        s["desc"] = B.make_preference_desc(s["tokens"], n, beta=s["beta"], label_smoothing=s["smooth"], margin=s["margin"],
                                           length_mean=s["case"]["mean"])
        s["ws"] = _bytes(B.mecefo_preference_workspace_bytes(s["desc"]))
        s["out"] = dict(loss=_f32(1), margins=_f32(n), rewards=_f32(2 * n), dlogp=_f32(s["tokens"]))
    o = s["out"]
    B.mecefo_preference_loss(s["desc"], s["logp"], s["ref"], s["mask"], s["off"], o["loss"], o["margins"], o["rewards"],
                             o["dlogp"], s["ws"])
    return o


def _own_policy(s):
    from paper_2510_16415_amd import binding as B
    case = s["case"]
    if "ws" not in s:
        s["desc"] = B.make_policy_desc(s["tokens"], case["seqs"], clip_low=s["low"], clip_high=s["high"], kl_coef=s["kl"],
                                       mean=B.MEAN_SEQUENCES if case["by_seq"] else B.MEAN_TOKENS,
                                       advantage_per_token=case["per_token"])
        s["ws"] = _bytes(B.mecefo_policy_workspace_bytes(s["desc"]))
        s["out"] = dict(loss=_f32(1), kl=_f32(1), clipped=_f32(1), dlogp=_f32(s["tokens"]))
    o = s["out"]
    B.mecefo_policy_loss(s["desc"], s["logp"], s["old"], s["ref"], s["adv"], s["mask"], s["off"], o["loss"], o["kl"],
                         o["clipped"], o["dlogp"], s["ws"])
    return o


def _own_head(s):
    from paper_2510_16415_amd import binding as B
    case = s["case"]
    b, d, v = case["tokens"], case["d"], case["vocab"]
    back = case["path"] == "head_bwd"
    if "ws" not in s:
        s["desc"] = B.make_head_desc(b, d, v, _code(B, case), _code(B, case))
        s["ws"] = _bytes(B.mecefo_head_workspace_bytes(s["desc"], back))
        s["out"] = (dict(dU=torch.empty_like(s["U"]), dW=torch.empty_like(s["W"])) if back else
                    dict(logp=_f32(b), lse=_f32(b)))
    o = s["out"]
    if back:
        B.mecefo_head_logprob_bwd(s["desc"], s["U"], None, s["W"], s["labels"], s["lse"], s["dlogp"], o["dU"], None, o["dW"],
                                  0, s["ws"])
    else:
        B.mecefo_head_logprob_fwd(s["desc"], s["U"], None, s["W"], s["labels"], o["logp"], o["lse"], s["ws"])
    return o


def _new_ckpt(B, rows, cols):
    n = _up(cols, GROUP)
    return B.ckpt(torch.empty(rows, n, dtype=torch.int8, device="cuda"),
                  torch.empty(rows, n // GROUP, dtype=torch.uint8, device="cuda"))


def _own_ckpt(s):
    from paper_2510_16415_amd import binding as B
    case, X = s["case"], s["X"]
    rows, cols = X.shape
    if "out" not in s:
        s["c"] = _new_ckpt(B, rows, cols)
        s["out"] = torch.empty(rows, _up(cols), dtype=X.dtype, device="cuda")[:, :cols]
    B.mecefo_checkpoint_pack(_code(B, case), X, rows, cols, X.stride(0), s["c"])
    B.mecefo_checkpoint_unpack(_code(B, case), s["c"], rows, cols, s["out"], X.stride(0))
    return s["out"]


def _own_ckpt_bwd(s):
    from paper_2510_16415_amd import binding as B
    case = s["case"]
    b, d, f, r, t = case["tokens"], case["d"], case["f"], case["rank"], _type(case)
    if "ws" not in s:
        code = _code(B, case)
        s["desc"] = B.make_desc(b, d, f, code, code, ld_act_f=_up(f), ld_w_df=_up(f), rms_eps=EPS)
        s["ws"] = _bytes(B.mecefo_block_ckpt_workspace_bytes(s["desc"], r, r, r))
        s["c"] = {k: B.ckpt(s[k][0].view(b, -1), s[k][1]) for k in ("H", "G", "Z") if k in s}
        s["P"] = [B.proj(s[k]) if r else None for k in ("Pg", "Pu", "Pd")]
        s["out"] = dict(dX=torch.empty(b, d, dtype=t, device="cuda"), dgamma=torch.empty(d, dtype=t, device="cuda"),
                        **{"d" + k: torch.empty_like(s[k]) for k in ("Wg", "Wu")},
                        dWd=torch.empty(d, _up(f), dtype=t, device="cuda")[:, :f])
    o, c = s["out"], s["c"]
    B.mecefo_block_bwd_skip_ckpt(s["desc"], c["H"], s["dOut"], s["gamma"], s["Wg"], s["Wu"], s["Wd"], *s["P"], B.SIDE_INPUT,
                                 o["dX"], o["dgamma"], o["dWg"], o["dWu"], o["dWd"], 0, s["ws"], G=c.get("G"), Z=c.get("Z"),
                                 exact_wgrad_mask=0 if r else 7)
    return o


_OWN = dict(preference=_own_preference, policy=_own_policy, head_fwd=_own_head, head_bwd=_own_head, ckpt=_own_ckpt,
            ckpt_bwd=_own_ckpt_bwd)


# ---- what a pass cannot do without ------------------------------------------------------------------
def work(case):
    path = case["path"]
    if path in ("preference", "policy"):
        n = case["pairs"] * 2 if path == "preference" else case["seqs"]
        tokens = n * case["mean_len"]
        arrays = 1 + case["ref"] + (1 + case["per_token"] if path == "policy" else 0)
        return {"bytes": tokens * (4 * arrays + 1 + 4) + n * 16, "flops": tokens * (4 if path == "preference" else 30)}
    if path in ("head_fwd", "head_bwd"):
        b, d, v, e = case["tokens"], case["d"], case["vocab"], 2 if case["dtype"] == "bf16" else 4
        if path == "head_fwd":
            return {"bytes": (b + v) * d * e + 16 * b, "flops": 2 * b * d * v}
        return {"bytes": 2 * (b + v) * d * e + 16 * b, "flops": 6 * b * d * v}
    e = 2 if case["dtype"] == "bf16" else 4
    if path == "ckpt":
        n = case["rows"] * case["cols"]
        return {"bytes": n * 2 * (e + 33 / 32), "flops": 4 * n}
    b, d, f, r = case["tokens"], case["d"], case["f"], case["rank"]
    kept = b * (d + (2 * f if case["saved"] else 0)) * 33 / 32
    grads = 6 * r * (d + f) * b + 6 * r * d * f if r else 6 * b * d * f
    return {"bytes": kept + 2 * b * d * e + 6 * d * f * e + (r * (2 * d + f)) * e,
            "flops": b * d * f * (6 if case["saved"] else 10) + grads}


# ---- the same in 64 bits, from the definitions --------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    return _EXACT[case["path"]](case, {k: v.double() if isinstance(v, torch.Tensor) and v.is_floating_point() else v
                                       for k, v in s.items()})


def _exact_scores(s, take, i):
    at = slice(int(s["off"][i]), int(s["off"][i + 1]))
    return at, s["mask"][at].bool(), take[at]


def _exact_preference(case, s):
    ratio = s["logp"] - s["ref"] if case["ref"] else s["logp"]
    n = case["pairs"]
    d = torch.zeros_like(ratio)
    rewards, margins, total = [], [], 0.0
    for i in range(n):
        (at_c, on_c, x_c), (at_r, on_r, x_r) = (_exact_scores(s, ratio, 2 * i + k) for k in (0, 1))
        div = [max(1, int(on.sum())) if case["mean"] else 1 for on in (on_c, on_r)]
        pair = [s["beta"] * float(x[on].sum()) / k for x, on, k in ((x_c, on_c, div[0]), (x_r, on_r, div[1]))]
        h = pair[0] - pair[1] - s["margin"]
        good, bad = (1 / (1 + math.exp(-h)), 1 / (1 + math.exp(h)))
        total += -(1 - s["smooth"]) * _log_sigmoid(h) - s["smooth"] * _log_sigmoid(-h)
        slope = s["beta"] * (s["smooth"] * good - (1 - s["smooth"]) * bad) / n
        d[at_c] = on_c * (slope / div[0])
        d[at_r] = on_r * (-slope / div[1])
        rewards += pair
        margins.append(h)
    make = lambda v: torch.tensor(v, dtype=torch.float64)      # noqa: E731
    return dict(loss=make([total / n]), margins=make(margins), rewards=make(rewards), dlogp=d)


def _log_sigmoid(h):
    return -math.log1p(math.exp(-h)) if h >= 0 else h - math.log1p(math.exp(h))


def _exact_policy(case, s):
    n = case["seqs"]
    parts = [_exact_scores(s, torch.arange(s["tokens"], device="cuda"), i) for i in range(n)]
    counts = [int(on.sum()) for _, on, _ in parts]
    live = max(1, sum(c > 0 for c in counts))
    every = max(1, sum(counts))
    d = torch.zeros_like(s["logp"])
    loss = kl_sum = share = 0.0
    for i, (at, on, tok) in enumerate(parts):
        if not counts[i]:
            continue
        w = 1 / (counts[i] * live) if case["by_seq"] else 1 / every
        t = tok[on]
        A = s["adv"][t] if case["per_token"] else s["adv"][i].expand(len(t))
        rho = torch.exp(s["logp"][t] - s["old"][t])
        bounded = torch.clamp(rho, 1 - s["low"], 1 + s["high"])
        gain = torch.minimum(rho * A, bounded * A)
        flat = bounded * A < rho * A
        u = torch.exp(s["ref"][t] - s["logp"][t]) if case["ref"] else torch.ones_like(rho)
        q = s["ref"][t] - s["logp"][t] if case["ref"] else torch.zeros_like(rho)
        k = u - q - 1
        loss += w * float((s["kl"] * k - gain).sum())
        kl_sum += w * float(k.sum())
        share += w * float(flat.sum())
        d[t] = w * (s["kl"] * (1 - u) - torch.where(flat, torch.zeros_like(rho), rho) * A)
    make = lambda v: torch.tensor([v], dtype=torch.float64)      # noqa: E731
    return dict(loss=make(loss), kl=make(kl_sum), clipped=make(share), dlogp=d)


def _exact_head_fwd(case, s):
    z = torch.matmul(s["U"], s["W"].t())
    top = z.max(1, keepdim=True).values
    lse = top[:, 0] + torch.log(torch.exp(z - top).sum(1))
    rows = torch.arange(case["tokens"], device="cuda")
    scored = s["labels"] >= 0
    logp = torch.where(scored, z[rows, s["labels"].clamp(min=0)] - lse, torch.zeros_like(lse))
    return dict(logp=logp, lse=lse)


def _exact_head_bwd(case, s):
    dz = torch.exp(torch.matmul(s["U"], s["W"].t()) - s["lse"][:, None]).neg_()
    rows = torch.arange(case["tokens"], device="cuda")
    scored = s["labels"] >= 0
    dz[rows, s["labels"].clamp(min=0)] += scored.double()
    dz *= (s["dlogp"] * scored)[:, None]
    return dict(dU=torch.matmul(dz, s["W"]), dW=torch.matmul(dz.t(), s["U"]))


def _exact_power(e):
    """2 ** e in 64 bits, by its bits."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _exact_ckpt(case, s):
    x = s["X"]
    out = torch.empty_like(x)
    for c in range(0, case["cols"], GROUP):
        part = x[:, c:c + GROUP]
        most = part.abs().amax(1, keepdim=True)
        step = _exact_power(torch.clamp(torch.frexp(most).exponent - 1, min=-120) - 6)
        out[:, c:c + GROUP] = torch.clamp(torch.round(part / step), -127, 127) * step
    return out


def _exact_ckpt_bwd(case, s):
    b, d, f = case["tokens"], case["d"], case["f"]
    back = lambda c, n: (c[0].double() * _exact_power(c[1].int() - 127)[:, :, None]).reshape(b, -1)[:, :n]      # noqa: E731
    H = back(s["H"], d)
    r = 1 / torch.sqrt((H * H).sum(1, keepdim=True) / d + EPS)
    U = H * r * s["gamma"]
    G = back(s["G"], f) if case["saved"] else U @ s["Wg"].t()
    Z = back(s["Z"], f) if case["saved"] else U @ s["Wu"].t()
    sig = 1 / (1 + torch.exp(-G))
    silu = G * sig
    dA = s["dOut"] @ s["Wd"]
    dZ, dG = dA * silu, dA * Z * (sig + silu * (1 - sig))
    dU = dG @ s["Wg"] + dZ @ s["Wu"]
    dN = dU * s["gamma"]
    dX = s["dOut"] + r * dN - H * r ** 3 * (dN * H).sum(1, keepdim=True) / d
    out = dict(dX=dX, dgamma=(dU * H * r).sum(0))
    for k, gy, x in (("g", dG, U), ("u", dZ, U), ("d", s["dOut"], silu * Z)):
        if case["rank"]:
            P = s["P" + k]
            out["dW" + k] = gy.t() @ (x @ P) @ P.t()
        else:
            out["dW" + k] = gy.t() @ x
    return out


_EXACT = dict(preference=_exact_preference, policy=_exact_policy, head_fwd=_exact_head_fwd, head_bwd=_exact_head_bwd,
              ckpt=_exact_ckpt, ckpt_bwd=_exact_ckpt_bwd)
