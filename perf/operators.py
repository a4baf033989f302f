"""The losses at a model's output head, as cases whose speed is watched.

The head is a dense bf16 matrix W [N][K] over the vocabulary (N rows), x [T][K] are the last hidden states, z = x W^T the
logits, which are never an output.  Two operators, each forward alone (scoring, validation) or forward and backward (a
training step, which returns the gradients too):

  ce       softmax cross entropy: loss[t] = log sum_i exp z[t][i] - z[t][labels[t]]; rows with a negative label are left
           out (loss 0, no gradient)
  distill  distillation from a teacher's top logits: q = softmax of the teacher's k logits / tau over the entries that are
           there (index >= 0), p = softmax of z / tau over the whole vocabulary, loss[t] = sum_j q_j (log q_j - log p_j);
           with `labels` the cross entropy of the same logits as well, in the same pass

Hidden sizes are those of the layers in the package's ``inputs.py`` and sizes around them; vocabularies run from a
thousand (characters, a domain's own tokens) to 150 thousand rows, most of them not a multiple of anything.
"""
from __future__ import annotations

import math

import torch

own = False

BF16, F32, F64 = torch.bfloat16, torch.float32, torch.float64


def _ce(T, K, N, train, ignored):
    return dict(kind="ce", T=T, K=K, N=N, train=train, ignored=ignored)


def _distill(T, K, N, top, tau, train, labels, teacher="f32", ignored=0.0):
    return dict(kind="distill", T=T, K=K, N=N, top=top, tau=tau, train=train, labels=labels, teacher=teacher, ignored=ignored)


def listed():
    return [
        # scoring the next token of one sequence against a given continuation: latency counts
        dict(_ce(1, 1024, 1009, False, 0.0), name="ce_score_1tok_small"),
        # the same at the 2B-shaped layers' hidden size and an ordinary vocabulary: the head streams from memory
        dict(_ce(1, 2560, 32000, False, 0.0), name="ce_score_1tok"),
        # validation perplexity over one sequence, odd vocabulary
        dict(_ce(2048, 2560, 50257, False, 0.0), name="ce_validate_2048tok"),
        # training step on a short ragged batch with padding
        dict(_ce(200, 1024, 10007, True, 0.25), name="ce_train_200tok"),
        # an ordinary training step
        dict(_ce(4096, 2560, 32000, True, 0.0), name="ce_train_4096tok"),
        # fine-tuning on answers: half of the tokens are prompt and carry no label
        dict(_ce(3001, 2048, 65537, True, 0.5), name="ce_train_half_ignored"),
        # the largest training step: a wide head and a large vocabulary
        dict(_ce(4096, 4096, 131072, True, 0.0), name="ce_train_large"),
        # distillation, smallest: few tokens, a small vocabulary
        dict(_distill(16, 1024, 4099, 8, 1.0, True, False), name="distill_train_16tok"),
        # measuring how far a student is from its teacher, no gradients
        dict(_distill(333, 2560, 32000, 20, 1.0, False, False, teacher="bf16"), name="distill_score_333tok"),
        # an ordinary distillation step together with the labels' loss
        dict(_distill(2048, 2560, 32000, 32, 2.0, True, True, ignored=0.1), name="distill_train_2048tok_labels"),
        # a long batch, a large vocabulary, many teacher entries
        dict(_distill(4096, 2048, 100003, 64, 2.0, True, False, teacher="bf16"), name="distill_train_4096tok"),
    ]


def draw(rng):
    # none larger than the largest training step above
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    most = 4096 * 4096 * 131072
    while True:
        T, N, K = log_int(1, 6000), log_int(1000, 152000), 128 * rng.randint(4, 32)
        if T * N * K > most:
            continue
        train, ignored = rng.random() < 0.67, rng.choice([0.0, 0.0, 0.1, 0.5])
        if rng.random() < 0.5:
            return _ce(T, K, N, train, ignored)
        return _distill(T, K, N, log_int(1, 128), rng.choice([1.0, 1.5, 2.0, 4.0]), train, rng.random() < 0.5,
                        teacher=rng.choice(["f32", "bf16"]), ignored=ignored)


# -- inputs ----------------------------------------------------------------------------------------
def prepare(case, seed):
    """Hidden states that lean towards their label's row (a partly trained model: some tokens are sure, some are not), a
    head of N(0, 0.02^2); `ignored` of the rows carry no label (-100) and, for the distillation, no teacher entries."""
    T, K, N = case["T"], case["K"], case["N"]
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def rand(*shape):
        return torch.rand(*shape, generator=gen, device="cuda")

    def randn(*shape):
        return torch.randn(*shape, generator=gen, device="cuda")

    head = (randn(N, K) * 0.02).to(BF16)
    y = torch.randint(0, N, (T,), generator=gen, device="cuda")
    sure = rand(T, 1) * (math.log(N) * 50.0 / K)                        # label logits up to log N: probabilities up to a half
    x = (randn(T, K) + sure * head[y].float() * 50.0).to(BF16)
    keep = rand(T) >= case["ignored"]
    s = dict(case=case, x=x, head=head)
    if case["kind"] == "ce" or case["labels"]:
        s["labels"] = torch.where(keep, y, torch.full_like(y, -100))
        s["d_ce"] = torch.full((T,), 1.0, device="cuda") / keep.sum().clamp(min=1)      # gradient of the mean
    if case["kind"] == "distill":
        k = case["top"]
        # distinct indices (one from each of k parts of the vocabulary) in random order, the label's among them
        index = ((torch.arange(k, device="cuda") + rand(T, k)) * (N / k)).long().clamp(max=N - 1)
        part = (y * k // N).clamp(max=k - 1)
        index.scatter_(1, part[:, None], y[:, None])
        index = index.gather(1, rand(T, k).argsort(1))
        logits = randn(T, k) * 2.0 + 8.0 * (index == y[:, None])
        # rows are not all full: the last entries of some are absent
        absent = (torch.arange(k, device="cuda")[None] >= 1 + (rand(T, 1) * 4 * k).long()) | ~keep[:, None]
        s["top_index"] = torch.where(absent, torch.full_like(index, -1), index)
        s["top_logits"] = logits.to(BF16 if case["teacher"] == "bf16" else F32)
        s["d_distill"] = (0.5 + rand(T)) * (case["tau"] ** 2 / T)                       # weights per token
    return s


# -- the passes ------------------------------------------------------------------------------------
def run(state):
    case = state["case"]
    if own:
        return _own_ce(state) if case["kind"] == "ce" else _own_distill(state)
    return _plain(state)


def _own_ce(s):
    from paper_2603_05168_b200 import binding as b
    case, x, head = s["case"], s["x"], s["head"]
    (T, K), N = x.shape, head.shape[0]
    loss, lse = x.new_empty(T, dtype=F32), x.new_empty(T, dtype=F32)
    b.sbn_head_cross_entropy(x, head, s["labels"], loss, lse, ws=b.alloc_head_ws(T, N, K))
    if not case["train"]:
        return dict(ce=loss, lse=lse)
    dx, dhead = torch.empty_like(x), torch.empty_like(head)
    b.sbn_head_cross_entropy_backward(x, head, s["labels"], lse, s["d_ce"], dx=dx, dhead=dhead,
                                      ws=b.alloc_head_ws(T, N, K, backward=True))
    return dict(ce=loss, dx=dx, dhead=dhead)


def _own_distill(s):
    from paper_2603_05168_b200 import binding as b
    case, x, head, labels = s["case"], s["x"], s["head"], s.get("labels")
    (T, K), N, top, tau = x.shape, head.shape[0], case["top"], case["tau"]
    out = dict(distill=x.new_empty(T, dtype=F32))
    if labels is not None:
        out["ce"] = x.new_empty(T, dtype=F32)
    lse = x.new_empty((2, T) if labels is not None else (1, T), dtype=F32)
    b.sbn_head_distill(x, head, s["top_index"], s["top_logits"], tau, out["distill"], lse, labels=labels, ce_loss=out.get("ce"),
                       ws=b.alloc_head_ws(T, N, K, top=top))
    if not case["train"]:
        return dict(out, lse=lse)
    out["dx"], out["dhead"] = torch.empty_like(x), torch.empty_like(head)
    b.sbn_head_distill_backward(x, head, s["top_index"], s["top_logits"], tau, lse, s["d_distill"], labels=labels,
                                d_ce=s.get("d_ce"), dx=out["dx"], dhead=out["dhead"],
                                ws=b.alloc_head_ws(T, N, K, top=top, backward=True))
    return out


def _log_sum_exp(z):
    m = z.max(1, keepdim=True).values
    return (z - m).exp().sum(1).log() + m[:, 0]


def _plain(s):
    """Everything in 32 bits, the logits and their gradient as whole matrices."""
    case, head, labels = s["case"], s["head"].float(), s.get("labels")
    there = torch.zeros(case["T"], dtype=torch.bool, device="cuda")
    if labels is not None:
        there |= labels >= 0
    if case["kind"] == "distill":
        present = s["top_index"] >= 0
        there |= present.any(1)
    x = torch.where(there[:, None], s["x"], 0.0).float()
    z = x @ head.T
    out, dz, lses = {}, 0.0, []
    if case["kind"] == "distill":
        tau = case["tau"]
        full = present.any(1)
        lse = _log_sum_exp(z / tau)
        lses.append(torch.where(full, lse, 0.0))
        l = torch.where(present, s["top_logits"].float() / tau, -math.inf)
        l = torch.where(full[:, None], l, 0.0)
        e = (l - l.max(1, keepdim=True).values).exp()
        q = torch.where(present, e / e.sum(1, keepdim=True), 0.0)
        at = s["top_index"].clamp(min=0)
        log_p = z.gather(1, at) / tau - lse[:, None]
        out["distill"] = torch.where(q > 0, q * (q.clamp(min=1e-45).log() - log_p), 0.0).sum(1)
        if case["train"]:
            g = torch.where(full, s["d_distill"] / tau, 0.0)
            dz = (z / tau - lse[:, None]).exp() * g[:, None]
            dz.scatter_add_(1, at, -q * g[:, None])
    if labels is not None:
        keep, at = labels >= 0, labels.clamp(min=0)[:, None]
        lse = _log_sum_exp(z)
        lses.append(torch.where(keep, lse, 0.0))
        out["ce"] = torch.where(keep, lse - z.gather(1, at)[:, 0], 0.0)
        if case["train"]:
            g = torch.where(keep, s["d_ce"], 0.0)
            dz = dz + (z - lse[:, None]).exp() * g[:, None]
            dz.scatter_add_(1, at, -g[:, None])
    if not case["train"]:
        out["lse"] = lses[0] if case["kind"] == "ce" else torch.stack(lses)
        return out
    out["dx"] = (dz @ head).to(BF16)
    out["dhead"] = (dz.T @ x).to(BF16)
    return out


# -- what a pass cannot do without -----------------------------------------------------------------
def work(case):
    """The products over the rows that count (z, and for training dx and dW); every input and output once."""
    T, K, N = case["T"], case["K"], case["N"]
    rows = T * (1.0 - case["ignored"])
    nbytes = 2.0 * K * (rows + N) + 8.0 * T
    if case["kind"] == "ce" or case["labels"]:
        nbytes += 12.0 * T
    if case["kind"] == "distill":
        nbytes += T * case["top"] * (8.0 + (2 if case["teacher"] == "bf16" else 4))
    if case["train"]:
        nbytes += 2.0 * K * (T + N)
    return dict(bytes=nbytes, flops=2.0 * rows * K * N * (3 if case["train"] else 1))


# -- the definition, in 64 bits --------------------------------------------------------------------
def exact(case, seed):
    """Token by token in blocks, in float64: probabilities from logits that have their row's maximum taken off, targets as a
    dense matrix."""
    s = prepare(case, seed)
    W = s["head"].to(F64)
    T, N, K = case["T"], case["N"], case["K"]
    labels = s.get("labels")
    out = {name: [] for name in ("distill", "ce", "lse0", "lse1", "dx")}
    dW = torch.zeros(N, K, dtype=F64, device="cuda") if case["train"] else None
    rows = max(1, min(T, (1 << 28) // N))
    for a in range(0, T, rows):
        b = min(T, a + rows)
        X = s["x"][a:b].to(F64)
        Z = X @ W.T
        G = torch.zeros_like(Z)
        counts = torch.zeros(b - a, dtype=torch.bool, device="cuda")
        if case["kind"] == "distill":
            index, tau = s["top_index"][a:b], case["tau"]
            Q = torch.zeros(b - a, N + 1, dtype=F64, device="cuda")          # column N takes the absent entries
            teacher = torch.softmax(torch.where(index < 0, torch.full_like(s["top_logits"][a:b], -math.inf, dtype=F64),
                                                s["top_logits"][a:b].to(F64) / tau), dim=1)
            full = (index >= 0).sum(1) > 0
            teacher = torch.nan_to_num(teacher, nan=0.0)
            Q.scatter_add_(1, torch.where(index < 0, N, index), teacher)
            Q = Q[:, :N]
            log_p = torch.log_softmax(Z / tau, dim=1)
            entropy = torch.special.xlogy(teacher, teacher).sum(1)
            out["distill"].append(torch.where(full, entropy - (Q * log_p).sum(1), 0.0))
            out["lse0"].append(torch.where(full, torch.logsumexp(Z / tau, 1), 0.0))
            if case["train"]:
                G += (log_p.exp() - Q) * torch.where(full, s["d_distill"][a:b].to(F64) / tau, 0.0)[:, None]
            counts |= full
            del Q, log_p
        if labels is not None:
            y = labels[a:b]
            has = y >= 0
            log_p = torch.log_softmax(Z, dim=1)
            pick = log_p.gather(1, torch.where(has, y, 0)[:, None])[:, 0]
            out["ce"].append(torch.where(has, -pick, 0.0))
            out["lse1"].append(torch.where(has, torch.logsumexp(Z, 1), 0.0))
            if case["train"]:
                P = log_p.exp()
                P[torch.arange(b - a, device="cuda")[has], y[has]] -= 1.0
                G += P * torch.where(has, s["d_ce"][a:b].to(F64), 0.0)[:, None]
                del P
            counts |= has
            del log_p
        if case["train"]:
            G[~counts] = 0.0
            out["dx"].append(G @ W)
            dW += G.T @ X
        del Z, G
    out = {k: torch.cat(v) for k, v in out.items() if v}
    if case["train"]:
        out["dhead"] = dW
        out.pop("lse0", None), out.pop("lse1", None)
        return out
    lses = [out.pop(k) for k in ("lse0", "lse1") if k in out]
    out["lse"] = lses[0] if case["kind"] == "ce" else torch.stack(lses)
    return out
