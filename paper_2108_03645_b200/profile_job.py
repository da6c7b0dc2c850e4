"""Profiles a language-model training job on this GPU and enters it into the search.

The search plans with a profiled step time per job, ``t = a + c * (B / g) + d * log2 g`` (Eq. 5 and the text after it:
the throughput X is measured on the job while it runs).  Here is a job that can be run and resized: `LanguageModelJob`
is the last block and the output head of a language model on synthetic token sequences,

    x = embedding[token];  h = layer_norm(x + gelu(x W1) W2);  loss = cross entropy of h against the head,

whose step uses the operators of `train` (layer norm, the cross entropy that never keeps the logits, the orthogonalised
update for the block's matrices; the plain matrix products are the library's). With `heads` in its shape the block has causal
attention within each sample before that, x = x + attention(rotated norms of q and k, v) Wo, and with `clip` the gradients are
scaled down to that norm before the update.  `profile` times the step at every
batch b0 << k that fits, `fit` turns the times into a and c (one GPU cannot measure d, which is passed in), `job_row` makes
the row of the job table, and the command

    python -m paper_2108_03645_b200.profile_job --b0 8 --kmax 4

prints the measured times, the fitted row and the schedule that the search finds for it beside other jobs.
"""
from __future__ import annotations

import argparse
import json
import math
from dataclasses import dataclass

import numpy as np

from .inputs import JOB_DTYPE


@dataclass(frozen=True)
class JobShape:
    width: int = 1024
    inner: int = 4096
    vocab: int = 32000
    seq: int = 256          # tokens per sample
    ignored: float = 0.1    # share of tokens without a target
    heads: int = 0          # query heads of the attention (0: a block without one)
    kv_heads: int = 0       # key and value heads, a divisor of heads (0: as many)
    clip: float = 0.0       # largest norm of all gradients together, finite (0: as they are)

    def __post_init__(self):
        kv = self.kv_heads or self.heads
        if self.heads < 0 or kv < 0 or (self.heads and (self.width % self.heads or self.heads % kv or self.width // self.heads > 128 or
                                                        self.heads // kv > 128 or self.heads > 1024)):
            raise ValueError("JobShape: at most 1024 heads have to divide the width into parts of at most 128, and kv_heads the heads into groups of at most 128")
        if not 0.0 <= self.clip < math.inf:
            raise ValueError("JobShape: clip is a finite norm, or 0")


def fit(batches, seconds) -> tuple[float, float]:
    """a, c >= 0 of t = a + c * B that fit best (least squares)."""
    b = np.asarray(batches, dtype=np.float64)
    t = np.asarray(seconds, dtype=np.float64)
    if b.shape != t.shape or b.ndim != 1 or b.size < 1 or not (np.isfinite(t).all() and (t > 0).all() and (b > 0).all()):
        raise ValueError("fit: one positive time for each batch is needed")
    if np.unique(b).size < 2:
        return 0.0, float(np.mean(t / b))
    db, dt = b - b.mean(), t - t.mean()
    c = float((db * dt).sum() / (db * db).sum())
    a = float(t.mean() - c * b.mean())
    if c < 0.0:                                     # the time does not grow with the batch
        return float(t.mean()), 0.0
    if a < 0.0:                                     # through the origin
        return 0.0, float((b * t).sum() / (b * b).sum())
    return a, c


def job_row(b0: int, kmax: int, max_per_gpu: int, a: float, c: float, d: float) -> np.ndarray:
    """One row of the job table: batches b0 << 0 .. b0 << kmax."""
    row = np.zeros(1, dtype=JOB_DTYPE)
    row[0] = (b0, max_per_gpu, 0, kmax, a, c, d, 1.0)
    return row


class LanguageModelJob:
    """The job's parameters (bfloat16, layer norm in float32), its momentum and one training step."""

    def __init__(self, shape: JobShape, *, seed: int = 0, device="cuda"):
        import torch
        self.shape, self.device = shape, torch.device(device)
        g = torch.Generator(device=self.device).manual_seed(seed)

        def normal(*size, std):
            return (torch.randn(*size, generator=g, device=self.device) * std).bfloat16()

        d, i, v = shape.width, shape.inner, shape.vocab
        self.embedding = normal(v, d, std=1.0)
        self.w1 = normal(d, i, std=1 / math.sqrt(d))
        self.w2 = normal(i, d, std=1 / math.sqrt(i))
        self.head = normal(v, d, std=0.02)
        self.gain = torch.ones(d, device=self.device)
        self.shift = torch.zeros(d, device=self.device)
        self.matrices = [self.w1, self.w2]
        if shape.heads:
            from . import train
            self.kv_heads = shape.kv_heads or shape.heads
            self.head_dim = d // shape.heads
            self.wqkv = normal(d, (shape.heads + 2 * self.kv_heads) * self.head_dim, std=1 / math.sqrt(d))
            self.wo = normal(d, d, std=1 / math.sqrt(d))
            self.q_gain, self.k_gain = (torch.ones(self.head_dim, device=self.device) for _ in range(2))
            self.frequencies = train.rotary_frequencies(self.head_dim // 2 * 2, device=self.device)
            self.matrices += [self.wqkv, self.wo]
        self.momentum = [torch.zeros_like(w, dtype=torch.float32) for w in self.matrices]

    def batch(self, samples: int, seed: int):
        """Synthetic sequences: the next token follows from the present one, some have no target."""
        import torch
        g = torch.Generator(device=self.device).manual_seed(seed)
        n, v = samples * self.shape.seq, self.shape.vocab
        token = torch.randint(0, v, (n,), generator=g, device=self.device)
        target = (token * 31 + 7) % v
        target[torch.rand(n, generator=g, device=self.device) < self.shape.ignored] = -100
        return token, target

    def attend(self, x):
        """The attention of each sample: (its sum with x, what the gradients need)."""
        import torch
        from . import train
        n, (h, kv, d) = x.shape[0], (self.shape.heads, self.kv_heads, self.head_dim)
        q, k, v = (x @ self.wqkv).view(n, h + 2 * kv, d).split([h, kv, kv], 1)
        position = torch.arange(n, device=x.device) % self.shape.seq
        offsets = torch.arange(0, n + 1, self.shape.seq, device=x.device)
        qn, kn = train.qk_norm(q, k, position, self.frequencies, self.q_gain, self.k_gain)
        out, lse = train.attention(qn, kn, v, offsets)
        return x + out.view(n, -1) @ self.wo, (x, q, k, v, position, offsets, qn, kn, out, lse)

    def attend_backward(self, dy, kept):
        """Gradients of wqkv, wo, q_gain and k_gain (embeddings are not trained)."""
        import torch
        from . import train
        x, q, k, v, position, offsets, qn, kn, out, lse = kept
        flat = out.view(x.shape[0], -1)
        dout = (dy @ self.wo.t()).view_as(out)
        dqn, dkn, dv = train.attention_backward(dout, qn, kn, v, out, lse, offsets)
        dq, dk, dqg, dkg = train.qk_norm_backward(dqn, dkn, q, k, position, self.frequencies, self.q_gain, self.k_gain)
        return x.t() @ torch.cat([dq, dk, dv], 1).view(x.shape[0], -1), flat.t() @ dy, dqg, dkg

    def gradients(self, token, target):
        """(mean loss, gradients of w1, w2, head, gain, shift, and with attention of wqkv, wo, q_gain, k_gain); the loss is a 0-d
        tensor, nothing synchronises."""
        import torch
        from . import train
        x = self.embedding[token]
        kept = None
        if self.shape.heads:
            x, kept = self.attend(x)
        u = x @ self.w1
        act = torch.nn.functional.gelu(u)
        z = x + act @ self.w2
        h, mean, rstd = train.layer_norm(z, self.gain, self.shift)
        loss, lse = train.linear_cross_entropy(h, self.head, target)
        live = ((target >= 0) & (target < self.shape.vocab)).sum().clamp(min=1)
        dloss = (1.0 / live).expand(loss.shape).contiguous()
        dh, dhead = train.linear_cross_entropy_backward(dloss, h, self.head, target, lse)
        dz, dgain, dshift = train.layer_norm_backward(dh, z, mean, rstd, self.gain)
        dw2 = act.t() @ dz
        du = torch.ops.aten.gelu_backward(dz @ self.w2.t(), u)
        dw1 = x.t() @ du
        grads = (dw1, dw2, dhead, dgain, dshift)
        if kept:
            grads += self.attend_backward(dz + du @ self.w1.t(), kept)
        return loss.sum() / live, grads

    def step(self, token, target, *, lr: float = 0.02, head_lr: float = 20.0, beta: float = 0.9):
        """One training step; returns the mean loss (0-d tensor)."""
        from . import train
        loss, grads = self.gradients(token, target)
        if self.shape.clip:
            train.clip_gradients(grads, self.shape.clip)
        dw1, dw2, dhead, dgain, dshift, *attention = grads
        for w, m, dw in zip(self.matrices, self.momentum, (dw1, dw2, *attention[:2])):
            m.mul_(beta).add_(dw)
            w.sub_(train.orthogonalize(m), alpha=lr * math.sqrt(max(1.0, w.shape[0] / w.shape[1])))
        self.head.sub_(dhead, alpha=head_lr)
        self.gain.sub_(dgain, alpha=lr)
        self.shift.sub_(dshift, alpha=lr)
        if attention:
            self.q_gain.sub_(attention[2], alpha=lr)
            self.k_gain.sub_(attention[3], alpha=lr)
        return loss


def profile(job: LanguageModelJob, batches, *, steps: int = 10, warmup: int = 3) -> list[float]:
    """Seconds per step at each batch (samples on the job's GPU), by CUDA events around `steps` steps."""
    import torch
    with torch.cuda.device(job.device):  # events and checks belong to the current device
        return _profile(job, batches, steps, warmup)


def _profile(job, batches, steps, warmup):
    import torch
    from . import train
    out = []
    for b in batches:
        data = [job.batch(b, s) for s in range(2)]
        for s in range(warmup):
            job.step(*data[s % 2])
        begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        begin.record()
        for s in range(steps):
            job.step(*data[s % 2])
        end.record()
        end.synchronize()
        train.check()
        out.append(begin.elapsed_time(end) * 1e-3 / steps)
    return out


def main(argv=None) -> dict:
    ap = argparse.ArgumentParser(description="Profile a language-model job at every batch and schedule it beside others.")
    ap.add_argument("--b0", type=int, default=8, help="smallest batch, in samples")
    ap.add_argument("--kmax", type=int, default=4, help="largest exponent: batches b0 << 0 .. b0 << kmax")
    ap.add_argument("--max-per-gpu", type=int, default=0, help="samples that one GPU takes (default: the largest batch)")
    ap.add_argument("--d", type=float, default=0.01, help="seconds per doubling of the GPUs (not measured on one GPU)")
    ap.add_argument("--width", type=int, default=JobShape.width)
    ap.add_argument("--vocab", type=int, default=JobShape.vocab)
    ap.add_argument("--seq", type=int, default=JobShape.seq)
    ap.add_argument("--heads", type=int, default=0, help="query heads of the block's attention (default: a block without one)")
    ap.add_argument("--kv-heads", type=int, default=0, help="key and value heads (default: as many)")
    ap.add_argument("--clip", type=float, default=0.0, help="largest norm of all gradients together (default: as they are)")
    ap.add_argument("--generations", type=int, default=50)
    a = ap.parse_args(argv)
    from . import binding, inputs

    most = a.max_per_gpu or a.b0 << a.kmax
    batches = [a.b0 << k for k in range(a.kmax + 1) if a.b0 << k <= most]
    job = LanguageModelJob(JobShape(width=a.width, inner=4 * a.width, vocab=a.vocab, seq=a.seq, heads=a.heads, kv_heads=a.kv_heads,
                                    clip=a.clip))
    seconds = profile(job, batches)
    fa, fc = fit(batches, seconds)
    w = inputs.paper_scale()
    jobs = np.concatenate([w.jobs, job_row(a.b0, a.kmax, most, fa, fc, a.d)])
    search = binding.Search(jobs, w.capacity, w.pop, w.params)
    search.randomize(w.seed)
    search.evolve(a.generations, w.seed)
    best = search.best(True)
    k = int(best["genome"][-1])
    out = {"batches": batches, "seconds": seconds, "a": fa, "c": fc, "scheduled_batch": (a.b0 << k) if k >= 0 else 0,
           "gpus": int(best["gpus_per_job"][-1]), "samples_per_second": float(best["rate_per_job"][-1]),
           "cluster_gpus": int(best["total_gpus"])}
    print(json.dumps(out))
    return out


if __name__ == "__main__":
    main()
