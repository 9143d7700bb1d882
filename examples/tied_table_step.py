"""Training steps on the embedding table, from encoder embeddings in the pool to the updated table, all on the library's calls:

    pool_gather_padded -> pool_layer_norm -> pool_token_loss_grad -> pool_layer_norm_grad -> pool_embed_grad -> pool_adamw_step

or, with norm="rms" and a limit to the gradients' norm,

    pool_gather_padded -> pool_rms_norm -> pool_token_loss_grad -> pool_rms_norm_grad -> pool_embed_grad -> pool_grad_norm -> pool_adamw_step

and pool_token_logprobs scores a microbatch against the table as it stands.

The table is tied: it is the model's input (assembled rows at text positions) and its output (the vocabulary of the loss),
so its fp32 gradient receives both.  What stands between the two in a model is left out here; a backbone's forward pass goes
between the gather and the norm, its backward pass between the norm's gradient and the table's.  Torch supplies memory only.

    python examples/tied_table_step.py [--workload image_mix_7b] [--samples 16] [--hidden 512] [--steps 8] [--state-bits 8]
                                       [--norm rms] [--max-norm 1.0]
"""
import argparse
import os
import sys

import numpy as np
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import workloads                                      # noqa: E402
from paper_2606_23087_b200 import binding as fp       # noqa: E402


def check(rc, what):
    if rc:
        raise fp.FlowpoolError(rc, what)


class TiedTable:
    """Pool, plan, table (fp32 master and the bf16 copy that the gather and the loss read), last norm and AdamW states."""

    def __init__(self, w, state_bits=32, lr=2e-3, weight_decay=0.1, norm="layer", max_norm=None):
        self.w, self.H, self.V, self.L = w, w.hidden, w.vocab, w.budget_L
        self.rms, self.max_norm = norm == "rms", max_norm
        self.pool = fp.Pool(fp.PoolConfig(
            page_bytes=w.page_bytes, hbm_pages=w.hbm_pages, host_pages=w.host_pages, max_text_tokens=w.total_text_tokens_capacity,
            ring_seed=0, bind_seed=0, gva_hbm_start=0, gva_host_start=0, max_size=0, hidden=w.hidden, max_samples=w.n_samples,
            max_spans_per_sample=w.max_spans_per_sample, max_pages_per_span=w.max_pages_per_span, max_seq_len=w.max_seq_len,
            placeholder_id=w.placeholder_id, ring_order=w.ring_order, bind_order=w.bind_order, world_size=1, rank=0,
            max_imported_pages=0))
        check(self.pool.rc, "pool_create")
        self._fill()
        rc, self.plan = self.pool.plan_microbatches(np.asarray(w.plan_order, np.uint32), fp.PlanConfig(
            coef_A=w.coef_A, coef_B=w.coef_B, budget_L=w.budget_L, n_buckets_K=w.n_buckets_K, n_ranks_N=1, flags=0), self._stream())
        check(rc, "pool_plan_microbatches")
        self.n_mb = self.plan.summary()[0]

        def new(*shape, dtype=torch.float32):
            return torch.zeros(shape, dtype=dtype, device="cuda")
        V, H, L = self.V, self.H, self.L
        self.table = workloads.embed_table(w, device="cuda")
        self.master, self.gain, self.shift = self.table.float(), new(H) + 0.25 * H ** -0.5, new(H)
        self.g_table, self.g_gain, self.g_shift = new(V, H), new(H), new(H)
        self.embeds, self.hidden, self.d_hidden = (new(L, H, dtype=torch.bfloat16) for _ in range(3))
        self.cu = new(w.n_samples + 2, dtype=torch.int32)
        self.pos3 = new(3, L, dtype=torch.int32)
        self.ids, self.labels, self.mask = new(L, dtype=torch.int32), new(L, dtype=torch.int32), new(L, dtype=torch.uint8)
        self.mean, self.rstd, self.loss, self.lse = new(L), new(L), new(L), new(L)
        grad_workspace = self.pool.rms_norm_grad_workspace if self.rms else self.pool.layer_norm_grad_workspace
        self.norm_ws = new(max(1, grad_workspace(L, H)), dtype=torch.uint8)
        self.loss_ws = new(self.pool.token_loss_workspace(L, H, V, True)[1], dtype=torch.uint8)
        # every label that counts has the same weight, whichever microbatch it is in
        n = 0
        for b in range(self.n_mb):
            self._gather(b)
            n += int(self.mask.sum())
        self.n_labels = n
        self.grad_loss = new(1) + 1.0 / n
        self.states, tensors = [], []
        learned = [(self.master, self.g_table, self.table, weight_decay), (self.gain, self.g_gain, None, 0.0)]
        if not self.rms:
            learned.append((self.shift, self.g_shift, None, 0.0))
        for p, g, copy, decay in learned:
            k = p.numel()
            bits = state_bits if p is self.master else 32
            m, v = (new(k, dtype=torch.uint8 if bits == 8 else torch.float32) for _ in range(2))
            sm, sv = (new(-(-k // 256)) if bits == 8 else None for _ in range(2))
            self.states.append((m, v, sm, sv))
            tensors.append(fp.AdamwTensor(param=p.data_ptr(), grad=g.data_ptr(), m=m.data_ptr(), v=v.data_ptr(),
                                          m_scale=sm.data_ptr() if bits == 8 else None, v_scale=sv.data_ptr() if bits == 8 else None,
                                          copy=None if copy is None else copy.data_ptr(), n=k, weight_decay=decay,
                                          param_dtype=fp.FT_F32, grad_dtype=fp.FT_F32, state_bits=bits, reserved=0))
        self.tensors = (fp.AdamwTensor * len(tensors))(*tensors)
        self.adamw = fp.AdamwConfig(lr=lr, beta1=0.9, beta2=0.95, eps=1e-8, grad_scale=None, step=0)
        if max_norm is not None:   # the factor goes from pool_grad_norm to pool_adamw_step on the device
            self.grads = (fp.GradTensor * len(learned))(*[fp.GradTensor(grad=g.data_ptr(), n=g.numel(), dtype=fp.FT_F32)
                                                          for _, g, _, _ in learned])
            self.grad_norm, self.clip = new(1), new(1)
            self.clip_ws = new(self.pool.grad_norm_workspace(), dtype=torch.uint8)
            self.adamw.grad_scale = self.clip.data_ptr()

    def _stream(self):
        return torch.cuda.current_stream().cuda_stream

    def _fill(self):
        """Registers every sample and writes its encoder embeddings, in the workload's calls."""
        w = self.w
        for call in w.write_calls:
            samples = sorted({s for s, _ in call}, key=[s for s, _ in call].index)
            ids = torch.from_numpy(np.concatenate([workloads.input_ids(w, s) for s in samples]).astype(np.int32)).cuda()
            spans = [w.spans_of(s) for s in samples]
            check(self.pool.register_samples(np.asarray(samples, np.uint32), w.seq_len[samples].astype(np.uint32),
                                             w.n_spans[samples].astype(np.uint32), np.concatenate([p for p, _ in spans]).astype(np.uint32),
                                             np.concatenate([t for _, t in spans]).astype(np.uint32), ids.data_ptr(), self._stream()),
                  "pool_register_samples")
            values = [workloads.span_values(w, s, j, device="cuda") for s, j in call]
            check(self.pool.write_embeddings(np.array([s for s, _ in call], np.uint32), np.array([j for _, j in call], np.uint32),
                                             np.array([w.spans_of(s)[1][j] for s, j in call], np.uint32),
                                             [t.data_ptr() for t in values], w.src_dtype, self._stream()), "pool_write_embeddings")
            torch.cuda.synchronize()   # the calls read ids and values in stream order; they are freed here

    def _gather(self, b):
        check(self.pool.gather_padded(self.plan, b, b + 1, self.table.data_ptr(), self.V, 0, self.embeds.data_ptr(), self.cu.data_ptr(),
                                      self.pos3.data_ptr(), self.ids.data_ptr(), self.labels.data_ptr(), self.mask.data_ptr(),
                                      self._stream()), "pool_gather_padded")

    def _norm(self):
        p, s, L, H = self.pool, self._stream(), self.L, self.H
        if self.rms:
            check(p.rms_norm(L, H, self.embeds.data_ptr(), H, 0, 0, fp.FT_BF16, self.gain.data_ptr(), fp.FT_F32, 1e-5, 0, 0,
                             self.hidden.data_ptr(), H, rstd_ptr=self.rstd.data_ptr(), stream=s), "pool_rms_norm")
        else:
            check(p.layer_norm(L, H, self.embeds.data_ptr(), H, fp.FT_BF16, self.gain.data_ptr(), self.shift.data_ptr(), fp.FT_F32, 1e-5,
                               self.hidden.data_ptr(), H, self.mean.data_ptr(), self.rstd.data_ptr(), s), "pool_layer_norm")

    def _norm_grad(self, more):
        p, s, L, H = self.pool, self._stream(), self.L, self.H
        if self.rms:
            check(p.rms_norm_grad(L, H, self.d_hidden.data_ptr(), H, self.embeds.data_ptr(), H, 0, 0, fp.FT_BF16, self.gain.data_ptr(),
                                  fp.FT_F32, self.rstd.data_ptr(), self.d_hidden.data_ptr(), H, self.g_gain.data_ptr(), more,
                                  self.norm_ws.data_ptr(), self.norm_ws.numel(), s), "pool_rms_norm_grad")
        else:
            check(p.layer_norm_grad(L, H, self.d_hidden.data_ptr(), H, self.embeds.data_ptr(), H, fp.FT_BF16, self.gain.data_ptr(),
                                    fp.FT_F32, self.mean.data_ptr(), self.rstd.data_ptr(), self.d_hidden.data_ptr(), H,
                                    self.g_gain.data_ptr(), self.g_shift.data_ptr(), more, self.norm_ws.data_ptr(),
                                    self.norm_ws.numel(), s), "pool_layer_norm_grad")

    def forward_backward(self, b):
        """Microbatch b: its losses into self.loss, its gradients on top of those of the microbatches before it."""
        p, s, L, H, V = self.pool, self._stream(), self.L, self.H, self.V
        more = b > 0
        self._gather(b)
        self._norm()
        check(p.token_loss_grad(L, H, V, self.hidden.data_ptr(), H, self.table.data_ptr(), H, self.labels.data_ptr(),
                                self.grad_loss.data_ptr(), 0, self.loss.data_ptr(), self.lse.data_ptr(), self.d_hidden.data_ptr(), H,
                                self.g_table.data_ptr(), fp.FT_F32, more, self.loss_ws.data_ptr(), self.loss_ws.numel(), s),
              "pool_token_loss_grad")
        self._norm_grad(more)
        check(p.embed_grad(self.plan, b, b + 1, True, self.d_hidden.data_ptr(), self.g_table.data_ptr(), V, s), "pool_embed_grad")

    def step(self):
        """One optimizer step over all microbatches; the mean loss before it (a device tensor)."""
        total = torch.zeros((), device="cuda")
        for b in range(self.n_mb):
            self.forward_backward(b)
            total += self.loss.sum()
        if self.max_norm is not None:
            check(self.pool.grad_norm(self.grads, self.max_norm, 0, 0, self.grad_norm.data_ptr(), self.clip.data_ptr(),
                                      self.clip_ws.data_ptr(), self.clip_ws.numel(), self._stream()), "pool_grad_norm")
        self.adamw.step += 1
        check(self.pool.adamw_step(self.tensors, self.adamw, self._stream()), "pool_adamw_step")
        return total / self.n_labels

    def score(self, b, top=4):
        """Microbatch b against the table: per row the label's log probability (0 where there is no label), the entropy, and the `top`
        likeliest tokens with their log probabilities."""
        L, H, V = self.L, self.H, self.V
        logprob, entropy, top_logprobs = (torch.empty(n, device="cuda") for n in (L, L, (L, top)))
        ids = torch.empty(L, top, dtype=torch.int32, device="cuda")
        ws = torch.empty(self.pool.token_logprobs_workspace(L, H, V, top)[1], dtype=torch.uint8, device="cuda")
        self._gather(b)
        self._norm()
        check(self.pool.token_logprobs(L, H, V, self.hidden.data_ptr(), H, self.table.data_ptr(), H, self.labels.data_ptr(), 1.0,
                                       logprob.data_ptr(), entropy.data_ptr(), top, ids.data_ptr(), top_logprobs.data_ptr(), ws.data_ptr(),
                                       ws.numel(), self._stream()), "pool_token_logprobs")
        return logprob, entropy, ids, top_logprobs

    def close(self):
        torch.cuda.synchronize()
        self.plan.destroy()
        self.pool.destroy()


def train(name="tiny", samples=None, hidden=None, steps=8, state_bits=32, page_bytes=None, norm="layer", max_norm=None):
    """Mean loss of each step."""
    run = TiedTable(workloads.make_workload(name, n_samples=samples, hidden=hidden, page_bytes=page_bytes), state_bits, norm=norm,
                    max_norm=max_norm)
    losses = [run.step() for _ in range(steps)]
    losses = [float(x) for x in losses]
    code, detail = run.pool.status()
    run.close()
    check(code, f"the pool's status word (detail {detail})")
    return losses


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--workload", default="tiny", choices=workloads.CONFIG_NAMES)
    ap.add_argument("--samples", type=int)
    ap.add_argument("--hidden", type=int)
    ap.add_argument("--steps", type=int, default=8)
    ap.add_argument("--state-bits", type=int, default=32, choices=(8, 32))
    ap.add_argument("--norm", default="layer", choices=("layer", "rms"))
    ap.add_argument("--max-norm", type=float)
    a = ap.parse_args()
    for i, x in enumerate(train(a.workload, a.samples, a.hidden, a.steps, a.state_bits, norm=a.norm, max_norm=a.max_norm)):
        print(f"step {i + 1}: mean loss {x:.4f}")
