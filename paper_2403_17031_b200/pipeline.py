"""The whole per-token path as one object: preallocated outputs + the chain of C-ABI calls in
the order a PPO iteration runs them. Pure call sequencing; every step runs in the CUDA library."""
from __future__ import annotations

from typing import Dict, Optional

import torch

from . import binding as _b


class PPOHotPath:
    """Buffers and call chain for a batch of B responses x T tokens over a vocabulary of V.

    step(...) runs: EOS trick -> log-prob/entropy of policy and reference -> KL rewards -> GAE ->
    advantage whitening -> clipped losses + gradients, all on the current CUDA stream, and
    returns the dict of output tensors (owned by this object, overwritten by the next step).
    Padding rows (after a response's first EOS) are masked out of every later step, so their logits
    are not read: log-prob and entropy are 0 there.
    """

    def __init__(self, B: int, T: int, V: int, logits_dtype: torch.dtype, params: _b.PPOParams,
                 device="cuda", want_dlogits: bool = True):
        self.B, self.T, self.V = B, T, V
        self.params = params
        self.device = torch.device(device)
        f32, i32, u8 = torch.float32, torch.int32, torch.uint8
        dev = self.device
        bt = lambda dt: torch.empty((B, T), dtype=dt, device=dev)
        self.workspace = _b.new_workspace(_b.workspace_bytes(B, T, V), dev)
        self.out: Dict[str, Optional[torch.Tensor]] = {
            "responses_out": bt(i32), "eos_index": torch.empty(B, dtype=i32, device=dev),
            "seq_len": torch.empty(B, dtype=i32, device=dev), "mask": bt(u8),
            "scores_out": torch.empty(B, dtype=f32, device=dev),
            "logprob": bt(f32), "entropy": bt(f32), "ref_logprob": bt(f32),
            "kl": bt(f32), "rewards": bt(f32), "advantages": bt(f32), "returns": bt(f32),
            "advantages_whitened": bt(f32), "whiten_stats": torch.empty(3, dtype=f32, device=dev),
            "losses": torch.empty(8, dtype=f32, device=dev),
            "dlogits": torch.empty((B, T, V), dtype=logits_dtype, device=dev) if want_dlogits else None,
            "dvalues": bt(f32), "new_logprob": bt(f32), "new_entropy": bt(f32), "dlogprob": bt(f32),
        }
        self._loss_out = {"losses": self.out["losses"], "dlogits": self.out["dlogits"],
                          "dvalues": self.out["dvalues"], "new_logprob": self.out["new_logprob"],
                          "entropy": self.out["new_entropy"], "dlogprob": self.out["dlogprob"]}

    def rollout_stats(self, policy_logits, ref_logits, responses, scores, values):
        """Steps 1-5, one C call per step: everything between sampling and the first PPO epoch."""
        o, p = self.out, self.params
        _b.truncate_and_score(responses, scores, p.eos_id, p.pad_id, p.no_eos_score,
                              out=(o["responses_out"], o["eos_index"], o["seq_len"], o["mask"], o["scores_out"]))
        m = o["mask"]
        _b.logprob_entropy(policy_logits, responses, p.temperature, mask=m, workspace=self.workspace,
                           out=(o["logprob"], o["entropy"], None))
        _b.logprob_entropy(ref_logits, responses, p.temperature, mask=m, workspace=self.workspace,
                           out=(o["ref_logprob"], None, None))
        _b.kl_rewards(o["logprob"], o["ref_logprob"], o["mask"], o["seq_len"], o["scores_out"], p.kl_coef,
                      out=(o["kl"], o["rewards"]))
        if p.whiten_rewards:   # optional reward whitening: mean kept, in place, before GAE
            _b.whiten(o["rewards"], o["mask"], False, p.whiten_eps, workspace=self.workspace, out=o["rewards"])
        _b.gae(o["rewards"], values, o["seq_len"], p.gamma, p.lam, out=(o["advantages"], o["returns"]))
        _b.whiten(o["advantages"], o["mask"], True, p.whiten_eps, workspace=self.workspace,
                  out=o["advantages_whitened"], stats=o["whiten_stats"])
        return o

    def loss(self, logits, responses, old_logprob, values_new, values_old, next_epoch: bool = False):
        """Step 6 on the loss-time logits, using the advantages/returns of rollout_stats or step.
        next_epoch: a later PPO epoch on the same batch (the call before this one on this object was loss() or
        step()): the row order left in the workspace is reused, one launch less."""
        o = self.out
        _b.loss_fwd_bwd(logits, responses, o["mask"], old_logprob, o["advantages_whitened"], values_new,
                        values_old, o["returns"], self.params, self.workspace, out=self._loss_out,
                        next_epoch=next_epoch)
        return o

    def step(self, policy_logits, ref_logits, responses, scores, values, values_new, old_logprob=None,
             loss_logits=None):
        """One pass of the whole path in one C call (ppo_step). old_logprob defaults to the rollout
        log-probs just computed (first PPO epoch: ratio = 1); loss_logits defaults to policy_logits."""
        io = self.step_io({"policy_logits": policy_logits, "ref_logits": ref_logits, "loss_logits": loss_logits,
                           "responses": responses, "scores": scores, "values": values, "values_new": values_new,
                           "old_logprob": old_logprob})
        _b.step(io, policy_logits.dtype, self.B, self.T, self.V, self.params)
        return self.out

    def capture_step(self, policy_logits, ref_logits, responses, scores, values, values_new, old_logprob=None,
                     loss_logits=None):
        """Record one step() on these (fixed) buffers into a CUDA graph; graph.replay() then runs the
        whole path with a single launch call. The caller must have run step() once before (the first
        call sets kernel attributes) and keeps the input tensors alive and in place."""
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            self.step(policy_logits, ref_logits, responses, scores, values, values_new, old_logprob=old_logprob,
                      loss_logits=loss_logits)
        return graph

    def step_io(self, inputs: dict, cuda: bool = True) -> "_b.PPOStepIO":
        """ppo_step_io for this object's output buffers plus the given input tensors."""
        o = self.out
        t = dict(inputs)
        t.update({k: o[k] for k in ("responses_out", "eos_index", "seq_len", "mask", "scores_out", "logprob", "entropy",
                                    "ref_logprob", "kl", "rewards", "advantages", "returns", "advantages_whitened",
                                    "whiten_stats", "losses", "dlogits", "dvalues", "new_logprob", "new_entropy",
                                    "dlogprob")})
        t["workspace"] = self.workspace
        return _b.PPOStepIO.from_tensors(t, cuda)

    def curves(self):
        """The three statistics the paper plots per PPO update, from the outputs of the last rollout_stats() / step():
        [mean RLHF reward, mean summed per-token KL, mean score] as a [3] f32 tensor (one small launch)."""
        o = self.out
        return _b.rollout_curves(o["kl"], o["mask"], o["scores_out"], self.params.kl_coef)

    def device_status(self) -> int:
        return _b.last_device_status(self.workspace)


class DPOStep:
    """One DPO step on materialised logits (section "Preliminaries", "RL-free approaches"), all on the
    current CUDA stream: token log-probs of the policy and of the frozen SFT reference on the response
    rows (prompt and padding rows are skipped, never read), the DPO loss with its implicit rewards, and
    the gradient back to the policy's logits. Leading axis of every tensor: 0 = chosen, 1 = rejected.
    Temperature is 1 (the loss is defined on the model's own distribution)."""

    def __init__(self, P: int, T: int, V: int, dtype: torch.dtype, beta: float, device="cuda"):
        dev = torch.device(device)
        self.P, self.T, self.V, self.beta = P, T, V, float(beta)
        f32 = torch.float32
        self.workspace = _b.new_workspace(_b.workspace_bytes(2 * P * T, 1, V), dev)
        self.out = {
            "logprob": torch.empty((2, P, T), dtype=f32, device=dev),
            "ref_logprob": torch.empty((2, P, T), dtype=f32, device=dev),
            "out4": torch.empty(4, dtype=f32, device=dev),
            "reward_c": torch.empty(P, dtype=f32, device=dev), "reward_r": torch.empty(P, dtype=f32, device=dev),
            "dlogprob": torch.empty((2, P, T), dtype=f32, device=dev),
            "dlogits": torch.empty((2, P, T, V), dtype=dtype, device=dev),
        }

    def step(self, policy_logits, ref_logits, tokens, mask):
        o = self.out
        _b.logprob_entropy_pair(policy_logits, ref_logits, tokens, 1.0, mask=mask, workspace=self.workspace,
                                out=(o["logprob"], None, o["ref_logprob"]))
        _b.dpo_loss(o["logprob"][0], o["logprob"][1], o["ref_logprob"][0], o["ref_logprob"][1], mask[0], mask[1],
                    self.beta, out={"out4": o["out4"], "reward_c": o["reward_c"], "reward_r": o["reward_r"],
                                    "dlp_c": o["dlogprob"][0], "dlp_r": o["dlogprob"][1]})
        _b.logprob_bwd(policy_logits, tokens, mask, o["dlogprob"], 1.0, self.workspace, dlogits=o["dlogits"])
        return o

    def device_status(self) -> int:
        return _b.last_device_status(self.workspace)


class Fp8LMHead:
    """A frozen LM head held in 8 bits: e4m3 values with one scale per 128 x 128 of the weight (half the memory of bf16,
    and the products run at the 8-bit rate). score() gives what step 1 needs of a model - log-probs of given tokens,
    entropy, log-sum-exp - and the k most likely alternatives; grad_hidden() takes gradients on those back to the hidden
    states. Hidden states and logit gradients are quantised per row and 128 columns on the way; logits are bf16.

    W [K, V] (bf16 or fp32) is quantised once, [V, K] for the logits and, with backward=True, [K, V] for the gradient.
    Masked rows are multiplied like the others (their results are left out): for scores of a large batch that is half padding the
    fused bf16 head, which leaves them out of its product, is the faster one.
    Buffers for M rows are kept and overwritten by the next call; everything runs on the current CUDA stream, and the
    calls can be captured into a CUDA graph.
    """

    def __init__(self, W: torch.Tensor, M: int, k: int, temperature: float, n: int = 1, backward: bool = False):
        K, V = W.shape
        self.M, self.K, self.V, self.k, self.n, self.temperature = M, K, V, k, n, float(temperature)
        self.backward = backward
        dev, f32, f8 = W.device, torch.float32, torch.float8_e4m3fn
        pitch = lambda cols: -(-cols // 16) * 16
        operand = lambda cols: (torch.empty((M, pitch(cols)), dtype=f8, device=dev)[:, :cols],
                                torch.empty((-(-cols // 128), M), dtype=f32, device=dev))
        scratch = lambda N, C: torch.empty(max(_b.fp8_scratch_bytes(M, N, C, dev), 256), dtype=torch.uint8, device=dev)
        self.workspace = _b.new_workspace(_b.workspace_bytes(M, 1, V), dev)
        self.weight = _b.fp8_quantize(W, 128, transpose=True)
        self.hidden = operand(K)
        # (rows of 16-byte multiples, whatever V is)
        self.logits = torch.empty((M, pitch(V)), dtype=torch.bfloat16, device=dev)[:, :V]
        self._scratch = scratch(V, K)
        self.out = {"logprob": torch.empty((M, n), dtype=f32, device=dev), "entropy": torch.empty(M, dtype=f32, device=dev),
                    "lse": torch.empty(M, dtype=f32, device=dev),
                    "top_ids": torch.empty((M, k), dtype=torch.int32, device=dev) if k else None,
                    "top_logprob": torch.empty((M, k), dtype=f32, device=dev) if k else None}
        if backward:
            self.weight_bwd = _b.fp8_quantize(W, 128)
            self.dlogits = torch.empty((M, pitch(V)), dtype=torch.bfloat16, device=dev)[:, :V]
            self.dlogits_q = operand(V)
            self.dhidden = torch.empty((M, K), dtype=torch.bfloat16, device=dev)
            self.mask = torch.ones(M, dtype=torch.uint8, device=dev)          # of the last score()
            self._mask_bwd = torch.empty_like(self.mask)
            self._scratch_bwd = scratch(K, V)

    def score(self, H, tokens, mask=None):
        """H [M, K], tokens [M] or [M, n] int32, mask [M] u8 (rows with 0 are scored as 0, ids -1). Returns the dict of
        logprob [M, n], entropy, lse [M], top_ids, top_logprob [M, k]. With backward=True the mask is kept (copied) for
        grad_hidden()."""
        _b.fp8_quantize(H, 1, out=self.hidden)
        _b.fp8_matmul(*self.hidden, *self.weight, workspace=self.workspace, out=self.logits, scratch=self._scratch)
        _b.logprob_topk(self.logits, tokens, self.k, self.temperature, mask=mask, workspace=self.workspace, out=self.out)
        if self.backward:
            if mask is None:
                self.mask.fill_(1)
            else:
                torch.ne(mask.view(self.M), 0, out=self.mask)
        return self.out

    def grad_hidden(self, tokens, dlogprob, dtop_logprob=None, dentropy=None, dlse=None, top_ids=None, mask=None):
        """Gradients on what the last score() returned -> gradient on its hidden states [M, K] bf16, zeros in the rows that it masked
        and in those with 0 in `mask`. top_ids: another model's alternatives (default: the ones score() found, where dtop_logprob
        is given)."""
        if not self.backward:
            raise ValueError("grad_hidden needs Fp8LMHead(..., backward=True)")
        o = self.out
        if mask is None:
            mask = self.mask
        else:
            _b.check_mask(mask, self.M, self.mask.device)
            mask = torch.logical_and(mask.view(self.M), self.mask, out=self._mask_bwd)
        ids = top_ids if top_ids is not None or dtop_logprob is None else o["top_ids"]
        _b.logprob_topk_bwd(self.logits, o["lse"], self.temperature, tokens=tokens, dlogprob=dlogprob, top_ids=ids,
                            dtop_logprob=dtop_logprob, entropy=o["entropy"], dentropy=dentropy, dlse=dlse, mask=mask,
                            workspace=self.workspace, dlogits=self.dlogits)
        _b.fp8_quantize(self.dlogits, 1, out=self.dlogits_q)
        return _b.fp8_matmul(*self.dlogits_q, *self.weight_bwd, workspace=self.workspace, out=self.dhidden,
                             scratch=self._scratch_bwd)

    def device_status(self) -> int:
        return _b.last_device_status(self.workspace)


class SFTStep:
    """The vocabulary-sized parts of one supervised fine-tuning step (the paper's first stage, before the reward model and PPO):
    the model's input out of the embedding table, cross entropy at the LM head with its gradients, the gradient of the table,
    and the clipping of all gradients by their common norm. The model between embed() and loss() is the caller's, and so are
    the weights and the optimiser. Everything runs on the current CUDA stream and can be captured into a CUDA graph; results
    are this object's buffers, overwritten by the next step.

    W [K, V] is the LM head's weight, stored by rows or by columns (the transpose of a linear layer's weight): its gradient is
    stored the same way. N: positions of a batch. grad_dtype: of the table's gradient.

    A batch in several parts (micro-batches): loss(denom=) divides each part's sum by the number of all parts' real positions,
    grad_embed(accumulate=True) adds to the table's gradient from the second part on. dW is a part's own: the caller adds the parts' up,
    in fp32 say, and gives the sum to clip(dW=). clip() refuses a dW of the last part beside a table's gradient of several."""

    def __init__(self, W: torch.Tensor, N: int, padding_id: int = -1, ignore_id: int = -100, temperature: float = 1.0,
                 embed_scale: float = 1.0, grad_dtype: torch.dtype = torch.bfloat16, piece_rows: int = 0):
        K, V = W.shape
        self.N, self.K, self.V = N, K, V
        self.padding_id, self.ignore_id, self.temperature = padding_id, ignore_id, float(temperature)
        self.embed_scale, self.piece_rows = float(embed_scale), piece_rows
        dev, f32, bf16, u8 = W.device, torch.float32, torch.bfloat16, torch.uint8
        self.workspace = _b.new_workspace(_b.workspace_bytes(N, 1, V), dev)
        scratch = lambda n: torch.empty(max(n, 256), dtype=u8, device=dev)          # noqa: E731
        # (one buffer: the two calls that need it do not overlap)
        self._scratch = scratch(max(_b.lmhead_xent_scratch_bytes(N, K, V, piece_rows), _b.embed_bwd_scratch_bytes(N, K, V)))
        self._clip_scratch = {}
        # loss() calls so far; how many there were when dE was begun (None: not since the last clip()), and whether others were added to it
        self._losses, self._begun, self._mixed = 0, None, False
        self.out = {"hidden": torch.empty((N, K), dtype=bf16, device=dev), "loss": torch.empty((), dtype=f32, device=dev),
                    "nll": torch.empty(N, dtype=f32, device=dev), "lse": torch.empty(N, dtype=f32, device=dev),
                    "dH": torch.empty((N, K), dtype=bf16, device=dev), "dW": torch.empty_like(W),
                    "dE": torch.empty((V, K), dtype=grad_dtype, device=dev), "norm": torch.empty(2, dtype=f32, device=dev)}

    def embed(self, table, tokens):
        """Rows of the table [V, K] for tokens [N] int32, times embed_scale, in bf16."""
        return _b.embed(table, tokens, scale=self.embed_scale, workspace=self.workspace, out=self.out["hidden"])

    def loss(self, H, W, labels, mask=None, scale: float = 1.0, denom: Optional[torch.Tensor] = None):
        """Mean cross entropy of labels [N] under the head's logits for the hidden states H [N, K], without masked rows and
        ignored labels; dH and dW are the gradients of scale * loss. denom: [1] f32, divides the sum instead of the number of
        real rows. Returns the dict of buffers."""
        o = self.out
        _b.lmhead_xent(H, W, labels, mask=mask, ignore_id=self.ignore_id, temperature=self.temperature, scale=scale, denom=denom,
                       piece_rows=self.piece_rows, workspace=self.workspace, scratch=self._scratch,
                       out={n: o[n] for n in ("loss", "nll", "lse", "dH", "dW")})
        self._losses += 1
        return o

    def grad_embed(self, dX, tokens, accumulate: bool = False):
        """Gradient dX [N, K] on embed()'s result -> gradient of the table (accumulate: added to the one there is)."""
        if not accumulate or self._begun is None:
            self._begun, self._mixed = self._losses, False
        self._mixed |= self._losses != self._begun
        return _b.embed_bwd(dX, tokens, self.V, scale=self.embed_scale, padding_id=self.padding_id, accumulate=accumulate,
                            workspace=self.workspace, scratch=self._scratch, out=self.out["dE"])

    def clip(self, max_norm: float, others=(), scale: float = 1.0, dW: Optional[torch.Tensor] = None):
        """Clips dW (the last loss()'s, or the caller's sum over several), dE and the model's other gradients together, in place.
        Returns [norm before clipping, factor]."""
        o = self.out
        if dW is None:
            if self._mixed:
                raise ValueError("the table's gradient is of several loss() calls and dW of the last one: give clip() the sum of theirs")
            dW = o["dW"]
        dW = dW if dW.is_contiguous() else dW.t()                                   # (the same elements, in memory's order)
        grads = [dW, o["dE"], *others]
        need = _b.grad_clip_scratch_bytes(len(grads))
        # (one for each size, all kept: a captured graph may hold the address of any)
        if need not in self._clip_scratch:
            self._clip_scratch[need] = torch.empty(need, dtype=torch.uint8, device=o["norm"].device)
        norm = _b.grad_clip(grads, max_norm, scale=scale, workspace=self.workspace, scratch=self._clip_scratch[need], norm=o["norm"])
        self._begun, self._mixed = None, False
        return norm

    def device_status(self) -> int:
        return _b.last_device_status(self.workspace)
