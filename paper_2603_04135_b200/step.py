"""One pruned-GRPO batch step on the device: buffers + the four library calls in order.

This is plumbing around :mod:`.binding`: it allocates device memory with torch, copies the small
per-batch inputs in, issues the library calls on the current CUDA stream and copies results back.
All arithmetic happens inside libdppo.
"""
import torch

from . import binding as B
from . import dp


def quantize_rows_i8(x, status=None):
    """8-bit codes and scales of the rows of x (bf16 or f32 [M, K] with rows on 16 bytes): (q int8 [M, K], scale f32 [M]), q a
    view of padded rows.  Weights are quantised once this way and kept; see DppoStep.score_hidden_i8."""
    M, K = x.shape
    ld = (K + 127) // 128 * 128            # whole 128-byte lines: the product's slabs then never straddle two
    q = torch.zeros(M, ld, dtype=torch.int8, device=x.device)
    scale = torch.zeros(M, dtype=torch.float32, device=x.device)
    B.quantize_rows_i8(B.QuantizeParams(M, K, B.BF16 if x.dtype is torch.bfloat16 else B.F32, x.stride(0) if M > 1 else max(x.stride(0), K), ld),
                       x, q, scale, status=status)
    return q[:, :K], scale


class DppoStep:
    """Buffers for a batch of P prompts x G completions and a loss sweep over at most T_max tokens.

    prune_pack():  rewards -> advantages -> candidate sets, masks, gamma, w_seq, H_next -> packing of the
                   retained completions (unit = prompt + response tokens) into rows of L_row, with
                   cu_seqlens over the response tokens in packed order.
    loss():        fused sweep over logits [T, V] of the retained response tokens in packed order.
    """

    def __init__(self, P, G, L_row, N_win, r_q, r_o, V, dtype, T_max, eps_lo=0.2, eps_hi=0.2, beta=0.04,
                 temperature=1.0, mode=0, reverse=0, policy=0, std_ddof=0, std_eps=1e-6, device="cuda", group=None):
        if not torch.cuda.is_available():
            raise RuntimeError("DppoStep needs a CUDA device: libdppo has no CPU path")
        self.P, self.G, self.n = P, G, P * G
        self.V, self.T_max = V, T_max
        self.dtype = dtype
        self.std_ddof, self.std_eps = std_ddof, std_eps
        dev = torch.device(device)
        self.device = dev
        self.group = group                       # torch.distributed process group of the data-parallel ranks (or None)
        self.H_table = None                      # dataset-wide history scores, owned by run_epochs
        n = self.n
        f32 = dict(dtype=torch.float32, device=dev)
        i32 = dict(dtype=torch.int32, device=dev)
        u8 = dict(dtype=torch.uint8, device=dev)
        self.rewards = torch.zeros(n, **f32)
        self.H_prev = torch.zeros(P, **f32)
        self.has_history = False
        self.unit_len = torch.zeros(n, **i32)
        self.loss_len = torch.zeros(n, **i32)
        self.adv = torch.zeros(n, **f32)
        self.mean_abs_adv = torch.zeros(P, **f32)
        self.cand_q = torch.zeros(P, **u8); self.cand_o = torch.zeros(n, **u8)
        self.keep_q = torch.zeros(P, **u8); self.keep_o = torch.zeros(n, **u8)
        self.n_keep_q = torch.zeros(1, **i32); self.n_keep_o = torch.zeros(P, **i32)
        self.gamma_q = torch.zeros(P, **f32); self.gamma_o = torch.zeros(n, **f32)
        self.w_seq = torch.zeros(n, **f32); self.H_next = torch.zeros(P, **f32)
        self.order = torch.zeros(n, **i32); self.row_of = torch.zeros(n, **i32)
        self.off_in_row = torch.zeros(n, **i32); self.row_fill = torch.zeros(n, **i32)
        self.cu_seqlens = torch.zeros(n + 1, **i32); self.counts = torch.zeros(4, **i32)
        self.status = torch.zeros(1, **i32)
        self.loss_out = torch.zeros(5, **f32)
        self.logp_out = torch.zeros(max(T_max, 1), **f32); self.lse_out = torch.zeros(max(T_max, 1), **f32)

        self.prune_params = B.PruneParams(P, G, r_q, r_o, mode, reverse, 0, 0)
        self.pack_params = B.PackParams(n, L_row, N_win, policy)
        self.loss_params = B.LossParams(T_max, V, B.BF16 if dtype == "bf16" else B.F32, V, n, 0,
                                        eps_lo, eps_hi, beta, temperature)
        self.pack_ws_bytes = B.pack_workspace_bytes(self.pack_params)
        self.pack_ws = torch.zeros(max(self.pack_ws_bytes, 16), dtype=torch.uint8, device=dev)
        self.loss_ws_bytes = B.grpo_loss_workspace_bytes(self.loss_params)
        self.loss_ws = torch.zeros(max(self.loss_ws_bytes, 16), dtype=torch.uint8, device=dev)

    # -- inputs ------------------------------------------------------------------------------------
    def set_batch(self, rewards, unit_len, loss_len, H_prev=None):
        """Copy the per-batch host inputs (numpy / torch) to the device."""
        self.rewards.copy_(torch.as_tensor(rewards, dtype=torch.float32).reshape(-1), non_blocking=True)
        self.unit_len.copy_(torch.as_tensor(unit_len, dtype=torch.int32).reshape(-1), non_blocking=True)
        self.loss_len.copy_(torch.as_tensor(loss_len, dtype=torch.int32).reshape(-1), non_blocking=True)
        self.has_history = H_prev is not None
        if self.has_history:
            self.H_prev.copy_(torch.as_tensor(H_prev, dtype=torch.float32).reshape(-1), non_blocking=True)

    # -- library calls -----------------------------------------------------------------------------
    def advantages(self, rewards=None, adv=None, mean_abs_adv=None):
        B.group_advantages(self.rewards if rewards is None else rewards, self.P, self.G,
                           self.adv if adv is None else adv,
                           self.mean_abs_adv if mean_abs_adv is None else mean_abs_adv,
                           self.std_ddof, self.std_eps, self.status)

    def prune(self, seed, step, u_q=None, u_o=None):
        self.prune_params.seed, self.prune_params.step = seed, step
        B.prune_and_rescale(self.prune_params, self.adv, self.mean_abs_adv,
                            self.H_prev if self.has_history else None, u_q, u_o,
                            self.cand_q, self.cand_o, self.keep_q, self.keep_o, self.n_keep_q, self.n_keep_o,
                            self.gamma_q, self.gamma_o, self.w_seq, self.H_next, self.status)

    def pack(self):
        B.pack_prompts(self.pack_params, self.unit_len, self.keep_o, self.loss_len, self.order, self.row_of,
                       self.off_in_row, self.row_fill, self.cu_seqlens, self.counts, self.pack_ws,
                       self.pack_ws_bytes, self.status)

    def prune_pack(self, seed=0, step=0, u_q=None, u_o=None):
        self.advantages()
        self.prune(seed, step, u_q, u_o)
        self.pack()

    def loss(self, logits, target, logp_old, logp_ref, dlogits=None, row_stride=None):
        """Loss sweep over the retained tokens; the true token count is read on the device from the
        packer's counts.  dlogits may be `logits` itself (in place) or None (forward only)."""
        self.loss_params.row_stride = self.V if row_stride is None else row_stride
        B.grpo_loss_fwd_bwd(self.loss_params, logits, target, logp_old, logp_ref, self.cu_seqlens,
                            self.counts[3:4], self.adv, self.w_seq, self.order, dlogits, self.logp_out,
                            self.lse_out, self.loss_out, self.loss_ws, self.loss_ws_bytes, self.status)

    # -- scoring: where logp_old and logp_ref come from ---------------------------------------------
    def _score_buffers(self, T, top_k, out):
        """Buffers of a scoring call over T rows: new ones, or `out`, what an earlier call with the same top_k returned."""
        if out is not None:
            row, k = (T,), (T, top_k)
            for n, want in (("logp", row), ("entropy", row), ("lse", row), ("stats", (T, 4)), ("top_ids", k), ("top_logp", k)):
                have = out[n].shape if n in out else want
                if have != want and (len(have) != len(want) or have[1:] != want[1:] or have[0] < T):
                    raise ValueError("out: %s has shape %s, this call needs %s" % (n, tuple(have), want))
            return out
        f32 = dict(dtype=torch.float32, device=self.device)
        out = {n: torch.zeros(T, **f32) for n in ("logp", "entropy", "lse")}
        out["stats"] = torch.zeros(T, 4, **f32)
        out["top_ids"] = torch.full((T, top_k), -1, dtype=torch.int32, device=self.device)
        out["top_logp"] = torch.zeros(T, top_k, **f32)
        return out

    def _score_call(self, logits, dtype, V, stride, target, n_tokens_dev, top_k, out, lo, hi):
        prm = B.LogprobParams(hi - lo, V, dtype, stride, top_k, 0, self.loss_params.temperature)
        part = {n: v[lo:hi] for n, v in out.items()} if lo > 0 else out
        B.token_logprobs(prm, logits, target, n_tokens_dev, part["logp"] if target is not None else None, part["entropy"],
                         part["lse"], part["top_ids"] if top_k else None, part["top_logp"] if top_k else None,
                         part["stats"], self.status)

    def score(self, logits, target=None, top_k=0, row_stride=None, n_tokens_dev=None, out=None):
        """Log-probs of the given tokens under the policy that made `logits` [T_max, V] (with the temperature of the
        loss), their entropy and top_k alternatives: a dict of logp, entropy, lse [T_max], top_ids, top_logp
        [T_max, top_k] and stats [T_max, 4] (for score_backward).  logp of a frozen policy is what loss() takes as
        logp_old or logp_ref.  Rows past the token count (the packer's, or n_tokens_dev) are left as they were.  `out`: the
        dict of an earlier call with the same top_k, to be written again (ValueError where its shapes do not fit)."""
        out = self._score_buffers(self.T_max, top_k, out)
        self._score_call(logits, self.loss_params.dtype, self.V, self.V if row_stride is None else row_stride, target,
                         self.counts[3:4] if n_tokens_dev is None else n_tokens_dev, top_k, out, 0, self.T_max)
        return out

    def score_backward(self, logits, target, scored, dlogp=None, dentropy=None, dlogits=None, row_stride=None,
                       n_tokens_dev=None):
        """Gradient with respect to `logits` of a loss with the per-token derivatives dlogp and dentropy (f32 [T_max], either
        may be None); `scored` is what score() returned.  Returns dlogits (`logits` itself for in place; a new tensor of the
        logits' shape and strides if None)."""
        if dlogits is None and logits.is_contiguous():
            dlogits = torch.zeros_like(logits)
        elif dlogits is None:                    # rows that are padded: the same pitch
            extent = 1 + sum((n - 1) * s for n, s in zip(logits.shape, logits.stride())) if logits.numel() else 0
            dlogits = logits.new_zeros(extent).as_strided(logits.shape, logits.stride())
        stride = self.V if row_stride is None else row_stride
        prm = B.LogprobParams(self.T_max, self.V, self.loss_params.dtype, stride, 0, 0, self.loss_params.temperature)
        B.token_logprobs_backward(prm, logits, target, self.counts[3:4] if n_tokens_dev is None else n_tokens_dev,
                                  scored["stats"], dlogp, dentropy, dlogits, self.status)
        return dlogits

    def score_hidden_i8(self, hidden, W_q, W_scale, target=None, top_k=0, n_tokens_dev=None, chunk_tokens=2048, out=None):
        """The same scores from hidden states [T_max, H] (bf16 or f32, rows on 16 bytes) and a frozen policy's LM-head in
        8 bits (quantize_rows_i8 of its [V, H] weight): rows quantised per token, product on the tensor cores, scores.
        The tokens are taken chunk_tokens at a time through an f32 logits scratch of that many rows, allocated for the call;
        the whole [T_max, V] is never formed."""
        T, H = hidden.shape
        if T != self.T_max:
            raise ValueError("hidden has %d rows, T_max is %d" % (T, self.T_max))
        if W_q.shape != (W_scale.numel(), H):
            raise ValueError("W_q has shape %s; %d scales and hidden states %d wide need (%d, %d)"
                             % (tuple(W_q.shape), W_scale.numel(), H, W_scale.numel(), H))
        out = self._score_buffers(T, top_k, out)
        if T == 0:
            return out
        V, C = W_scale.numel(), min(chunk_tokens, T)
        ldq, ldv = (H + 127) // 128 * 128, (V + 3) // 4 * 4
        # of this call alone, so that calls on several streams, or captured ones, do not write each other's; nothing of it is read
        # before it is written
        logits = torch.empty(C, ldv, dtype=torch.float32, device=self.device)
        q = torch.empty(C, ldq, dtype=torch.int8, device=self.device)
        q_scale = torch.empty(C, dtype=torch.float32, device=self.device)
        T_dev = self.counts[3:4] if n_tokens_dev is None else n_tokens_dev
        if T <= C and T_dev.dtype is torch.int32 and T_dev.dim() == 1:
            left = T_dev                         # one chunk: the kernels bound the count by the rows themselves
        else:
            left = torch.clamp(T_dev - torch.arange(0, T, C, dtype=torch.int32, device=self.device), 0, C).to(torch.int32)
        dtype = B.BF16 if hidden.dtype is torch.bfloat16 else B.F32
        for i, lo in enumerate(range(0, T, C)):
            hi, n = min(lo + C, T), left[i:i + 1]
            B.quantize_rows_i8(B.QuantizeParams(hi - lo, H, dtype, hidden.stride(0), ldq), hidden[lo:hi], q, q_scale, n, self.status)
            B.linear_i8(B.LinearI8Params(hi - lo, V, H, ldq, W_q.stride(0), ldv, B.F32), q, q_scale, W_q, W_scale, logits, n,
                        self.status)
            self._score_call(logits, B.F32, V, ldv, None if target is None else target[lo:hi], n, top_k, out, lo, hi)
        return out

    def step_from_host(self, batch_host, token_host, dev_tokens, seed=0, step=0, dlogits=None):
        """The whole path from HOST buffers: copies the batch inputs and the token inputs (logits, targets,
        old / reference log-probs; pinned host tensors) to the device, runs advantages -> prune -> pack ->
        loss sweep, and returns the five loss scalars on the host (this synchronises).

        batch_host: dict with pinned tensors rewards, unit_len, loss_len and optionally H_prev.
        token_host / dev_tokens: dicts with logits, target, logp_old, logp_ref (host source, device
        destination).  A host tensor with fewer rows than its destination is treated as a window that is
        copied repeatedly (same bytes over the bus, for hosts that cannot pin the whole input).  Returns (loss_out as a host tensor, bytes copied host->device, bytes device->host).
        """
        h2d = 0
        for name in ("rewards", "unit_len", "loss_len"):
            getattr(self, name).copy_(batch_host[name], non_blocking=True)
            h2d += batch_host[name].numel() * batch_host[name].element_size()
        self.has_history = batch_host.get("H_prev") is not None
        if self.has_history:
            self.H_prev.copy_(batch_host["H_prev"], non_blocking=True)
            h2d += batch_host["H_prev"].numel() * 4
        for name in ("logits", "target", "logp_old", "logp_ref"):
            src, dst = token_host[name], dev_tokens[name]
            if src.shape[0] >= dst.shape[0]:
                dst.copy_(src[:dst.shape[0]], non_blocking=True)
            else:
                # the pinned host buffer is a window of `src.shape[0]` rows (host memory is short): the
                # same number of bytes crosses the bus, window by window
                for a in range(0, dst.shape[0], src.shape[0]):
                    b = min(dst.shape[0], a + src.shape[0])
                    dst[a:b].copy_(src[:b - a], non_blocking=True)
            h2d += dst.numel() * dst.element_size()
        self.prune_pack(seed, step)
        self.loss(dev_tokens["logits"], dev_tokens["target"], dev_tokens["logp_old"], dev_tokens["logp_ref"], dlogits)
        out = self.loss_out.cpu()                         # device -> host read of the result; synchronises
        return out, h2d, out.numel() * 4

    # -- several ranks ---------------------------------------------------------------------------
    def shard(self, world, rank):
        """This rank's contiguous range of the packed rows of the last prune_pack (reads the packer's
        outputs: synchronises).  See dp.shard_rows."""
        n_units = int(self.counts[0].item())
        order = self.order[:n_units].long()
        return dp.shard_rows(self.row_of[order].cpu().tolist(), self.cu_seqlens.cpu().tolist(), n_units, world, rank)

    def loss_shard(self, shard, logits, target, logp_old, logp_ref, dlogits=None, row_stride=None):
        """Loss sweep over one rank's share of the packed rows: `logits` (and the other per-token inputs) hold the
        tokens [tok_lo, tok_hi) of the batch, in packed order.  The sequence weights are those of the WHOLE batch,
        so the five scalars of all ranks add up to the batch's (all_reduce_loss)."""
        lo, hi = shard["seq_lo"], shard["seq_hi"]
        T_r = shard["tok_hi"] - shard["tok_lo"]
        prm = B.LossParams.from_buffer_copy(self.loss_params)
        prm.T_max, prm.S_max = T_r, max(hi - lo, 1)
        prm.row_stride = self.V if row_stride is None else row_stride
        cu_local = (self.cu_seqlens[lo:hi + 1] - shard["tok_lo"]).contiguous() if hi > lo else self.cu_seqlens[:2] * 0
        seg_map = self.order[lo:max(hi, lo + 1)].contiguous()
        B.grpo_loss_fwd_bwd(prm, logits, target, logp_old, logp_ref, cu_local, None, self.adv, self.w_seq, seg_map,
                            dlogits, self.logp_out, self.lse_out, self.loss_out, self.loss_ws, self.loss_ws_bytes,
                            self.status)

    def all_reduce_loss(self, average=False):
        """Combines loss_out over the ranks of `group` (a no-op for a single process); see dp.all_reduce_loss."""
        return dp.all_reduce_loss(self.loss_out, self.group, average)

    # -- several epochs ----------------------------------------------------------------------------
    def run_epochs(self, n_prompts, batches_by_epoch, rewards_fn, seed, lengths_fn=None, on_batch=None):
        """Algorithm 1's outer loops around the small steps, with the dataset-wide history table of Eq. 16.

        The table H (one score per dataset prompt, zero at the start) lives on the device and is owned by this
        object (self.H_table).  For batch b of epoch t (a list of P dataset prompt ids): gather the prompts'
        scores -> advantages -> candidate sets, masks and weights (no prompt pruning in the first epoch; the
        generator's step word is t * 1,000,000 + b) -> scatter the updated scores back (retained prompts get their
        fresh mean |A|, pruned ones keep the old score) -> pack the retained completions.  Every step is a library
        call on the current stream; nothing is read back unless `on_batch` does.

        rewards_fn(t, ids) -> float32 [P, G] rewards of those prompts in epoch t (host array)
        lengths_fn(t, ids) -> (unit_len, loss_len) int32 [P*G] each, or None to skip the packing step
        on_batch(t, b, self)  called after each batch with the results in this object's buffers
        Returns self.H_table.
        """
        self.H_table = torch.zeros(n_prompts, dtype=torch.float32, device=self.device)
        ids_dev = torch.zeros(self.P, dtype=torch.int32, device=self.device)
        for t, batches in enumerate(batches_by_epoch):
            for b, ids in enumerate(batches):
                if len(ids) != self.P:
                    raise ValueError("a batch must hold P = %d prompt ids, got %d" % (self.P, len(ids)))
                ids_dev.copy_(torch.as_tensor(ids, dtype=torch.int32), non_blocking=False)
                self.rewards.copy_(torch.as_tensor(rewards_fn(t, ids), dtype=torch.float32).reshape(-1))
                if lengths_fn is not None:
                    unit_len, loss_len = lengths_fn(t, ids)
                    self.unit_len.copy_(torch.as_tensor(unit_len, dtype=torch.int32).reshape(-1))
                    self.loss_len.copy_(torch.as_tensor(loss_len, dtype=torch.int32).reshape(-1))
                B.history_gather(self.H_table, n_prompts, ids_dev, self.P, self.H_prev, self.status)
                self.has_history = t > 0
                self.advantages()
                self.prune(seed, t * 1000000 + b)
                B.history_scatter(self.H_table, n_prompts, ids_dev, self.P, self.H_next, self.status)
                if lengths_fn is not None:
                    self.pack()
                if on_batch is not None:
                    on_batch(t, b, self)
        return self.H_table

    # -- results -----------------------------------------------------------------------------------
    def n_tokens(self):
        """Retained loss tokens T of the last prune_pack (synchronises)."""
        return int(self.counts[3].item())

    def prune_results(self):
        names = ["adv", "mean_abs_adv", "cand_q", "cand_o", "keep_q", "keep_o", "n_keep_q", "n_keep_o",
                 "gamma_q", "gamma_o", "w_seq", "H_next"]
        return {k: getattr(self, k).cpu().numpy() for k in names}

    def pack_results(self):
        names = ["order", "row_of", "off_in_row", "row_fill", "cu_seqlens", "counts", "status"]
        return {k: getattr(self, k).cpu().numpy() for k in names}
