"""Call-by-name front end over the C-ABI binding, with the argument names of the paper's
``compute_*`` functions (Section 6.1): picks the entry point from dtype and layout, keeps one carry
workspace per (device, stream, shape) so that repeated calls allocate nothing, and accepts
``torch.bool`` masks.  Workspace sharing rule: calls that use the same cached workspace are those
issued on the same stream, which orders them; calls on different streams get different workspaces.
A caller that passes ``workspace=`` itself must keep the calls sharing it ordered on the GPU.  Argument marshalling only -- every step runs in the CUDA kernels, there is no CPU path.

    adv, ret = compute_gae(rewards, values, dones, truncateds, bootstrap_values, bootstrap,
                           gamma=0.99, lam=0.95)

float32 tensors go to the fp32 entry points, bfloat16 tensors to the ``*_bf16`` ones (row-major
only); ``time_major=True`` takes ``[T, N]`` tensors (float32 only).  ``bootstrap_values`` is the
paper's 2-D tensor of continuation values at truncated steps, ``bootstrap`` its 1-D window-edge
vector (Section 4.2).
"""
from __future__ import annotations

from . import binding as _B

_workspaces: dict = {}


def _torch():
    import torch
    return torch


def _mask(m):
    """bool masks are reinterpreted as uint8 (same storage), uint8 passes through."""
    if m is None:
        return None
    torch = _torch()
    return m.view(torch.uint8) if m.dtype == torch.bool else m


def _workspace(like, N: int, T: int, nbytes: int | None = None, stream=None):
    """One initialised workspace per (device, stream, N, T, size), reused by every later call on that
    shape and stream.  The stream is part of the key because two calls share carry records and a
    call counter in the workspace: only calls ordered on one stream may share one."""
    if not like.is_cuda:
        raise TypeError("rlcs takes CUDA tensors (device pointers); there is no CPU path")
    s = _torch().cuda.current_stream(like.device) if stream is None else stream
    key = (like.device, int(s.cuda_stream), N, T, nbytes)
    ws = _workspaces.get(key)
    if ws is None:
        ws = _B.Workspace(N, T, device=like.device, stream=s, nbytes=nbytes)
        _workspaces[key] = ws
    return ws


def _kind(t, time_major: bool) -> str:
    torch = _torch()
    if t.dtype == torch.float32:
        return "tm" if time_major else "f32"
    if t.dtype == torch.bfloat16:
        if time_major:
            raise ValueError("time_major=True takes float32 tensors (the bfloat16 entry points are row-major)")
        return "bf16"
    raise TypeError(f"expected float32 or bfloat16 tensors, got {t.dtype}")


def _shape(t, time_major: bool):
    if t.dim() != 2:
        raise ValueError("expected 2-D [num_envs, seq_len] tensors ([seq_len, num_envs] with time_major=True)")
    return (t.shape[1], t.shape[0]) if time_major else (t.shape[0], t.shape[1])


def _ws_for(kind: str, like, N: int, T: int, workspace, stream=None):
    if workspace is not None:
        return workspace
    if kind == "tm":
        nbytes = int(_B.lib().rlcs_time_major_workspace_bytes(N, T))
        return _workspace(like, N, T, max(nbytes, 256), stream=stream) if nbytes else None
    return _workspace(like, N, T, stream=stream)


def compute_gae(rewards, values, dones, truncateds=None, bootstrap_values=None, bootstrap=None, *, gamma=0.99,
                lam=0.95, time_major=False, normalize=False, eps=1e-8, skip_mask=None, workspace=None, stream=None):
    """GAE advantages and returns (Section 3.3.1).  ``normalize``: advantages standardised over the
    whole batch (returns from the raw advantages).  ``skip_mask``: observation-skip masking (masked
    steps are transparent); returns (advantages, returns, filled values) then."""
    kind = _kind(rewards, time_major)
    N, T = _shape(rewards, time_major)
    dones, truncateds, skip_mask = _mask(dones), _mask(truncateds), _mask(skip_mask)
    if normalize or skip_mask is not None:
        if kind != "f32" or (normalize and skip_mask is not None):
            raise ValueError("normalize / skip_mask take row-major float32 tensors, one of the two at a time")
    if normalize:
        ws = workspace if workspace is not None else _workspace(
            rewards, N, T, int(_B.lib().rlcs_gae_normalized_workspace_bytes(N, T)), stream=stream)
        return _B.rlcs_gae_normalized(rewards, values, dones, truncateds, bootstrap_values, bootstrap, gamma=gamma, lam=lam,
                                      eps=eps, workspace=ws, stream=stream)
    ws = _ws_for(kind, rewards, N, T, workspace, stream)
    if skip_mask is not None:
        return _B.rlcs_gae_skip(rewards, values, dones, truncateds, bootstrap_values, bootstrap, skip=skip_mask, gamma=gamma,
                                lam=lam, workspace=ws, stream=stream)
    fn = {"f32": _B.rlcs_gae, "bf16": _B.rlcs_gae_bf16, "tm": _B.rlcs_gae_time_major}[kind]
    return fn(rewards, values, dones, truncateds, bootstrap_values, bootstrap, gamma=gamma, lam=lam, workspace=ws, stream=stream)


def compute_vtrace(rewards, values, log_rhos, dones, truncateds=None, bootstrap_values=None, bootstrap=None, *, gamma=0.99,
                   rho_bar=1.0, c_bar=1.0, time_major=False, workspace=None, stream=None):
    """V-Trace targets and policy-gradient advantages (Section 3.3.2); ``log_rhos = log pi - log mu``."""
    kind = _kind(rewards, time_major)
    N, T = _shape(rewards, time_major)
    fn = {"f32": _B.rlcs_vtrace, "bf16": _B.rlcs_vtrace_bf16, "tm": _B.rlcs_vtrace_time_major}[kind]
    return fn(rewards, values, log_rhos, _mask(dones), _mask(truncateds), bootstrap_values, bootstrap, gamma=gamma,
              rho_bar=rho_bar, c_bar=c_bar, workspace=_ws_for(kind, rewards, N, T, workspace, stream), stream=stream)


def compute_retrace(rewards, q_sa, expected_q, log_rhos, dones, truncateds=None, bootstrap_values=None, bootstrap=None, *,
                    gamma=0.99, lam=0.95, c_bar=1.0, time_major=False, workspace=None, stream=None):
    """Retrace(lambda) targets from per-step scalars (Section 3.3.3): Q(s_t,a_t), E_pi Q(s_t,.), log pi/mu."""
    kind = _kind(rewards, time_major)
    N, T = _shape(rewards, time_major)
    fn = {"f32": _B.rlcs_retrace, "bf16": _B.rlcs_retrace_bf16, "tm": _B.rlcs_retrace_time_major}[kind]
    return fn(rewards, q_sa, expected_q, log_rhos, _mask(dones), _mask(truncateds), bootstrap_values, bootstrap, gamma=gamma,
              lam=lam, c_bar=c_bar, workspace=_ws_for(kind, rewards, N, T, workspace, stream), stream=stream)


def compute_retrace_from_probs(rewards, q_values, target_probs, behaviour_probs, actions, dones, truncateds=None,
                               bootstrap_values=None, bootstrap=None, *, gamma=0.99, lam=0.95, c_bar=1.0, workspace=None,
                               stream=None):
    """Retrace(lambda) from the [N, T, A] Q-values and action probabilities (Section 7.3's input form)."""
    N, T = rewards.shape
    return _B.rlcs_retrace_probs(rewards, q_values, target_probs, behaviour_probs, actions, _mask(dones), _mask(truncateds),
                                 bootstrap_values, bootstrap, gamma=gamma, lam=lam, c_bar=c_bar,
                                 workspace=workspace if workspace is not None else _workspace(rewards, N, T, stream=stream),
                                 stream=stream)


def compute_td_lambda_returns(rewards, values, dones, truncateds=None, bootstrap_values=None, bootstrap=None, *, gamma=0.99,
                              lam=0.95, time_major=False, workspace=None, stream=None):
    """TD(lambda) returns (Section 3.3.4)."""
    kind = _kind(rewards, time_major)
    N, T = _shape(rewards, time_major)
    fn = {"f32": _B.rlcs_td_lambda, "bf16": _B.rlcs_td_lambda_bf16, "tm": _B.rlcs_td_lambda_time_major}[kind]
    return fn(rewards, values, _mask(dones), _mask(truncateds), bootstrap_values, bootstrap, gamma=gamma, lam=lam,
              workspace=_ws_for(kind, rewards, N, T, workspace, stream), stream=stream)


def compute_discounted_returns(rewards, dones, truncateds=None, bootstrap_values=None, bootstrap=None, *, gamma=0.99,
                               time_major=False, workspace=None, stream=None):
    """Discounted returns (Section 3.3.4, lambda = 1 without a value function)."""
    kind = _kind(rewards, time_major)
    N, T = _shape(rewards, time_major)
    fn = {"f32": _B.rlcs_discounted_return, "bf16": _B.rlcs_discounted_return_bf16,
          "tm": _B.rlcs_discounted_return_time_major}[kind]
    return fn(rewards, _mask(dones), _mask(truncateds), bootstrap_values, bootstrap, gamma=gamma,
              workspace=_ws_for(kind, rewards, N, T, workspace, stream), stream=stream)


def compute_eligibility_traces(x, dones, *, gamma=0.99, lam=0.95, beta=None, time_major=False, workspace=None, stream=None):
    """Eligibility traces (Section 3.3.5).  x [N, T]: scalar traces; x [N, T, D]: vector traces with the
    shared decay gamma*lam, or with a decay per component and step when ``beta`` [N, T, D] is given."""
    if x.dim() == 3:
        if time_major:
            raise ValueError("vector traces take [N, T, D] tensors")
        N, T, D = x.shape
        query = _B.lib().rlcs_elig_trace_vec_workspace_bytes if beta is None else _B.lib().rlcs_elig_trace_vec_beta_workspace_bytes
        nbytes = int(query(N, T, D))
        if workspace is None and nbytes:                       # few long rows: chunk records, cached like the others
            workspace = _workspace(x, N, T, nbytes, stream=stream)
        if beta is not None:
            return _B.rlcs_elig_trace_vec_beta(x, beta, _mask(dones), workspace=workspace, stream=stream)
        return _B.rlcs_elig_trace_vec(x, _mask(dones), gamma=gamma, lam=lam, workspace=workspace, stream=stream)
    if beta is not None:
        raise ValueError("beta goes with [N, T, D] vector traces")
    kind = _kind(x, time_major)
    N, T = _shape(x, time_major)
    fn = {"f32": _B.rlcs_elig_trace, "bf16": _B.rlcs_elig_trace_bf16, "tm": _B.rlcs_elig_trace_time_major}[kind]
    return fn(x, _mask(dones), gamma=gamma, lam=lam, workspace=_ws_for(kind, x, N, T, workspace, stream), stream=stream)


def compute_episodic_prefix_sum(x, dones, *, boundary="ends_at", time_major=False, workspace=None, stream=None):
    """Episodic prefix sums (Section 3.3.6); boundary = "ends_at" (dones marks last steps) or "starts_at"."""
    if boundary not in ("ends_at", "starts_at"):
        raise ValueError('boundary must be "ends_at" or "starts_at"')
    kind = _kind(x, time_major)
    N, T = _shape(x, time_major)
    fn = {"f32": _B.rlcs_episodic_prefix_sum, "bf16": _B.rlcs_episodic_prefix_sum_bf16,
          "tm": _B.rlcs_episodic_prefix_sum_time_major}[kind]
    return fn(x, _mask(dones), starts_at=(boundary == "starts_at"), workspace=_ws_for(kind, x, N, T, workspace, stream), stream=stream)


# ------------------------------------------------------------------ rollout and policy operators
def _flat_rows(logits):
    """[..., A] logits as [rows, A] (a view) and the leading shape, None where it is [rows, A] already."""
    if logits.dim() == 2:
        return logits, None
    return logits.view(-1, logits.shape[-1]), logits.shape[:-1]


def _by_dtype(logits, f32, bf16):
    return {"f32": f32, "bf16": bf16}[_kind(logits, False)]


def sample_actions(logits, uniforms, *, temperature=None, top_k=None, top_p=None, min_p=None, stream=None):
    """Actions drawn from logits [..., A] (float32 or bfloat16) with one given uniform in [0, 1) a row, and their log-probabilities:
    (actions int32, log_probs, kept_log_probs).  kept_log_probs is the log-probability with which the action was drawn, under what
    top_k, min_p and top_p leave: the behaviour policy that importance ratios (V-trace, Retrace) divide by.  log_probs is under
    the whole softmax at that temperature, as compute_log_probs and compute_policy_gradient score actions: a clipped loss that compares
    the learner's policy with the acting one wants it, so that its ratios start at 1.  Without a cut both say the same.  Parameters
    are numbers or tensors of one value a row; temperature 0 takes the most likely action; a row that allows none (all -inf) gets action -1."""
    fn = _by_dtype(logits, _B.rlcs_sample_actions, _B.rlcs_sample_actions_bf16)
    rows, lead = _flat_rows(logits)
    flat = lambda v: v.reshape(-1) if lead is not None and hasattr(v, "reshape") else v
    got = fn(rows, flat(uniforms), temperature=flat(temperature), top_k=flat(top_k), top_p=flat(top_p), min_p=flat(min_p), stream=stream)
    return got if lead is None else tuple(v.view(lead) for v in got)


def compute_policy_gradient(logits, actions, advantages, *, old_log_probs=None, mask=None, temperature=1.0, clip=0.2,
                            entropy_coef=0.0, scale=1.0, in_place=False, stream=None):
    """Policy loss of the given actions and its gradient in the logits [..., A]: (loss, log_probs, entropy, dlogits).  Without
    old_log_probs the policy-gradient loss -scale (adv lp + entropy_coef H), with them the clipped-ratio one.  loss is per row:
    its sum is what dlogits differentiates, so scale = 1 / rows gives the mean.  Rows with mask 0 or an action outside [0, A)
    count as absent.  in_place=True overwrites the logits with the gradient."""
    rows, lead = _flat_rows(logits)
    flat = lambda v: v.reshape(-1) if lead is not None and v is not None else v
    fn = _by_dtype(logits, _B.rlcs_policy_grad, _B.rlcs_policy_grad_bf16)
    loss, lp, ent, grad = fn(rows, flat(actions), flat(advantages), old_log_probs=flat(old_log_probs), mask=flat(_mask(mask)),
                             temperature=temperature, clip=clip, entropy_coef=entropy_coef, scale=scale,
                             dlogits=rows if in_place else None, stream=stream)
    if lead is None:
        return loss, lp, ent, grad
    return loss.view(lead), lp.view(lead), ent.view(lead), grad.view(logits.shape)


def compute_log_probs(logits, actions, *, mask=None, temperature=1.0, stream=None):
    """Log-probability of the given actions and entropy of each row of logits [..., A]: (log_probs, entropy)."""
    rows, lead = _flat_rows(logits)
    flat = lambda v: v.reshape(-1) if lead is not None and v is not None else v
    fn = _by_dtype(logits, _B.rlcs_policy_grad, _B.rlcs_policy_grad_bf16)
    got = fn(rows, flat(actions), mask=flat(_mask(mask)), temperature=temperature, stream=stream)
    return got if lead is None else tuple(v.view(lead) for v in got)


def shared_prefix_attention(q, k_cache, v_cache, prefix_table, prefix_lens, group_offsets, block_table, lens, *, scale=None,
                            max_prefix_len=None, max_len=None, workspace=None, stream=None):
    """Attention of one query a trajectory, q [B, H, d] bfloat16, over the paged prompt that its group shares and its own pages:
    (out [B, H, d], lse [B, H]).  Caches [pages, page, Hk, d]; group g holds rows group_offsets[g] to group_offsets[g+1]-1.
    scale defaults to d ** -0.5; max_prefix_len and max_len bound the lengths (by default what the tables can hold): closer
    bounds give better launches and a smaller workspace (it grows with rows, heads and both bounds).  workspace: a uint8 tensor of
    at least rlcs_prefix_attention_workspace_bytes bytes, whose calls the caller keeps ordered on the GPU; by default every call
    takes one of its own from torch's allocator, so that calls of several threads, streams and captured graphs share none."""
    scale = q.shape[-1] ** -0.5 if scale is None else scale
    return _B.rlcs_prefix_attention_bf16(q, k_cache, v_cache, prefix_table, prefix_lens, group_offsets, block_table, lens, scale=scale,
                                         max_prefix_len=max_prefix_len, max_len=max_len, workspace=workspace, stream=stream)


def build_block_tables(cached, added, free_pages, block_table, *, page_size, num_slots, stream=None):
    """Page table, slot map and positions of one step of a paged cache, from lengths on the GPU: (slots, positions, offsets,
    pages_used); block_table is extended in place with pages taken from free_pages in row order.  pages_used (one element) above
    free_pages.numel() says that the list ran out: the rows without a page have -1 in the table and in slots."""
    slots, positions, offsets, page_offsets = _B.rlcs_block_tables(cached, added, free_pages, block_table, page_size=page_size,
                                                                   num_slots=num_slots, stream=stream)
    return slots, positions, offsets, page_offsets[-1:]


# ------------------------------------------------------------------ speculative rollouts and distillation
def chunk_attention(q, k_cache, v_cache, block_table, offsets, lens, *, scale=None, max_new=None, max_len=None, workspace=None, stream=None):
    """Attention of chunks of new tokens over a paged cache that holds them already: whole prompts, parts of prompts, drafts, single
    tokens, mixed as they come.  q [T, H, d] bfloat16; tokens offsets[b] to offsets[b+1]-1 (int32 [B + 1], as build_block_tables gives
    them) are the last of trajectory b's lens[b] tokens, and each sees the keys up to its own: (out [T, H, d], lse [T, H]).  Caches
    [pages, page, Hk, d]; scale defaults to d ** -0.5; max_new and max_len bound the chunks and the lengths (by default T, and what the table can hold):
    closer bounds give better launches and a smaller workspace.  Tokens outside every trajectory (a padded step) are not written.
    workspace: as for shared_prefix_attention, of rlcs_chunk_attention_workspace_bytes bytes; by default one of the call's own."""
    scale = q.shape[-1] ** -0.5 if scale is None else scale
    return _B.rlcs_chunk_attention_bf16(q, k_cache, v_cache, block_table, offsets, lens, scale=scale, max_new=max_new, max_len=max_len,
                                        workspace=workspace, stream=stream)


def verify_drafts(logits, tokens, offsets, uniforms, draw_uniforms, *, draft_logits=None, temperature=None, stream=None):
    """Which drafted tokens stay, and the token that follows them: (out_tokens int32 [T], log_probs [T], accepted int32 [B]).  tokens [T]
    holds, trajectory after trajectory (offsets [B + 1]), the last token and the drafts; logits [T, A] (float32 or bfloat16) the target's
    prediction after each, draft_logits [T, A] the one each following draft was drawn from at the same temperature (None: drafts were
    given, not drawn).  One uniform in [0, 1) a row decides on its draft, one a trajectory draws the token that follows.  out_tokens[t] is
    the token after tokens[t]: kept drafts, the drawn token, then -1; log_probs are the target's, so they serve as old_log_probs
    of a policy loss.  temperature is a number or a tensor of one a trajectory; 0 keeps and takes the most likely token.  Rows
    outside every trajectory are not written.  Verification knows no top_k, top_p or min_p: where drafts were drawn with them (sample_actions), or
    the target is to be, give both rows with -inf for what the filter leaves out, or the tokens follow neither distribution."""
    fn = _by_dtype(logits, _B.rlcs_verify_drafts, _B.rlcs_verify_drafts_bf16)
    return fn(logits, tokens, offsets, uniforms, draw_uniforms, draft_logits=draft_logits, temperature=temperature, stream=stream)


def compute_distillation(logits, teacher_ids, teacher_logits, *, mask=None, temperature=1.0, scale=1.0, in_place=False, stream=None):
    """Loss of a student's logits [..., A] towards the strongest logits of a teacher, [..., K] with their indices teacher_ids (int32; -1 for
    entries that are not there), and its gradient: (loss [...], dlogits [..., A]).  The loss is the divergence from the teacher's
    probabilities over its K entries to the student's over all A, both at `temperature`, times scale (temperature ** 2 / rows gives
    the usual mean).  loss is per row: its sum is what dlogits differentiates.  Rows with mask 0 count as absent.  in_place=True
    overwrites the logits with the gradient."""
    rows, lead = _flat_rows(logits)
    flat = lambda v: v.reshape(-1) if lead is not None and v is not None else v
    pairs = lambda v: v if lead is None else v.reshape(-1, v.shape[-1])
    fn = _by_dtype(logits, _B.rlcs_distill_grad, _B.rlcs_distill_grad_bf16)
    loss, grad = fn(rows, pairs(teacher_ids), pairs(teacher_logits), mask=flat(_mask(mask)), temperature=temperature, scale=scale,
                    dlogits=rows if in_place else None, stream=stream)
    return (loss, grad) if lead is None else (loss.view(lead), grad.view(logits.shape))


def fork_block_tables(block_table, lens, sources, free_pages, *, page_size, stream=None):
    """Trajectories continued from others (branches, resampling): row i of the new table continues row sources[i].  Whole pages are
    shared; a part-filled last page is copied for every row but the first that ends in it (for all where another new row has that page
    whole), to pages taken from free_pages: (new_table, copy_from, copy_to, pages_used).  copy_pages makes the copies, layer by layer;
    pages_used (one element) above the number of free pages says that the list ran out.  Branches share pages: after lengths were lowered into
    pages that other rows name, fork with sources 0 to B-1 before the rows grow, or they write over one another's keys."""
    return _B.rlcs_fork_block_tables(block_table, lens, sources, free_pages, page_size=page_size, stream=stream)


def copy_pages(k_cache, v_cache, copy_from, copy_to, *, stream=None):
    """Copies pages copy_from[i] -> copy_to[i] of both caches [pages, page, Hk, d] in place; pairs with a negative number are passed over."""
    return _B.rlcs_copy_pages_bf16(k_cache, v_cache, copy_from, copy_to, stream=stream)


def list_free_pages(block_table, lens, *, num_pages, page_size, prefix_table=None, prefix_lens=None, stream=None):
    """The pages that no trajectory (and no shared prompt) names any more, ascending: (free_pages int32 [num_pages], -1 behind the last,
    count [1]).  Freeing a trajectory is setting its length to 0, turning tokens down is lowering it (into a page that another row shares: see
    fork_block_tables); the list serves build_block_tables and fork_block_tables as it is, without a word from the host."""
    return _B.rlcs_free_pages(block_table, lens, prefix_table, prefix_lens, num_pages=num_pages, page_size=page_size, stream=stream)
