"""What the layer-forward and scoring functions of the pipeline do on the host, with the library's calls replaced by stand-ins: no GPU."""
import math

import pytest
import torch

from paper_2510_03246_b200 import api, pipeline

D, HEADS = 8, 2


class Calls:
    """Stand-ins that record their status words; the call named `late` reports a wait that ran out."""

    def __init__(self, monkeypatch, late=None):
        self.late, self.seen = late, []
        for name in ("sp_linear", "sp_attention", "sp_token_logprobs", "sp_token_logprobs_grad", "sp_gemm", "sp_gram_accumulate",
                     "sp_symmetrize", "sp_struct_scores", "sp_apply_mask", "sp_linear_refit"):
            monkeypatch.setattr(api, name, getattr(self, name))
        monkeypatch.setattr(api, "new_status", lambda device="cpu": torch.zeros(4, dtype=torch.int32, device=device))

    def note(self, name, status):
        self.seen.append((name, status))
        if name == self.late and status is not None:
            status[0], status[1] = 7, 3

    def sp_linear(self, X, W, bias=None, act=0, other=None, combine=0, out=None, out_dtype=None, status=None):
        self.note("sp_linear", status)
        return torch.zeros(X.shape[0], W.shape[0], dtype=X.dtype) if out is None else out

    def sp_attention(self, Q, K, V, cu_q, cu_k, n_heads, n_kv_heads=None, causal=True, scale=None, out=None, lse=None, want_lse=False,
                     ws=None, status=None):
        self.note("sp_attention", status)
        out = torch.full_like(Q, math.nan) if out is None else out
        out[int(cu_q[0]):int(cu_q[-1])] = 1.0                      # rows of the sequences, and no others
        return out, lse

    def sp_token_logprobs(self, logits, targets=None, n_alts=0, scale=1.0, want_entropy=True, status=None):
        self.note("sp_token_logprobs", status)
        z = torch.zeros(logits.shape[0])
        return api.TokenLogprobs(z, z, None, None, None)

    def sp_token_logprobs_grad(self, logits, targets, lse, g_logp, entropy=None, g_entropy=None, scale=1.0, out=None):
        return out

    def sp_gemm(self, A, B, C_, status=None, **kw):
        self.note("sp_gemm", status)

    def sp_gram_accumulate(self, Xc, Yc, G, R=None, rowstats=None, status=None, ws=None):
        self.note("sp_gram_accumulate", status)

    def sp_symmetrize(self, G):
        pass

    def sp_struct_scores(self, kind, n_units, *a, **kw):
        return torch.zeros(n_units), None, None

    def sp_apply_mask(self, scores, k, **kw):
        return torch.ones(scores.numel(), dtype=torch.uint8), None, None

    def sp_linear_refit(self, R, G, mask, k_keep, rho, status=None, **kw):
        self.note("sp_linear_refit", status)
        return R


def tensors():
    return dict(X=torch.zeros(6, D), Wqkv=torch.zeros(3 * D, D), W_O=torch.zeros(D, D), cu=torch.tensor([0, 4, 6], dtype=torch.int32))


def head_outputs(t, **kw):
    return pipeline.attention_head_outputs(t["X"], t["Wqkv"], t["cu"], HEADS, **kw)


def module(t, **kw):
    return pipeline.prune_attention_module(t["X"], t["Wqkv"], t["W_O"], t["cu"], HEADS, 1, **kw)


def ffn(t, **kw):
    return pipeline.ffn_forward(t["X"], torch.zeros(5, D), torch.zeros(D, 5), **kw)


def gated(t, **kw):
    return pipeline.ffn_forward(t["X"], torch.zeros(5, D), torch.zeros(D, 5), torch.zeros(5, D), **kw)


def loss(t):
    return pipeline.token_loss(t["X"], torch.zeros(9, D), torch.zeros(6, dtype=torch.int64), with_grad=True)


USED = [(head_outputs, ["sp_linear", "sp_attention"]), (module, ["sp_linear", "sp_attention", "sp_gram_accumulate", "sp_linear_refit"]),
        (ffn, ["sp_linear"]), (gated, ["sp_linear"]), (loss, ["sp_linear", "sp_token_logprobs", "sp_gemm"])]


@pytest.mark.parametrize("call,name", [(c, n) for c, names in USED for n in names])
def test_waits_that_ran_out_in_a_call_are_raised(monkeypatch, call, name):
    seen = Calls(monkeypatch, late=name).seen
    with pytest.raises(api.SpError) as e:
        call(tensors())
    assert e.value.code == 7
    assert {n for n, _ in seen} == set(dict((c, names) for c, names in USED)[call])


@pytest.mark.parametrize("call", [c for c, _ in USED])
def test_every_call_has_the_same_status_word(monkeypatch, call):
    seen = Calls(monkeypatch).seen
    call(tensors())
    assert all(s is not None and s is seen[0][1] for _, s in seen)


@pytest.mark.parametrize("call", [head_outputs, module, ffn, gated])
def test_a_status_word_of_the_caller_is_left_to_the_caller(monkeypatch, call):
    """Nothing is raised then, and nothing waits for the device."""
    seen = Calls(monkeypatch, late="sp_linear").seen
    status = torch.zeros(4, dtype=torch.int32)
    call(tensors(), status=status)
    assert int(status[0]) == 7 and all(s is status for _, s in seen)


def test_head_outputs_of_rows_outside_the_sequences_are_zero(monkeypatch):
    Calls(monkeypatch)
    t = tensors()
    t["cu"] = torch.tensor([1, 3, 5], dtype=torch.int32)
    H = head_outputs(t)
    assert H.shape == (6, D) and (H[1:5] == 1).all() and (H[0] == 0).all() and (H[5] == 0).all()


def test_perplexity():
    def of(nll, tokens):
        return pipeline.TokenLoss(nll, tokens, torch.zeros(1), None, None).perplexity
    assert of(6.0, 2) == math.exp(3.0)
    assert math.isnan(of(0.0, 0))                                  # of no tokens there is none
    assert of(2000.0, 1) == math.inf and of(math.inf, 3) == math.inf and math.isnan(of(math.nan, 3))


def test_status_words_of_another_kind_are_refused(monkeypatch):
    Calls(monkeypatch)
    t = tensors()
    H = torch.zeros(6, D)
    for bad in (torch.zeros(4), torch.zeros(3, dtype=torch.int32), torch.zeros(8, dtype=torch.int32)[::2]):
        with pytest.raises(ValueError):
            pipeline.prune_attention_heads(H, H, t["W_O"], HEADS, 1, status=bad)
    pipeline.prune_attention_heads(H, H, t["W_O"], HEADS, 1, status=torch.zeros(4, dtype=torch.int32))
    pipeline.prune_attention_heads(H, H, t["W_O"], HEADS, 1)
