"""The training loop's operators in a model's place (CPU: the operators themselves are stood in for)."""
import copy
import gc
import weakref

import torch


def _model():
    from transformers import GPT2Config, GPT2LMHeadModel
    return GPT2LMHeadModel(GPT2Config(n_layer=2, n_embd=64, n_head=4, vocab_size=100, n_positions=32, bos_token_id=0,
                                      eos_token_id=0))


def test_a_model_on_the_operators_is_freed_with_its_last_name():
    """Without waiting for a collection: the next optimizer's run begins with the memory that it has."""
    from paper_2608_05088_amd.train import use_operators
    gc.collect()
    gc.disable()
    try:
        model = _model()
        use_operators(model)
        left = [weakref.ref(p) for p in model.parameters()]
        del model
        assert [p for p in left if p() is not None] == []
    finally:
        gc.enable()


def test_a_copy_of_a_model_on_the_operators_has_weights_of_its_own(monkeypatch):
    from paper_2608_05088_amd import ops
    from paper_2608_05088_amd.train import use_operators
    seen = []
    monkeypatch.setattr(ops, "embedding", lambda ids, w: seen.append(w) or w[ids])
    monkeypatch.setattr(ops, "fp8_linear", lambda x, w, transposed: seen.append(w) or x @ w)
    model = _model().eval()
    ids = torch.arange(6)[None]
    want = model(input_ids=ids).logits
    use_operators(model)
    other = copy.deepcopy(model)
    for m in (model, other):
        seen.clear()
        assert torch.allclose(m(input_ids=ids).logits, want, atol=1e-5)
        assert len(seen) == 1 + 2 * 4 and all(any(w is p for p in m.parameters()) for w in seen)
    assert [n for n, _ in model.named_parameters()] == [n for n, _ in _model().named_parameters()]


def test_a_micro_batch_without_next_tokens(monkeypatch):
    """Sequences of one token: no loss and no gradient, as a mean over nothing, not a division by zero."""
    from types import SimpleNamespace

    from paper_2608_05088_amd import ops
    from paper_2608_05088_amd.train import distill_backward
    z = torch.randn(3, 1, 40, requires_grad=True)

    def step(logits, top, top_ids, labels, tau, alpha, grad, out):
        assert bool((top_ids == -1).all()) and bool((labels == -100).all())   # rows of neither: zeros
        return torch.zeros(3, 1), torch.zeros_like(logits)

    monkeypatch.setattr(ops, "distill_step", step)
    loss = distill_backward(lambda input_ids: SimpleNamespace(logits=z * 1.0),
                            lambda input_ids: SimpleNamespace(logits=torch.randn(3, 1, 40)),
                            torch.zeros(3, 1, dtype=torch.int64), top_k=5)
    assert float(loss) == 0.0 and bool((z.grad == 0).all())
