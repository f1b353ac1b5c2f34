"""The operators together, as the training loop runs them: a small GPT-2 student
on a teacher's top logits, stepped by MALT."""
import copy

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2608_05088_amd import libmalt as lm
    lm.lib()


def _tiny(seed, width=128):
    from transformers import GPT2Config, GPT2LMHeadModel
    cfg = GPT2Config(n_layer=2, n_embd=width, n_head=4, vocab_size=1000, n_positions=64, bos_token_id=0, eos_token_id=0,
                     resid_pdrop=0.0, embd_pdrop=0.0, attn_pdrop=0.0)
    torch.manual_seed(seed)
    return GPT2LMHeadModel(cfg).cuda().train()


def _plain_loss(student, teacher, ids, k, tau, alpha):
    """The same loss from torch's own operations."""
    z = student(input_ids=ids).logits[:, :-1].double()
    with torch.no_grad():
        a, i = teacher(input_ids=ids).logits[:, :-1].topk(k, dim=-1)
    p = torch.softmax(a.double() / tau, -1)
    lq = torch.log_softmax(z / tau, -1).gather(-1, i)
    kl = (p * (p.log() - lq)).sum(-1)
    ce = torch.nn.functional.cross_entropy(z.flatten(0, 1), ids[:, 1:].flatten(), reduction="none").view_as(kl)
    return ((1 - alpha) * tau ** 2 * kl + alpha * ce).mean()


def test_distilled_gradients_match_torch():
    """Without 8-bit layers the step's loss and every parameter's gradient are torch's to float32."""
    from paper_2608_05088_amd.train import distill_backward
    student, teacher = _tiny(0), _tiny(1)
    plain = copy.deepcopy(student)
    ids = torch.randint(0, 1000, (3, 40), device="cuda", generator=torch.Generator(device="cuda").manual_seed(2))
    loss = distill_backward(student, teacher, ids, top_k=16, tau=2.0, alpha=0.3, scale=0.5)
    want = _plain_loss(plain, teacher, ids, 16, 2.0, 0.3)
    (want * 0.5).backward()
    assert abs(float(loss) - float(want)) <= 1e-5 * abs(float(want))
    for (n, p), q in zip(student.named_parameters(), plain.parameters()):
        assert float((p.grad - q.grad).norm()) <= 1e-4 * float(q.grad.norm()) + 1e-9, n


def test_operators_train_a_student():
    """Table, 8-bit layers, loss and MALT together: gradients near float32's (8-bit products of 3 mantissa bits are
    some percent off), and the loss on a fixed batch falls."""
    from paper_2608_05088_amd.optim import MALT
    from paper_2608_05088_amd.train import block_matrix, distill_backward, use_operators
    student, teacher = _tiny(3), _tiny(4)
    plain = copy.deepcopy(student)
    use_operators(student)
    ids = torch.randint(0, 1000, (4, 64), device="cuda", generator=torch.Generator(device="cuda").manual_seed(5))
    distill_backward(student, teacher, ids)
    distill_backward(plain, teacher, ids)
    for (n, p), q in zip(student.named_parameters(), plain.parameters()):
        if block_matrix(n, p) or n.endswith("wte.weight"):
            cos = torch.nn.functional.cosine_similarity(p.grad.flatten(), q.grad.flatten(), dim=0)
            assert float(cos) > 0.95, (n, float(cos))
    mats = {id(p) for n, p in student.named_parameters() if block_matrix(n, p)}
    opt = MALT(student.parameters(), lr=2e-3, variant="malt", adamw_lr=1e-3, matrix_filter=lambda p: id(p) in mats)
    losses = []
    for _ in range(12):
        opt.zero_grad()
        losses.append(float(distill_backward(student, teacher, ids)))
        opt.step()
    assert losses[-1] < 0.9 * losses[0], losses
