"""GPU: drafted tokens against the target's probabilities, against the definition in fractions and
whole numbers (tests/sharing_reference.py). All outputs are whole numbers and have to be equal."""
import numpy as np
import pytest

import sharing_reference as S
from gpu_helpers import say, torch_cuda
from test_gpu_kv8 import ints, make

pytestmark = pytest.mark.gpu


def check(torch, target, drafts, u, draft=None, counts=None, lengths=None, name=""):
    cache = make(torch, 1, 1, 64)
    more = {"draft": draft, "counts": None if counts is None else ints(torch, counts),
            "lengths": None if lengths is None else ints(torch, lengths)}
    got = cache.verify(target, ints(torch, drafts.tolist()).view(drafts.shape),
                       torch.tensor(u, dtype=torch.float32, device="cuda"), **more)
    wide = lambda t: None if t is None else t.double().cpu().numpy()
    want = S.verify(wide(target), drafts, np.asarray(u, np.float32), wide(draft), counts, lengths)
    for what, a, b in zip(("tokens", "accepted", "lengths"), got, want):
        a = a.cpu().numpy()
        assert np.array_equal(a, b), (name, what, a.tolist(), b.tolist())
    return [x.cpu().numpy() for x in got]


def case(torch, seed, n, k, vocab, dtype, near=0.5, sharp=2.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    logits = sharp * torch.randn((n, k + 1, vocab), generator=g, device="cuda")
    other = logits[:, :k] + near * torch.randn((n, k, vocab), generator=g, device="cuda")
    target = torch.softmax(logits, -1).to(dtype)
    draft = torch.softmax(other, -1).to(dtype)
    noise = -torch.log(-torch.log(torch.rand(other.shape, generator=g, device="cuda")
                                  .clamp(1e-20, 1 - 1e-7)))
    drafts = (other + noise).argmax(-1).cpu().numpy().astype(np.int32)
    u = torch.rand((n, k + 1), generator=g, device="cuda").cpu().numpy()
    return target, draft, drafts, u


@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("n,k,vocab", [(1, 4, 32000), (5, 3, 4096), (3, 2, 4097), (4, 1, 4095),
                                       (7, 0, 1000), (2, 7, 1), (6, 5, 3), (2, 70, 300),
                                       (3, 2, 50257), (1, 1, 1 << 20), (1030, 2, 130)])
def test_verify(n, k, vocab, dtype):
    torch = torch_cuda()
    dt = getattr(torch, dtype)
    target, draft, drafts, u = case(torch, n + vocab, n, k, vocab, dt)
    rng = np.random.default_rng(vocab)
    lengths = rng.integers(0, 1000, n).tolist()
    counts = rng.integers(-1, k + 2, n).tolist()
    check(torch, target, drafts, u, draft, None, lengths, "drawn")
    check(torch, target, drafts, u, None, counts, lengths, "sure")
    check(torch, target, drafts, u, draft, counts, None, "counts")


def test_all_or_none_accepted():
    torch = torch_cuda()
    target, draft, drafts, u = case(torch, 1, 6, 5, 2000, torch.float32)
    low, high = u.copy(), u.copy()
    low[:, :5], high[:, :5] = 0.0, 1.0 - 2.0 ** -24
    tokens, accepted = check(torch, target, drafts, low, draft)
    assert (accepted == 5).all() and (tokens[:, :5] == drafts).all()
    check(torch, target, drafts, high, draft)
    # the same distribution: max(p - q, 0) is nothing, and u < 1 accepts everything
    tokens, accepted = check(torch, target, drafts, high, target[:, :5].contiguous())
    assert (accepted == 5).all()


@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("vocab", [1056, 6000, 50257])
def test_sure_drafts_that_hold_most_of_a_row(vocab, dtype):
    """Sure drafts are the likeliest tokens: what they leave out of a row is more than what other parts
    of it weigh, wherever in the row they lie."""
    torch = torch_cuda()
    target, _, _, u = case(torch, vocab, 61, 3, vocab, getattr(torch, dtype), sharp=3.0)
    drafts = target[:, :3].argmax(-1).cpu().numpy().astype(np.int32)
    _, accepted = check(torch, target, drafts, u)
    assert (accepted < 3).any()
    lone = torch.zeros_like(target)                # nearly all at the draft, a little elsewhere
    at = torch.randint(0, vocab, (61, 4, 3), device="cuda",
                       generator=torch.Generator(device="cuda").manual_seed(vocab))
    lone.scatter_(2, at, 2.0 ** -9)
    lone.scatter_(2, torch.from_numpy(drafts).cuda().long()[:, :1].expand(61, 4)[..., None], 0.75)
    u[:, :3] = 0.9
    check(torch, lone, np.repeat(drafts[:, :1], 3, 1), u)


def test_values_that_are_no_probabilities():
    """NaN, infinities, negative values, values above 1, subnormals and zeros, in rows and at the
    drafts; rows without weight draw -1 or p's own."""
    torch = torch_cuda()
    n, k, vocab = 12, 2, 9000
    target, draft, drafts, u = case(torch, 5, n, k, vocab, torch.float32)
    odd = torch.tensor([float("nan"), float("inf"), -float("inf"), -0.5, 7.0, 1e-40, -0.0, 1.0,
                        2.0 ** -43, 3 * 2.0 ** -43, 2.0 ** -42], device="cuda")
    g = torch.Generator(device="cuda").manual_seed(7)
    for x in (target, draft):
        at = torch.randint(0, vocab, (n, x.shape[1], 40), generator=g, device="cuda")
        x.scatter_(2, at, odd[torch.randint(0, len(odd), at.shape, generator=g, device="cuda")])
    for b in range(n):                              # at the drafts themselves
        target[b, 0, drafts[b, 0]] = odd[b % len(odd)]
        draft[b, 0, drafts[b, 0]] = odd[(3 * b + 1) % len(odd)]
    target[3], draft[4] = 0.0, 0.0
    target[5] = float("nan")
    target[6, :, 1:] = 0.0
    draft[7] = target[7, :k]
    draft[8] = 1.0
    for name, d in (("draft", draft), ("sure", None)):
        check(torch, target, drafts, u, d, None, [5] * n, name)


def test_random_numbers_at_their_ends():
    torch = torch_cuda()
    ends = [0.0, 2.0 ** -24, 2.0 ** -30, 1e-45, 0.5, 1 - 2.0 ** -24, 1.0, 2.0, -1.0, float("nan"),
            float("inf"), -0.0]
    n, vocab = len(ends), 5000
    target, draft, drafts, u = case(torch, 9, n, 2, vocab, torch.float32)
    u[:, 2] = ends
    check(torch, target, drafts, u, draft)
    u[:, 0] = ends
    check(torch, target, drafts, u, draft)
    flat = torch.full((n, 1, 4096 * 3 + 1), 1.0, device="cuda")      # sums of many whole ones
    check(torch, flat, np.zeros((n, 0), np.int32), u[:, 2:])


def test_tokens_outside_the_vocabulary():
    torch = torch_cuda()
    n, k, vocab = 6, 3, 500
    target, draft, drafts, u = case(torch, 11, n, k, vocab, torch.float32)
    drafts[0, 0], drafts[1, 1], drafts[2, 2], drafts[3, 0] = -1, vocab, 1 << 30, -(1 << 31)
    u[:, :k] = 0.0
    for d in (draft, None):
        check(torch, target, drafts, u, d, [3, 3, 3, 3, 0, -1], [0, 1, 2, 3, 4, 5])


def test_edges_between_accepted_and_not():
    """u q against p where they are equal, and one step of a product of 48 bits apart."""
    torch = torch_cuda()
    n, vocab = 64, 40
    rng = np.random.default_rng(2)
    q = (rng.integers(1 << 23, 1 << 24, n) * 2.0 ** -24).astype(np.float32)
    u = (rng.integers(1 << 23, 1 << 24, n) * 2.0 ** -24).astype(np.float32)
    p = (q.astype(np.float64) * u).astype(np.float32)      # u q rounded: above it or not
    target = torch.full((n, 2, vocab), 1e-3, device="cuda")
    draft = torch.full((n, 1, vocab), 1e-3, device="cuda")
    target[:, 0, 3], draft[:, 0, 3] = torch.from_numpy(p).cuda(), torch.from_numpy(q).cuda()
    us = np.stack([u, np.full(n, 0.3, np.float32)], 1)
    _, accepted = check(torch, target, np.full((n, 1), 3, np.int32), us, draft)
    assert 0 < accepted.sum() < n
    # equal: not below, not accepted
    target[:, 0, 3], draft[:, 0, 3], us[:, 0] = 0.25, 0.5, 0.5
    _, accepted = check(torch, target, np.full((n, 1), 3, np.int32), us, draft)
    assert not accepted.any()


def test_strides_and_given_outputs():
    torch = torch_cuda()
    n, k, vocab = 4, 3, 5001
    target, draft, drafts, u = case(torch, 13, n, k, vocab, torch.bfloat16)
    wide_t = torch.zeros((k + 1, n, vocab + 9), dtype=target.dtype, device="cuda")
    wide_t[:, :, 3:3 + vocab] = target.transpose(0, 1)
    wide_d = torch.zeros((n, k, vocab + 1), dtype=target.dtype, device="cuda")
    wide_d[:, :, 1:] = draft
    check(torch, wide_t.transpose(0, 1)[:, :, 3:3 + vocab], drafts, u, wide_d[:, :, 1:])
    cache = make(torch, 1, 1, 64)
    lengths = ints(torch, [7, 2, 100, 0])
    want = S.verify(target.double().cpu().numpy(), drafts, u, draft.double().cpu().numpy(), None,
                    lengths.tolist())
    cache.verify(target, ints(torch, drafts.tolist()), torch.from_numpy(u).cuda(), draft=draft,
                 lengths=lengths, new_lengths=lengths)
    assert lengths.tolist() == want[2].tolist()


def test_how_the_tokens_are_distributed():
    """Over many random numbers the first token is distributed as the target's first row: each
    share within five standard deviations."""
    torch = torch_cuda()
    n, vocab = 40000, 6
    p = torch.tensor([0.4, 0.05, 0.25, 0.1, 0.0, 0.2], device="cuda")
    q = torch.tensor([0.1, 0.3, 0.2, 0.1, 0.2, 0.1], device="cuda")
    g = torch.Generator(device="cuda").manual_seed(3)
    drafts = torch.multinomial(q.expand(n, -1), 1, generator=g).to(torch.int32)
    u = torch.rand((n, 2), generator=g, device="cuda")
    cache = make(torch, 1, 1, 64)
    tokens, _ = cache.verify(p.expand(n, 2, vocab), drafts, u, draft=q.expand(n, 1, vocab))
    share = torch.bincount(tokens[:, 0].long(), minlength=vocab).double().cpu() / n
    want = p.double().cpu()
    assert bool(((share - want).abs() <= 5 * (want * (1 - want) / n).sqrt() + 1e-12).all()), share
