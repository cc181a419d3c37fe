"""Views of one buffer as the tensors of a step: side by side they are ordinary tensors, overlapping ones are refused before anything changes."""
import pytest
import torch

from paper_2309_11071_amd import head

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


def views(flat, starts, n=300):
    return [flat[s:s + n] for s in starts]


@pytest.mark.parametrize("bits", [8, 32])
def test_overlapping_views_are_refused(bits):
    flat, grads = torch.zeros(1000, device="cuda"), [torch.ones(300, device="cuda") for _ in range(2)]
    mom = head.adamw_moments(grads, bits)
    apart = [torch.zeros(300, device="cuda") for _ in range(2)]
    held = torch.zeros(1000, dtype=mom[0][0].dtype if bits == 32 else torch.uint8, device="cuda").view(mom[0][0].dtype)
    scales = torch.zeros(8, device="cuda")
    bad = [(views(flat, (0, 200)), grads, mom, None), (views(flat, (299, 0)), grads, mom, None),
           (apart, views(apart[0].new_zeros(1000), (0, 100)), [(held[:300], *mom[0][1:]), (held[200:500], *mom[1][1:])], None),
           ([flat[:300], apart[1]], [grads[0], flat[100:400]], mom, None), ([flat[:300], apart[1]], [grads[0], flat[299:599]], mom, None),
           (apart, grads, mom, views(torch.zeros(1000, dtype=BF16, device="cuda"), (0, 150)))]
    if bits == 8:
        bad.append((apart, grads, [(mom[0][0], scales[:3], mom[0][2], mom[0][3]), (mom[1][0], mom[1][1], mom[1][2], scales[2:5])], None))
    for p, g, m, c in bad:
        with pytest.raises((ValueError, head.InkError)):
            head.adamw(p, g, m, 1, copies=c)
    # of several types, in several launches: seen before the first
    wide = torch.zeros(1000, device="cuda")
    p = [apart[0], wide[:300], wide[299:].view(BF16)[:300]]
    m = head.adamw_moments(p, bits)
    with pytest.raises(ValueError):
        head.adamw(p, [torch.ones_like(x) for x in p], m, 1)
    other = [wide[:300], torch.zeros(300, dtype=BF16, device="cuda")]
    with pytest.raises(ValueError):
        head.adamw(other, [grads[0], wide[200:350].view(BF16)], m[:2], 1)
    torch.cuda.synchronize()
    assert not any(x.float().any() for x in (flat, wide, held, scales, *apart, *(y for e in mom for y in e))), "nothing was changed"


@pytest.mark.parametrize("bits", [8, 32])
def test_views_side_by_side_are_ordinary_tensors(bits):
    """Parameters, gradients, moments, scales and copies, each pieces of one buffer without a gap, against tensors of their own."""
    sizes = [128, 256, 384]
    ends = [sum(sizes[:i]) for i in range(4)]
    cut = lambda flat, by=1: [flat[a // by:b // by] for a, b in zip(ends, ends[1:])]          # noqa: E731
    rand = torch.Generator().manual_seed(2)
    flat, grad = torch.randn(768, generator=rand).cuda(), torch.randn(768, generator=rand).cuda()
    own = [x.clone() for x in cut(flat)]
    own_m, own_c = head.adamw_moments(own, bits), [x.to(BF16) for x in own]
    whole = head.adamw_moments([flat], bits)[0]
    pieces = [cut(x, 128 if x.numel() < 768 else 1) for x in whole]
    copy = torch.zeros(768, dtype=BF16, device="cuda")
    for step in (1, 2):
        head.adamw(cut(flat), cut(grad), list(zip(*pieces)), step, copies=cut(copy), seed=3)
        head.adamw(own, [x.clone() for x in cut(grad)], own_m, step, copies=own_c, seed=3)
    assert torch.equal(flat, torch.cat(own)) and torch.equal(copy, torch.cat(own_c))
    for x, y in zip(whole, zip(*own_m)):
        assert torch.equal(x.view(torch.uint8), torch.cat([z.view(torch.uint8) for z in y]))
    # of two types, beside each other in one buffer
    wide = torch.zeros(600, device="cuda")
    p = [wide[:300], wide[300:450].view(BF16)]
    head.adamw(p, [torch.ones_like(x) for x in p], head.adamw_moments(p, bits), 1, lr=0.5, weight_decay=0.0)
    assert torch.allclose(p[0], torch.full_like(p[0], -0.5)) and torch.allclose(p[1].float(), torch.full((300,), -0.5, device="cuda"), atol=2.0 ** -8) and not wide[450:].any()
