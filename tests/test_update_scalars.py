"""What the update reads from the device besides its tensors (the norm, the learning rate, the step's number) may not lie in what it writes: workgroups that start later would read what became of it."""

import pytest
import torch

from test_training_refusals import adamw, built  # noqa: F401

# p, m, v: 4000 bytes each from 0x10000, 0x30000, 0x40000
INSIDE = [0x10000, 0x10008, 0x10000 + 3992, 0x30008, 0x40010]


@pytest.mark.parametrize("name", ["norm", "lr_at", "step_at"])
def test_scalars_in_what_is_written(name):
    for at in INSIDE:
        assert adamw(**{name: at}) == -9
    assert adamw(**{name: 0x50008}, copy=0x50000) == -9
    # moments in 8 bits: rows up to the next multiple of 128, a byte of scale for each
    eight = dict(m_scale=0x60000, v_scale=0x70000)
    for at in (0x30000 + 1016, 0x40000, 0x60000, 0x70000):
        assert adamw(**{name: at}, **eight) == -9
    # in another tensor of the call
    far = dict(p=0x110000, g=0x120000, m=0x130000, v=0x140000)
    assert adamw([{}, far], **{name: 0x130008}) == -9
    assert adamw([dict(numel=0), far], **{name: 0x140000}) == -9


def test_a_scalar_whose_end_reaches_in():
    assert adamw(step_at=0x10000 - 8, p=0x10000 - 4) == -9


@pytest.mark.gpu
def test_scalars_of_tensors():
    """As a caller meets it: one buffer of everything.  What is only read may hold them."""
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_1803_03288_amd import binding, layers
    room = torch.full((4096,), 0.5, device="cuda")
    p, d, one = room[:1000], torch.full((1000,), 0.25, device="cuda"), torch.full((1000,), 0.25, device="cuda")
    moments = layers.adamw_moments([p], 32)
    for more in (dict(norm=room[999:1000], max_norm=1.0), dict(lr=p[:1]), dict(lr=moments[0].v[5:6]), dict(norm=moments[0].m[:1])):
        with pytest.raises(binding.TicTacError) as e:
            layers.adamw_step([p], [d], moments, 1, **more)
        assert e.value.code == -9
    with pytest.raises(binding.TicTacError):
        layers.adamw_step([p], [d], moments, room[998:1000].view(torch.int64))
    assert torch.equal(room, torch.full_like(room, 0.5))
    want = torch.full((1000,), 0.5, device="cuda")
    layers.adamw_step([want], [d], layers.adamw_moments([want], 32), 1, lr=0.25, norm=one[:1], max_norm=1.0)
    layers.adamw_step([p], [d], moments, 1, lr=d[3:4], norm=d[7:8], max_norm=1.0)      # in the gradient
    room[3000] = 0.25
    layers.adamw_step([room[2000:3000]], [d], layers.adamw_moments([p], 32), 1, lr=0.25, norm=room[3000:3001], max_norm=1.0)       # right behind the parameter
    # (the rate on the device: its factors are formed by other functions)
    assert float((p - want).abs().max()) <= 2.0 ** -22 and torch.equal(room[2000:3000], want)
