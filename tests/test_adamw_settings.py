"""AdamW's settings are taken as the numbers they are at the call (CPU)."""
import numpy as np
import pytest

import paper_1909_08029_amd as rip


def scalars(**change):
    return rip.rip_adamw_scalars(**dict(dict(step=3, lr=1e-3), **change)).numpy().view(np.uint32).tolist()


@pytest.mark.parametrize("name", ["lr", "eps", "weight_decay", "grad_scale"])
def test_a_tensor_changed_in_place(name):
    """A schedule that scales one tensor: the second call takes its new value."""
    import torch
    x = torch.tensor(1e-3, dtype=torch.float64)
    before = scalars(**{name: x})
    x.mul_(0.5)
    assert before == scalars(**{name: 1e-3})
    assert scalars(**{name: x}) == scalars(**{name: 5e-4})


def test_betas_changed_in_place():
    import torch
    beta = torch.tensor(0.5, dtype=torch.float64)
    before = scalars(betas=[beta, 0.999])
    beta.mul_(0.5)
    assert before == scalars(betas=(0.5, 0.999)) != scalars(betas=[beta, 0.999])
    assert scalars(betas=[beta, 0.999]) == scalars(betas=(0.25, 0.999))


@pytest.mark.parametrize("lr", [np.float32(0.25), np.float64(0.25), np.array(0.25), 0.25])
@pytest.mark.parametrize("seed", [np.int64(7), np.uint64(7), np.array(7), 7, 7 + 2 ** 64])
def test_other_numbers(lr, seed):
    assert scalars(lr=lr, seed=seed) == scalars(lr=0.25, seed=7)


@pytest.mark.parametrize("bad", [dict(lr="1"), dict(lr=None), dict(seed=1.5), dict(betas=(0.9,)),
                                 dict(betas=(0.9, 0.99, 0.999))])
def test_refused(bad):
    with pytest.raises((TypeError, ValueError)):
        scalars(**bad)
