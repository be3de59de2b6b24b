"""The binding with a library built before its functions (CPU only)."""
import pytest

import paper_1909_08029_amd as rip
from paper_1909_08029_amd import _train_ops


class Older:
    """The library without one function."""

    def __init__(self, lacks):
        self.lacks = lacks

    def __getattr__(self, name):
        if name == self.lacks:
            raise AttributeError(name)
        return getattr(rip.lib, name)


@pytest.mark.parametrize("name", ["rip_embed_lookup", "rip_ckpt_wgrad_workspace", "rip_policy_loss"])
def test_an_older_library_is_named_with_its_version(monkeypatch, name):
    monkeypatch.setattr(_train_ops, "lib", Older(name))
    with pytest.raises(ImportError, match=rf"ABI version {rip.abi_version()}.*no {name};.*build\(\)"):
        _train_ops._declare()


def test_the_library_at_hand_is_taken():
    _train_ops._declare()
