"""The losses refuse, before any launch, small arrays that overlap or are not aligned
(CPU only; the addresses are never used)."""
import pytest

import paper_1909_08029_amd as rip
from test_train_ops_host import A, B, C, D, E, POLICY, PREF, W, call

OVERLAP, ALIGN = rip.RIP_E_OVERLAP, rip.RIP_E_ALIGN


@pytest.mark.parametrize("fn,defaults,change,code", [
    ("rip_policy_loss", POLICY, dict(logp=C), OVERLAP),                 # over old_logp
    ("rip_policy_loss", POLICY, dict(logp=C + 4096), OVERLAP),          # advantage
    ("rip_policy_loss", POLICY, dict(w=D + 128), OVERLAP),              # weight under logp
    ("rip_policy_loss", POLICY, dict(ref=D + 128, kl=0.1), OVERLAP),
    ("rip_policy_loss", POLICY, dict(ref=D + 156, kl=0.1), OVERLAP),    # the last element
    ("rip_policy_loss", POLICY, dict(loss=C + 28), OVERLAP),            # loss in old_logp
    ("rip_policy_loss", POLICY, dict(loss=D + 128), OVERLAP),           # in logp
    ("rip_policy_loss", POLICY, dict(logp=B), OVERLAP),                 # over targets
    ("rip_policy_loss", POLICY, dict(logp=A + 64), OVERLAP),            # over logits
    ("rip_policy_loss", POLICY, dict(logp=E + 64), OVERLAP),            # over grad
    ("rip_policy_loss", POLICY, dict(loss=W + 8), OVERLAP),             # in the workspace
    ("rip_policy_loss", POLICY, dict(adv=E + 64), OVERLAP),             # grad over advantage
    ("rip_policy_loss", POLICY, dict(old=W), OVERLAP),                  # workspace over old_logp
    ("rip_policy_loss", POLICY, dict(grad=A, adv=A + 64), OVERLAP),     # in place
    ("rip_policy_loss", POLICY, dict(grad=B), OVERLAP),
    ("rip_policy_loss", POLICY, dict(logp=D + 130), ALIGN),
    ("rip_policy_loss", POLICY, dict(old=C + 1), ALIGN),
    ("rip_policy_loss", POLICY, dict(loss=D + 2), ALIGN),
    ("rip_pref_loss", PREF, dict(seq=D + 120), OVERLAP),                # into logp
    ("rip_pref_loss", PREF, dict(seq=C + 4096), OVERLAP),               # over ref_logp
    ("rip_pref_loss", PREF, dict(seq=C), OVERLAP),                      # over the offsets
    ("rip_pref_loss", PREF, dict(loss=D + 64), OVERLAP),
    ("rip_pref_loss", PREF, dict(logp=C + 16), OVERLAP),
    ("rip_pref_loss", PREF, dict(logp=W), OVERLAP),
    ("rip_pref_loss", PREF, dict(off=E), OVERLAP),
    ("rip_pref_loss", PREF, dict(grad=A, ref=A + 16), OVERLAP),
    ("rip_pref_loss", PREF, dict(off=C + 2), ALIGN),
    ("rip_pref_loss", PREF, dict(ref=C + 4098), ALIGN),
    ("rip_pref_loss", PREF, dict(seq=D + 65), ALIGN),
])
def test_refused_before_any_launch(fn, defaults, change, code):
    assert call(fn, defaults, **change) == code
    assert rip.lib.rip_last_error()
