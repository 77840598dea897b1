"""Host-side checks of eco_head_*: arguments are refused before any device work, with a status and a text, and the workspace's
size follows the descriptor.  No GPU is needed: addresses are numbers that nothing reads."""
import ctypes as C
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def eco():
    if not os.path.exists(os.path.join(ROOT, "paper_2601_22101_amd", "libeco.so")):
        from paper_2601_22101_amd import build
        build.build()
    from paper_2601_22101_amd import binding
    return binding


def _head(eco, **kw):
    base = dict(rows=7, vocab=1000, dim=64, hidden=0x10000, weights=0x20000, labels=0x30000, top_ids=0x40000, top_logits=0x50000, grad_ce=0x60000, grad_kd=0x70000,
                ce=0x80000, kd=0x90000, lse=0xA0000, lse_tau=0xB0000, picked=0xC0000, grad_hidden=0xD0000, grad_weights=0xE0000, top_k=4, temperature=2.0)
    return eco.make_head(**{**base, **kw})


def _status(eco, fn, *args):
    try:
        fn(*args)
    except eco.EcoError as e:
        assert str(e)
        return e.status
    return 0


def test_struct_layout(eco, tmp_path):
    assert C.sizeof(eco.eco_head_t) == 224
    src = tmp_path / "size.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "eco.h"\nint main(void) { printf("%u %u %u %u\\n", (unsigned)sizeof(eco_head_t), '
                   '(unsigned)offsetof(eco_head_t, rows), (unsigned)offsetof(eco_head_t, temperature), (unsigned)offsetof(eco_head_t, grad_weights_dtype)); return 0; }\n')
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Wextra", "-pedantic", "-Werror", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(tmp_path / "size")], check=True)
    out = subprocess.run([str(tmp_path / "size")], stdout=subprocess.PIPE, text=True, check=True).stdout.split()
    t = eco.eco_head_t
    assert [int(x) for x in out] == [C.sizeof(t), t.rows.offset, t.temperature.offset, t.grad_weights_dtype.offset]


BOTH = [
    (dict(rows=0), "EINVAL"), (dict(vocab=0), "EINVAL"), (dict(dim=0), "EINVAL"),
    (dict(rows=2 ** 23 + 1), "EUNSUPPORTED"), (dict(vocab=2 ** 24 + 1), "EUNSUPPORTED"), (dict(dim=2 ** 16 + 1), "EUNSUPPORTED"),
    (dict(hidden=None), "EINVAL"), (dict(weights=None), "EINVAL"), (dict(labels=None, top_k=0), "EINVAL"),
    (dict(fmt=4), "EINVAL"), (dict(fmt=-1), "EINVAL"), (dict(hidden_dtype=2), "EINVAL"), (dict(top_dtype=7), "EINVAL"),
    (dict(fmt=0), "EINVAL"),                                                       # no scales
    (dict(fmt=0, scales=0x1000), "EINVAL"),                                        # no group
    (dict(fmt=0, scales=0x1000, group_size=100), "EUNSUPPORTED"), (dict(fmt=1, scales=0x1000, group_size=8200), "EUNSUPPORTED"),
    (dict(fmt=0, scales=0x1008, group_size=64), "EALIGN"), (dict(fmt=0, scales=0x1000, group_size=64, scale_dtype=3), "EINVAL"),
    (dict(fmt=0, scales=0x1000, group_size=64, weight_stride=72), "EUNSUPPORTED"),
    (dict(weights=0x20008), "EALIGN"), (dict(hidden=0x10001), "EALIGN"), (dict(hidden=0x10002, hidden_dtype=0), "EALIGN"), (dict(labels=0x30004), "EALIGN"),
    (dict(top_ids=0x40002), "EALIGN"), (dict(top_logits=0x50002), "EALIGN"), (dict(picked=0xC0002), "EALIGN"),
    (dict(hidden_stride=63), "EINVAL"), (dict(weight_stride=63), "EINVAL"), (dict(top_stride=3), "EINVAL"),
    (dict(top_k=1025), "EUNSUPPORTED"), (dict(top_ids=None), "EINVAL"), (dict(top_logits=None), "EINVAL"),
    (dict(temperature=0.0), "EINVAL"), (dict(temperature=-1.0), "EINVAL"), (dict(temperature=float("nan")), "EINVAL"), (dict(temperature=float("inf")), "EINVAL"),
    (dict(picked=None), "EINVAL"), (dict(lse=None), "EINVAL"), (dict(lse_tau=None), "EINVAL"),
]


@pytest.mark.parametrize("kw,want", BOTH)
def test_refused_by_every_call(eco, kw, want):
    h, ws = _head(eco, **kw), 0x100000
    want = getattr(eco, "ECO_" + want)
    assert _status(eco, eco.eco_head_loss, h, ws, 1 << 40, 0) == want
    assert _status(eco, eco.eco_head_loss_backward, h, ws, 1 << 40, 0) == want
    assert _status(eco, eco.eco_head_loss_workspace, h, False) == want


def test_refused_by_one_direction(eco):
    ws = 0x100000
    for kw in (dict(ce=None), dict(kd=None)):
        assert _status(eco, eco.eco_head_loss, _head(eco, **kw), ws, 1 << 40, 0) == eco.ECO_EINVAL
    assert _status(eco, eco.eco_head_loss, _head(eco, ce=0x80002), ws, 1 << 40, 0) == eco.ECO_EALIGN
    for kw in (dict(grad_hidden=None), dict(grad_weights=None), dict(grad_ce=None, grad_kd=None), dict(grad_ce=None, top_k=0), dict(grad_weights_dtype=5),
               dict(grad_hidden_stride=63), dict(grad_weights_stride=63)):
        assert _status(eco, eco.eco_head_loss_backward, _head(eco, **kw), ws, 1 << 40, 0) == eco.ECO_EINVAL, kw
    for kw in (dict(grad_weights=0xE0008), dict(grad_hidden=0xD0001), dict(grad_ce=0x60002)):
        assert _status(eco, eco.eco_head_loss_backward, _head(eco, **kw), ws, 1 << 40, 0) == eco.ECO_EALIGN, kw


def test_workspace(eco):
    h = _head(eco)
    for fn, backward in ((eco.eco_head_loss, False), (eco.eco_head_loss_backward, True)):
        need = eco.eco_head_loss_workspace(h, backward)
        assert need > 0 and need % 256 == 0
        assert _status(eco, fn, h, None, need, 0) == eco.ECO_EINVAL
        assert _status(eco, fn, h, 0x100080, need, 0) == eco.ECO_EALIGN
        assert _status(eco, fn, h, 0x100000, need - 1, 0) == eco.ECO_EINVAL and str(need) in eco.eco_last_error()
    # the logits are not kept: far less than rows x vocab, in either direction
    big = _head(eco, rows=1 << 16, vocab=262144, dim=1152)
    for backward in (False, True):
        assert eco.eco_head_loss_workspace(big, backward) < (1 << 16) * 262144 * 2 // 16
    assert _status(eco, lambda: eco._check(eco.lib.eco_head_loss_workspace(C.byref(h), 0, None))) == eco.ECO_EINVAL
    assert eco.lib.eco_head_loss_workspace(None, 0, C.byref(C.c_size_t())) == eco.ECO_EINVAL
    # every size that the checks let through has a workspace that a 64-bit size holds
    assert 0 < eco.eco_head_loss_workspace(_head(eco, rows=2 ** 23, vocab=2 ** 24, dim=2 ** 16, top_k=1024, fmt=3, hidden_dtype=0), True) < 2 ** 60
