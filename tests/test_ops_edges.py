"""Edges of the operators that make a worker's gradient that need no GPU."""
import copy
import pickle

import pytest
import torch

from paper_1905_10936_b200 import binding as ef
from paper_1905_10936_b200 import build as efbuild
from paper_1905_10936_b200 import ops


@pytest.fixture(scope="module", autouse=True)
def built():
    efbuild.build_library()
    efbuild.build_torch_binding()


def host_checkpoint(n, c):
    """A checkpoint whose memory is on the host: no call takes it."""
    size = n * ops.checkpoint_pitch(c) + 4 * n * ops.checkpoint_groups(c)
    return ops.Checkpoint._of(torch.randint(-127, 128, (size,), dtype=torch.int8), n, c)


@pytest.mark.parametrize("how", [copy.deepcopy, lambda k: pickle.loads(pickle.dumps(k))], ids=["deepcopy", "pickle"])
def test_a_copied_checkpoint_refers_to_its_own_memory(how):
    kept = host_checkpoint(3, 200)
    other = how(kept)
    assert (other.rows, other.cols) == (3, 200) and torch.equal(other.codes, kept.codes)
    assert not any(isinstance(v, int) and v > 1 << 20 for v in other._where), "an address"
    before = kept.codes.clone()
    other.codes.zero_()
    assert torch.equal(kept.codes, before) and not bool(other._where[2][:other.codes.numel()].any())


def test_a_checkpoint_that_is_not_on_a_gpu_is_refused():
    """As one that was unpickled to the host is: its addresses mean nothing there."""
    kept = host_checkpoint(4, 40)
    for call in (lambda: ops.checkpoint_load(kept), lambda: ops.checkpoint_weight_grad(kept, torch.ones(4, 8))):
        with pytest.raises(ValueError, match="CUDA"):
            call()


BUF = 4096                                   # any non-null, aligned value: never dereferenced on the host


def test_widths_whose_bytes_overflow_are_too_large():
    for dtype, c in ((0, (1 << 62) + 8), (1, (1 << 63) - 8), (0, 409601), (1, 819201)):
        for name, args in (("ef_token_logprob", (dtype, 4, c, BUF, c, BUF, 1.0, BUF, 0)),
                           ("ef_policy_loss", (dtype, 4, c, BUF, c, BUF, BUF, BUF, BUF, None, 0.2, 0.2, 0.0, 1.0, BUF, BUF, BUF, None, 0, 0))):
            with pytest.raises(ef.EFError) as ei:
                getattr(ef, name)(*args)
            assert ei.value.status == ef.EF_ERR_TOO_LARGE, (name, c)


def test_a_stride_past_the_copy_engine_s_limit_goes_through_the_workspace():
    need = ef.ef_checkpoint_weight_grad_workspace_bytes
    assert need(1, 1, 128, 128, BUF, (1 << 39) - 8) == 0
    assert need(1, 1, 128, 128, BUF, 1 << 39) >= 64 * 128 * 2


def test_the_native_half_belongs_to_one_torch(monkeypatch):
    """Built again where another torch is installed, and refused if it was not."""
    class Compiled(Exception):
        pass

    def run(*args, **kwargs):
        raise Compiled

    monkeypatch.setattr(efbuild.subprocess, "run", run)
    assert efbuild.build_torch_binding() == efbuild.TORCH_BINDING              # up to date: nothing is compiled
    monkeypatch.setattr(torch, "__version__", "0.0.0")
    with pytest.raises(Compiled):
        efbuild.build_torch_binding()
    monkeypatch.setattr(ops, "_bound", None)
    with pytest.raises(OSError, match="built against torch"):
        ops.checkpoint_load(host_checkpoint(1, 8))
