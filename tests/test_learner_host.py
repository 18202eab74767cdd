"""Host-side checks of include/echo_learner.h that need no GPU: exported symbols, sizes, refusals with a message."""
import ctypes as C
import os
import re

import numpy as np
import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def learner():
    from paper_2602_02192_amd import learner as l
    return l


def test_library_exports_every_declared_entry_point(learner):
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "echo_learner.h")).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(echo_[a-z0-9_]+)\s*\(", text)))
    assert names == sorted(learner.EXPORTS)
    for n in names:
        assert hasattr(learner.lib, n)


def message(learner):
    return learner.lib.echo_last_error(None).decode()


@pytest.mark.parametrize("change,word", [(dict(dtype=3), "ECHO_F32"), (dict(rows=-1), "rows"), (dict(rows=1 << 31), "rows"), (dict(vocab=0), "vocab"), (dict(row_stride=9), "row_stride"),
                                         (dict(row_stride=1 << 62), "row_stride"), (dict(temperature=0.0), "temperature"), (dict(temperature=float("inf")), "temperature"),
                                         (dict(temperature=1e-39), "temperature"), (dict(logits=None), "NULL"), (dict(logits=66), "aligned"), (dict(targets=33), "targets")])
def test_descriptions_of_logits_that_are_refused(learner, change, word):
    x = learner._Logits(64, 64, 2, 10, 10, 0, 1.0)
    for k, v in change.items():
        setattr(x, k, v)
    for call in (lambda: learner.lib.echo_token_logprobs(C.byref(x), 0, 64, 64, 64, None, None, 256, 1 << 40, None),
                 lambda: learner.lib.echo_token_logprobs_grad(C.byref(x), 64, 64, 64, 64, 64, 10, None),
                 lambda: learner.lib.echo_policy_loss(C.byref(x), 64, 64, None, None, None, C.byref(learner._LossOpts(0.2, 0.2, 4, 2, 0, 0)), 64, 64, 64, 64, 10, 256, 1 << 40, None)):
        assert call() == -1 and word in message(learner)


def test_arguments_that_are_refused(learner):
    x = learner._Logits(64, None, 2, 10, 10, 0, 1.0)
    L = learner.lib
    assert L.echo_token_logprobs(None, 0, None, None, None, None, None, None, 0, None) == -1
    assert L.echo_token_logprobs(C.byref(x), 0, 64, None, None, None, None, 256, 1 << 40, None) == -1 and "targets" in message(learner)
    assert L.echo_token_logprobs(C.byref(x), 3, None, None, None, 64, None, 256, 1 << 40, None) == -1 and "top_k" in message(learner)
    assert L.echo_token_logprobs(C.byref(x), 11, None, None, None, 64, 64, 256, 1 << 40, None) == -1 and "top_k" in message(learner)
    assert L.echo_token_logprobs(C.byref(x), 0, None, 65, None, None, None, 256, 1 << 40, None) == -1 and "aligned" in message(learner)
    big = learner._Logits(64, 64, 2, 151936, 151936, 1, 1.0)
    need = L.echo_token_logprobs_workspace(C.byref(big), 8)
    if need:
        assert L.echo_token_logprobs(C.byref(big), 8, 64, 64, 64, 64, 64, 256, need - 1, None) == -2 and "workspace" in message(learner)
        assert L.echo_token_logprobs(C.byref(big), 8, 64, 64, 64, 64, 64, 128, need, None) == -2 and "aligned" in message(learner)
    assert L.echo_token_logprobs_workspace(C.byref(big), 65) == 0 and L.echo_policy_loss_workspace(None) == 0
    assert L.echo_policy_loss(C.byref(big), 64, 64, None, None, None, None, 64, 64, 64, 64, 151936, 256, 1 << 40, None) == -1 and "opts" in message(learner)
    assert L.echo_token_logprobs_grad(C.byref(big), 64, 64, 64, 64, 64, 151935, None) == -1 and "stride" in message(learner)
    assert L.echo_token_logprobs_grad(C.byref(big), None, 64, 64, 64, 64, 151936, None) == -1 and "lse" in message(learner)


@pytest.mark.parametrize("rows,vocab,taken", [((1 << 24) - 1, 8, True), (1 << 24, 8, False), (1 << 24, 8192, False), ((1 << 23) - 1, 8193, True), (1 << 23, 8193, False),
                                              ((1 << 24) - 1, 1, True), (1 << 24, 1, False), (511, 1 << 28, True), (512, 1 << 28, False)])
def test_logits_of_more_workgroups_than_a_launch_has(learner, rows, vocab, taken):
    """A launch has less than 2^32 threads; what would need more is refused before anything is queued, and has no workspace."""
    x = learner._Logits(None, None, rows, vocab, vocab, 1, 1.0)    # (no logits: what is taken is refused for that)
    for call in (lambda: learner.lib.echo_token_logprobs(C.byref(x), 0, None, 64, 64, None, None, 256, 1 << 60, None),
                 lambda: learner.lib.echo_token_logprobs_grad(C.byref(x), 64, 64, None, 64, 64, vocab, None),
                 lambda: learner.lib.echo_policy_loss(C.byref(x), 64, 64, None, None, None, C.byref(learner._LossOpts(0.2, 0.2, 4, 2, 0, 0)), 64, 64, 64, 64, vocab, 256, 1 << 60, None)):
        assert call() == -1 and ("logits are NULL" if taken else "2^24") in message(learner)
    if not taken:
        assert learner.lib.echo_token_logprobs_workspace(C.byref(x), 0) == 0 and learner.lib.echo_policy_loss_workspace(C.byref(x)) == 0


def test_no_parameters(learner):
    with pytest.raises(ValueError, match="no params"):
        learner.AdamW([], 1e-3)


def test_a_loss_in_parts_has_room_for_them(learner):
    """Rows of few vectors are never cut; a cut row has two parts of 16 bytes at least, whatever its type, its length and their number."""
    for dtype, entries in ((0, 4), (1, 8), (2, 8)):
        for vocab in (1, 7, 8, 1024, 35000, 65536, 65537, 70000, 73728, 73729, 100003, 151936, 262144, 500000):
            for rows in (1, 8, 32, 95, 96, 128, 175, 176, 256, 257, 300, 512, 4096):
                need = learner.lib.echo_policy_loss_workspace(C.byref(learner._Logits(64, 64, rows, vocab, vocab, dtype, 1.0)))
                if -(-vocab // entries) <= 8192:
                    assert need == 0
                assert need == 0 or (need >= rows * 2 * 16 and need % 256 == 0)
    assert learner.lib.echo_policy_loss_workspace(C.byref(learner._Logits(64, 64, 32, 151936, 151936, 1, 1.0))) > 0


def test_sizes_of_the_update(learner):
    def i64(*v):
        return np.array(v, np.int64)

    L = learner.lib
    for sizes, states in ((i64(1), 256), (i64(256, 0, 257), 768), (i64(), 0)):
        assert L.echo_adamw_state_numel(sizes.ctypes.data, sizes.size) == states == learner.state_numel([torch.empty(n) for n in sizes])
        assert L.echo_grad_norm_workspace(sizes.ctypes.data, sizes.size) >= 8
    bad = i64(5, -1)
    assert L.echo_adamw_state_numel(bad.ctypes.data, 2) == -1 and L.echo_grad_norm_workspace(bad.ctypes.data, 2) == 0
    assert L.echo_adamw_state_numel(None, 2) == -1
    grads = np.array([64], np.uint64)
    assert L.echo_grad_norm(grads.ctypes.data, i64(5).ctypes.data, 1, 3, 64, 256, 1 << 20, None) == -1
    assert L.echo_grad_norm(grads.ctypes.data, i64(5).ctypes.data, 1, 0, None, 256, 1 << 20, None) == -1 and "out_norm" in message(learner)
    assert L.echo_grad_norm(grads.ctypes.data, i64(5).ctypes.data, 1, 0, 64, 256, 8, None) == -2
    assert L.echo_adamw_step(None, None) == -1


def test_tensors_that_are_not_on_a_gpu(learner):
    z = torch.zeros(3)
    with pytest.raises(ValueError):
        learner.token_logprobs(torch.zeros(3, 5), torch.zeros(3, dtype=torch.int32))
    with pytest.raises(ValueError):
        learner.policy_loss(torch.zeros(3, 5), torch.zeros(3, dtype=torch.int32), z, z)
    with pytest.raises(ValueError):
        learner.adamw_step([z], [z.clone()], torch.zeros(256), torch.zeros(256), step=1, lr=1e-3)
    with pytest.raises(ValueError):
        learner.grad_norm([z])
