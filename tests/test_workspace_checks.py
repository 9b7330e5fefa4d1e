"""CPU tests: workspaces that the calls over a paged cache do not take, refused before any library call.  (The marshalling of CPU tensors ends at
that check here: the tests give it nothing that passes.)"""
import pytest
import torch

from paper_2511_02043_amd import functional as F

B, H, HKV, D, PAGE = 1, 4, 2, 64, 16
CACHE = torch.zeros(4, PAGE, HKV, D, dtype=torch.bfloat16)
LENS, TABLE = torch.full((B,), 5, dtype=torch.int32), torch.zeros(B, 4, dtype=torch.int32)
VARIANT = (0.125, 0, 0.0, 1, 0, None)                # scale, score_mod, soft-cap, mask, window, slopes


def decode(ws):
    F._host().paged(True, torch.zeros(B, H, D, dtype=torch.bfloat16), CACHE, CACHE, LENS, TABLE, 64, *VARIANT, ws, False, 0)


def prefill(ws):
    F._host().paged(False, torch.zeros(B, H, 3, D, dtype=torch.bfloat16), CACHE, CACHE, LENS, TABLE, 64, *VARIANT, ws, False, 0)


def decode_weights(ws):
    F._host().decode_weights(torch.zeros(B, H, D, dtype=torch.bfloat16), CACHE, CACHE, torch.zeros(B, HKV, 64), LENS, TABLE, 64, *VARIANT, ws, False, 0)


def key_weights(ws):
    F._host().key_weights(torch.zeros(B, H, 3, D, dtype=torch.bfloat16), CACHE, torch.zeros(B, H, 3), torch.zeros(B, HKV, 64), LENS, TABLE, 64, *VARIANT, ws, 0)


@pytest.mark.parametrize("call", [decode, prefill, decode_weights, key_weights])
@pytest.mark.parametrize("ws,what", [
    (torch.empty(1 << 22, dtype=torch.uint8, device="meta"), "on cpu"),              # memory of another device
    (torch.empty(1 << 22, dtype=torch.uint8)[::2], "contiguous"), (torch.empty(1 << 11, 1 << 11, dtype=torch.uint8)[:, 1:], "contiguous"),
    (torch.empty(1, dtype=torch.uint8).expand(1 << 22), "contiguous"),               # (a byte that claims to be four million)
], ids=["device", "every other byte", "columns", "expanded"])
def test_workspaces_that_are_refused(call, ws, what):
    with pytest.raises(ValueError, match=f"workspace must be .*{what}"):
        call(ws)
