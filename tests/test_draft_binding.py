"""What the binding of the steps of several new tokens hands to the library:
counts that int32 does not hold are its invalid argument, not their low bits,
and a workspace is one piece of memory (CPU, no kernel is launched)."""
import pytest
import torch

from paper_2607_06827_amd import speechkv as skv
from test_draft_abi import E_ARG, host

FAR = 2 ** 32 + 3  # 3 in its low 32 bits


def one_sequence():
    x = host()
    c = x["cache"]
    return skv.PagedKV(c.k_pages, c.v_pages, c.block_table[:1].contiguous()), x["i32"]


def test_append_refuses_more_rows_than_int32_holds():
    cache, i32 = one_sequence()
    k = torch.zeros(1, 1, 2, 64, dtype=torch.bfloat16).expand(1, FAR, 2, 64)
    with pytest.raises(skv.SpeechKVError) as e:
        skv.speechkv_append_kv(k, k, cache, i32(1), stream=0)
    assert e.value.status == E_ARG


def test_commit_refuses_more_entries_than_int32_holds():
    cache, i32 = one_sequence()
    path = torch.empty(1, FAR, dtype=torch.int32)  # (never touched)
    with pytest.raises(skv.SpeechKVError) as e:
        skv.speechkv_tree_commit(skv.CacheStack([cache], [i32(1)]), path, i32(1), 5, stream=0)
    assert e.value.status == E_ARG


def stub(monkeypatch, name):
    got = []
    monkeypatch.setattr(skv, "_lib", type("Lib", (), {name: staticmethod(lambda *a: got.append(a) or 0)}))
    return got


class Rows(torch.Tensor):
    """A tensor that says it has one value for each of FAR sequences."""

    def numel(self):
        return FAR


def far_batch(monkeypatch):
    """A cache of FAR sequences (its packing aside)."""
    cache = one_sequence()[0]
    packed, shape, _ = cache._paged_kv_for(None)
    monkeypatch.setattr(cache, "_paged_kv_for", lambda wanted: (packed, shape, FAR), raising=False)
    return cache, torch.zeros(1, dtype=torch.int32).as_subclass(Rows)


def test_append_and_tree_refuse_more_sequences_than_int32_holds(monkeypatch):
    cache, lens = far_batch(monkeypatch)
    got = stub(monkeypatch, "speechkv_append_kv")
    k = torch.zeros(1, 1, 2, 64, dtype=torch.bfloat16).expand(FAR, 1, 2, 64)
    skv.speechkv_append_kv(k, k, cache, lens, stream=0)
    assert got[0][10] == -1  # batch
    got = stub(monkeypatch, "speechkv_tree_attn")

    class Query(torch.Tensor):
        def is_contiguous(self):
            return True

    q = torch.zeros(1, 1, 4, 64, dtype=torch.bfloat16).expand(FAR, 1, 4, 64).as_subclass(Query)
    skv.speechkv_tree_attn(q, cache, lens, 5, q, stream=0)
    assert got[0][1] == -1


def test_commit_refuses_more_sequences_than_int32_holds(monkeypatch):
    cache, i32 = one_sequence()
    stack = skv.CacheStack([cache], [i32(1)])
    stack.batch = FAR
    path = torch.empty(FAR, 1, dtype=torch.int32)  # (never touched)
    got = stub(monkeypatch, "speechkv_tree_commit")
    skv.speechkv_tree_commit(stack, path, path[:, 0], 5, stream=0)
    assert got[0][2] == -1


@pytest.mark.parametrize("ws", [torch.empty(1, dtype=torch.uint8).expand(1 << 20),
                                torch.empty(1 << 12, dtype=torch.float32)[::2],
                                torch.empty(64, 64).t()])
def test_tree_refuses_a_workspace_that_is_not_one_piece(ws):
    x = host()
    with pytest.raises(ValueError):
        skv.speechkv_tree_attn(x["q"], x["cache"], x["lens"], 5, x["q"].clone(), workspace=ws, stream=0)
