"""Whose workspace the 8-bit cache's attention uses, on the host: never the one of the 16-bit calls,
which a graph captured with them goes on using wherever it is replayed."""
import os

from paper_2606_18394_amd import binding, build


def test_not_shared_with_the_16_bit_calls(monkeypatch):
    monkeypatch.setattr(binding, "_workspaces", {})
    theirs = binding.workspace("attn", 5000, "cpu", 0)       # what a captured 16-bit call holds
    ours = binding._attention_workspace(4000, "cpu", 0)
    assert ours.data_ptr() != theirs.data_ptr() and not ours.any() and ours.numel() >= 4000
    assert binding._attention_workspace(100, "cpu", 0) is ours
    assert binding.workspace("attn", 100, "cpu", 0) is theirs


def test_both_halves_ask_for_the_same_kind(monkeypatch):
    asked = []
    monkeypatch.setattr(binding, "workspace", lambda kind, *a: asked.append(kind))
    binding._attention_workspace(4000, "cpu", 0)
    with open(os.path.join(build.CSRC, "tv_binding.cpp")) as f:
        assert f'PyUnicode_FromString("{asked[0]}")' in f.read() and asked != ["attn"]
