"""Host side of the operators of speculative rollouts and distillation: workspaces by device (no GPU needed)."""
import pytest

torch = pytest.importorskip("torch")


def test_workspace_sizes_are_remembered_by_device(monkeypatch):
    """A size may depend on the device's multiprocessors: what one device needs says nothing about another."""
    from paper_2608_17641_b200 import binding
    current = {"device": 0, "asked": 0}

    class Library:
        @staticmethod
        def rlcs_verify_drafts_workspace_bytes(T, B):
            current["asked"] += 1
            return 1000 * (current["device"] + 1) + T

    monkeypatch.setattr(binding, "lib", lambda: Library)
    monkeypatch.setattr(binding, "_new", lambda shape, dtype, device: torch.empty(shape, dtype=dtype))
    monkeypatch.setattr(binding, "_scratch_bytes", {})
    for _ in range(2):
        for device in (0, 1):
            current["device"] = device
            _, room, workspace = binding._scratch("rlcs_verify_drafts_workspace_bytes", (6, 2), None, device)
            assert room == workspace.numel() == 1000 * (device + 1) + 6
    assert current["asked"] == 2
