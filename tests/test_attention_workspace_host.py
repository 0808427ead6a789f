"""What the attention's workspace needs from the binding and the header (no GPU)."""
import ctypes
import re
from pathlib import Path

import pytest

ROOT = Path(__file__).resolve().parent.parent


@pytest.fixture(scope="module")
def gs(built_lib):
    from paper_2609_33977_gb300 import groupsparse
    return groupsparse


def test_counter_bytes_are_the_headers(gs):
    text = (ROOT / "include" / "groupsparse.h").read_text()
    assert int(re.search(r"#define GS_ATTENTION_COUNTER_BYTES (\d+)", text).group(1)) == gs.ATTENTION_COUNTER_BYTES


def test_the_legacy_stream_is_in_no_capture(gs):
    v = ctypes.c_uint64(7)
    assert gs.lib.gs_capture_id(None, ctypes.byref(v)) == 0 and v.value == 0
    assert gs.lib.gs_capture_id(None, None) == 1


def test_a_timeout_drops_the_streams_workspaces(gs, monkeypatch):
    monkeypatch.setattr(gs, "_stream_ptr", lambda stream=None: 0)
    monkeypatch.setattr(gs, "_attention_ws", {(0, 0): "counters of a kernel that gave up"})
    monkeypatch.setattr(gs.lib, "gs_device_status", lambda s: 0)
    assert gs.device_status() == gs.GS_OK and gs._attention_ws
    monkeypatch.setattr(gs.lib, "gs_device_status", lambda s: 5)
    assert gs.device_status() == gs.GS_ERR_DEVICE_TIMEOUT and not gs._attention_ws


def test_the_attentions_wait_hook_checks_its_arguments(gs):
    f = gs.lib.gs_debug_inject_attention_wait
    assert f(2, 1000) == 1 and f(-1, 1000) == 1 and f(0, 1_000_000_001) == 1
    assert f(0, 0) == 0 and f(1, 0) == 0
