"""Workspaces of beam search's calls that are large enough but not 256-byte aligned are refused, before anything touches a GPU."""
import pytest

import paper_2412_16434_amd as S

EUNSUPPORTED, EWORKSPACE = -2, -4
BIG = 1 << 40


def _select(ws, ws_bytes):
    return S.load_library().symph_beam_select(0x10, 100, 0, 4, 100, 0x20, 0x30, 0x40, 2, 8, 4, 3, 0x50, 0x60, 0x70, None, ws, ws_bytes,
                                              None)


def _free(ws, ws_bytes):
    return S.load_library().symph_kv_free(0x10, 0x20, None, 4, 0x30, 8, 16, 64, 0x40, 0x50, 0x60, 0x70, None, None, None, 0, None, None, ws,
                                          ws_bytes, None)


def _compact(ws, ws_bytes):
    return S.load_library().symph_kv_compact(0x10, 64, -1, 0x20, None, 4, 0x30, 8, 16, 0x40, 0x50, 0x60, 0x70, 0x80, 32, 0x90, ws,
                                             ws_bytes, None)


@pytest.mark.parametrize("call", [_select, _free, _compact])
@pytest.mark.parametrize("address", [0x1001, 0x1002, 0x1004, 0x1010, 0x1080])
def test_workspaces_at_other_addresses_are_refused(call, address):
    assert call(address, BIG) == EUNSUPPORTED
    assert call(address, 3) == EWORKSPACE  # (too small comes first, as in the attention call)
