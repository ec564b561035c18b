"""Outputs and workspaces of the position operators that lie over something else are
refused, without a GPU: every call here fails validation."""
import pytest

import paper_2403_10266_amd as dsp
from tests.test_abi_position_cpu import A, BF, F32, _norm, _relpos, _st


@pytest.fixture(scope="module")
def lib():
    return dsp.lib()


# a call whose keys are split, so that it needs a workspace
LONG = dict(X=1, Lq=1, Lk=5000, H=8, Hkv=2, qs=_st(576, 576, 576), os=_st(576, 576, 576),
            ks=_st(5000 * 144, 5000 * 144, 144))
POS = dict(q_pos=A[13], kv_len=A[14])


def test_log_sum_exp_over_something(lib):
    for n in ("q", "k", "v", "o", "bias", "bk", "q_pos", "kv_len"):
        at = dict(q=A[0], k=A[1], v=A[2], o=A[3], bias=A[5], bk=A[6], **POS)[n]
        assert _relpos(lib, **POS, lse=at) == dsp.DSP_ERR_ARG, n
    # 2 x 3 x 4 x 5 floats: their end over the first row, their start over the last
    assert _relpos(lib, lse=A[0] - 4 * 119) == dsp.DSP_ERR_ARG
    assert _relpos(lib, lse=A[0] + 2 * (2 * 15 * 288) - 4) == dsp.DSP_ERR_ARG


def test_forward_outputs_over_tables_and_positions(lib):
    for n in ("bias", "bk", "q_pos", "kv_len"):
        at = dict(bias=A[5], bk=A[6], **POS)[n]
        assert _relpos(lib, **POS, o=at) == dsp.DSP_ERR_ARG, n


def test_workspace_over_something(lib):
    need = lib.dsp_attn_relpos_workspace_bytes(2, 1, 1, 5000, 8, 2, 72, BF)
    for at in (A[0], A[1], A[2], A[3], A[4], A[5], A[6], A[13], A[14], A[2] - need + 16):
        assert _relpos(lib, **LONG, **POS, ws=at) == dsp.DSP_ERR_ARG, hex(at)
    need = lib.dsp_attn_relpos_bwd_workspace_bytes(2, 3, 5, 7, 4, 2, 72, 16, BF)
    for at in (*(A[i] for i in (0, 1, 2, 3, 4, 5, 6, 8, 9, 10, 11, 12, 13, 14)), A[9] - need + 16):
        assert _relpos(lib, True, **POS, ws=at) == dsp.DSP_ERR_ARG, hex(at)


def test_gradients_over_something(lib):
    for n in ("dq", "dk", "dv", "db"):
        for at in (A[4], A[5], A[6], A[13], A[14]):
            assert _relpos(lib, True, **POS, **{n: at}) == dsp.DSP_ERR_ARG, (n, hex(at))
    for at in (A[0], A[1], A[2], A[3], A[8], A[9], A[10], A[11]):
        assert _relpos(lib, True, db=at) == dsp.DSP_ERR_ARG, hex(at)


def test_blocks_between_rows(lib):
    """A block in a gap between rows shares nothing with them: such a call gets as far as
    its workspace.  One element more at either end, and it is refused."""
    # rows of 4 x 72 at a pitch of 904, 5 of them, in units 6000 apart, in batches of 20000
    for es, dt in ((2, BF), (4, F32)):
        wide = _st(20000, 6000, 904)
        for b in range(2):
            for x in range(3):
                for l in range(5):
                    row = A[0] + es * (20000 * b + 6000 * x + 904 * l)
                    last = (b, x, l) == (1, 2, 4)
                    gap = row + es * 288
                    for at, status in ((gap, dsp.DSP_ERR_WORKSPACE), (gap - es * 4, dsp.DSP_ERR_ARG),
                                       (row - 4, dsp.DSP_ERR_ARG), (row, dsp.DSP_ERR_ARG)):
                        kw = dict(qs=wide, dt=dt, db=at, nb=2, ws=None)   # 2 x 4 elements
                        assert _relpos(lib, True, **kw) == status, (es, b, x, l, at - row)
                    if not last:
                        pitch = 6000 - 4 * 904 if l == 4 and x < 2 else 20000 - 2 * 6000 - 4 * 904 if l == 4 else 904
                        end = row + es * (pitch - 8)     # the block's last place before the next row
                        assert _relpos(lib, True, qs=wide, dt=dt, db=end, nb=2, ws=None) == dsp.DSP_ERR_WORKSPACE
                        assert _relpos(lib, True, qs=wide, dt=dt, db=end + es, nb=2, ws=None) == dsp.DSP_ERR_ARG


def test_blocks_beside_rows_that_share_memory(lib):
    """Rows of any stride (one key for every position, rows that overlap): what lies
    inside their span is over them, what lies past it is not (and the call gets as far
    as its workspace)."""
    for st, span in ((_st(1008, 0, 0), 1008 + 144), (_st(1008, 0, 8), 1008 + 4999 * 8 + 144)):
        kw = LONG | dict(ks=st, ws=None)
        for at, status in ((A[1], dsp.DSP_ERR_ARG), (A[1] + 2 * span - 4, dsp.DSP_ERR_ARG),
                           (A[1] + 2 * span, dsp.DSP_ERR_WORKSPACE), (A[1] - 4 * 15, dsp.DSP_ERR_ARG),
                           (A[1] - 4 * 16, dsp.DSP_ERR_WORKSPACE)):      # 2 x 8 floats
            assert _relpos(lib, **kw, lse=at) == status, (span, at - A[1])


def test_norm_outputs_over_gains_and_tables(lib):
    for bwd in (False, True):
        for n in ("yq", "yk"):
            for at in (A[4], A[5], A[6], A[7], A[13], A[6] - 64, A[7] + 4 * 5 * 36 - 4):
                assert _norm(lib, bwd, pos=A[13], **{n: at}) == dsp.DSP_ERR_ARG, (bwd, n, hex(at))


def test_norm_gain_gradients_over_something(lib):
    for n in ("dgq", "dgk"):
        for at in (A[0], A[1], A[2], A[3], A[4], A[5], A[6], A[7], A[8], A[9], A[13], A[0] - 4 * 71,
                   A[1] + 2 * (2 * 15 * 144) - 4):
            assert _norm(lib, True, pos=A[13], **{n: at}) == dsp.DSP_ERR_ARG, (n, hex(at))
    assert _norm(lib, True, dgk=A[10] + 4 * 71) == dsp.DSP_ERR_ARG
    assert _norm(lib, True, dgk=A[10] + 4 * 72, ws=None) == dsp.DSP_ERR_WORKSPACE


def test_norm_workspace_over_something(lib):
    need = lib.dsp_qk_norm_rope_bwd_workspace_bytes(2, 3, 5, 4, 2, 72)
    for at in (*(A[i] for i in range(12)), A[13], A[3] - need + 16):
        assert _norm(lib, True, pos=A[13], ws=at) == dsp.DSP_ERR_ARG, hex(at)


def test_norm_blocks_between_rows(lib):
    """Gains' gradients in a gap between the rows of q and its gradient are apart."""
    wide = _st(20000, 6000, 904)
    gap = A[0] + 2 * (6000 + 904 + 288)
    for at, status in ((gap, dsp.DSP_ERR_WORKSPACE), (gap - 4, dsp.DSP_ERR_ARG), (gap + 2 * 616 - 288, dsp.DSP_ERR_WORKSPACE),
                       (gap + 2 * 616 - 284, dsp.DSP_ERR_ARG)):
        assert _norm(lib, True, qs=wide, dgq=at, ws=None) == status, at - gap


def test_norm_without_rotation_or_a_side(lib):
    """Tables without rotation, and an absent side's arguments, are not looked at."""
    assert _norm(lib, True, rot=0, dgq=A[6], ws=None) == dsp.DSP_ERR_WORKSPACE
    assert _norm(lib, True, Hkv=0, dgq=A[5], ws=None) == dsp.DSP_ERR_WORKSPACE
    assert _norm(lib, True, H=0, dgk=A[4], ws=None) == dsp.DSP_ERR_WORKSPACE
