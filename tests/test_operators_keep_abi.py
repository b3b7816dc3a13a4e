"""The flag of the gated feed-forward entries for FP32 G and U: checked on the host, nothing is launched."""
import paper_2511_16041_b200 as atb

P, KEEP, ARGUMENT, NULL, SMALL = 1 << 20, 256, 9, 1, 7


def test_flag():
    lib = atb.load_library()
    M, D, F = 4, 64, 136
    need = lib.atb_gated_ffn_workspace_bytes(M, D, F)
    ok = dict(M=M, D=D, F=F, act=0, x=P, ldx=D, wg=P, wu=P, ldw=F, wd=P, ldwd=D, y=P, ldy=D, h=P, g=P, u=P, ws=P, n=need, stream=None)
    call = lambda **k: lib.atb_gated_ffn(*{**ok, **k}.values())  # noqa: E731
    for act in (KEEP + 3, KEEP + 255, 2 * KEEP, 3 * KEEP, -KEEP, -1):
        assert call(act=act) == ARGUMENT, act
    assert call(act=KEEP, g=None) == NULL and call(act=KEEP + 1, x=None) == NULL and call(act=KEEP, M=0) == 0
    need = lib.atb_gated_ffn_backward_workspace_bytes(M, D, F)
    ok = dict(M=M, D=D, F=F, act=0, dy=P, lddy=D, x=P, ldx=D, wg=P, wu=P, ldw=F, wd=P, ldwd=D, h=P, g=P, u=P, dx=P, lddx=D, dwg=P, dwu=P, lddw=F,
              dwd=P, lddwd=D, ws=P, n=need, stream=None)
    back = lambda **k: lib.atb_gated_ffn_backward(*{**ok, **k}.values())  # noqa: E731
    for act in (KEEP + 3, 2 * KEEP, -KEEP):
        assert back(act=act) == ARGUMENT, act
    assert back(act=KEEP + 2, u=None) == NULL and back(act=KEEP, n=need - 1) == SMALL
