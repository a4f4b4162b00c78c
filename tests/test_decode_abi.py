"""Decode entry points on the CPU: scaled tables against the oracle, and every
argument check, which fires before any HIP call (nothing here launches a kernel:
tests that would reach a launch skip when a device is present)."""
import numpy as np
import pytest
import torch

from oracle import decode as od

kvb = pytest.importorskip("paper_2608_21362_amd.kvb")

NO_GPU = torch.cuda.device_count() == 0
FAKE = 0x10000  # never dereferenced: validation rejects the call first
EINVAL, EUNSUPPORTED = kvb.KVB_EINVAL, kvb.KVB_EUNSUPPORTED


def _status(call, **over):
    with pytest.raises(kvb.KvbError) as e:
        call(**over)
    assert e.value.message
    return e.value.status


# ---- tables -------------------------------------------------------------------

SCALINGS = [
    (od.NONE, {}), (od.LINEAR, dict(factor=8.0)), (od.NTK, dict(factor=4.0)),
    (od.PARTS, dict(factor=8.0, original_len=8192, low=1.0, high=4.0)),
    (od.PARTS, dict(factor=4.0, original_len=4096, low=1.0, high=32.0, attn_factor=1.2)),
    (od.INDEX, dict(factor=4.0, original_len=32768, low=1.0, high=32.0, attn_factor=1.138629436)),
    (od.INDEX, dict(factor=16.0, original_len=64, low=1.0, high=32.0)),
]


@pytest.mark.parametrize("theta,rot", [(1e4, 64), (1e6, 128), (5e5, 16)])
@pytest.mark.parametrize("kind,args", SCALINGS)
def test_scaled_table(kind, args, theta, rot):
    pos = np.array([0, 1, -1, 77, 4095, 32768, 1 << 20, 2 ** 31 - 1, -(2 ** 31)], np.int32)
    c, s = kvb.kvb_rope_scaled_table(theta, rot, kvb.rope_scaling(kind, **args), pos)
    factor = args.get("attn_factor", 1.0)
    w = od.frequencies(theta, rot, kind, **{k: v for k, v in args.items() if k != "attn_factor"})
    oc, os_ = od.table(w, pos, factor)
    # both in double: frequencies are a few 2^-53 apart, so angles up to 2^31 are 2^-20 apart
    # at most, on top of one rounding to float
    near = 2.0 ** -23 * factor + np.abs(pos.astype(np.float64))[:, None] * 2.0 ** -51 * factor
    assert np.all(np.abs(c.astype(np.float64) - oc) <= near) and np.all(np.abs(s.astype(np.float64) - os_) <= near)


def test_unscaled_table_is_the_plain_one():
    pos = np.arange(-300, 300, 7)
    for scaling in (None, kvb.rope_scaling(kvb.KVB_ROPE_NONE), kvb.rope_scaling(kvb.KVB_ROPE_LINEAR, factor=1.0)):
        a, b = kvb.kvb_rope_scaled_table(1e6, 128, scaling, pos), kvb.kvb_rope_delta_table(1e6, 128, pos)
        assert np.array_equal(a[0], b[0]) and np.array_equal(a[1], b[1])
    c, s = kvb.kvb_rope_scaled_table(1e4, 64, None, [])
    assert c.shape == (0, 32)


def test_scaling_keeps_fast_pairs_and_stretches_slow_ones():
    for kind in (od.PARTS, od.INDEX):
        w = od.frequencies(1e4, 128, kind, factor=8.0, original_len=4096, low=1.0, high=32.0)
        plain = od.frequencies(1e4, 128)
        assert np.allclose(w[:10], plain[:10]) and np.allclose(w[-10:], plain[-10:] / 8)
        assert np.all(np.diff(w) < 0)


@pytest.mark.parametrize("theta,rot,over", [
    (0.0, 64, {}), (float("nan"), 64, {}), (float("inf"), 64, {}), (1e4, 63, {}), (1e4, 0, {}),
    (1e4, 64, dict(kind=5)), (1e4, 64, dict(kind=-1)), (1e4, 64, dict(kind=1, factor=0.5)),
    (1e4, 64, dict(kind=1, factor=float("nan"))), (1e4, 2, dict(kind=2, factor=2.0)),
    (1e4, 64, dict(kind=3, factor=2.0, original_len=0.0)), (1e4, 64, dict(kind=3, factor=2.0, low=4.0, high=4.0)),
    (1e4, 64, dict(kind=4, factor=2.0, low=0.0)), (1.0, 64, dict(kind=4, factor=2.0)),
    (1e4, 64, dict(kind=0, attn_factor=0.0))])
def test_table_rejects(theta, rot, over):
    sc = kvb.rope_scaling(**over) if over else None
    assert _status(lambda: kvb.kvb_rope_scaled_table(theta, rot, sc, [1, 2])) == EINVAL


# ---- norms and rotation ---------------------------------------------------------

def _norm_rope(**over):
    a = dict(n_tokens=4, n_q_heads=4, n_kv_heads=2, head_dim=64, dtype=kvb.KVB_BF16, q=FAKE, q_token_stride=512,
             q_head_stride=64, k=FAKE, k_token_stride=512, k_head_stride=64, q_weight=FAKE, k_weight=FAKE, eps=1e-6,
             pos=FAKE, table_cos=FAKE, table_sin=FAKE, table_len=10, rot_dim=64, pairing=0, q_out=FAKE,
             q_out_token_stride=256, q_out_head_stride=64, k_out=FAKE, k_out_token_stride=64, k_out_head_stride=256,
             stream=0)
    a.update(over)
    kvb.kvb_qk_norm_rope(**a)


@pytest.mark.parametrize("over,status", [
    (dict(n_tokens=0), EINVAL), (dict(n_tokens=2 ** 31), EINVAL), (dict(n_tokens=2 ** 29), EINVAL),
    (dict(n_q_heads=0, n_kv_heads=0), EINVAL), (dict(n_kv_heads=-1), EINVAL), (dict(head_dim=0), EINVAL),
    (dict(head_dim=60, rot_dim=32), EUNSUPPORTED), (dict(head_dim=264), EUNSUPPORTED), (dict(rot_dim=12), EUNSUPPORTED),
    (dict(rot_dim=72), EINVAL), (dict(rot_dim=-8), EINVAL), (dict(dtype=kvb.KVB_F64), EINVAL), (dict(pairing=2), EINVAL),
    (dict(eps=-1.0), EINVAL), (dict(eps=float("nan")), EINVAL), (dict(q=None), EINVAL), (dict(q_out=None), EINVAL),
    (dict(k=None), EINVAL), (dict(k_out=FAKE + 8), EINVAL), (dict(q=FAKE + 2), EINVAL), (dict(q_weight=FAKE + 4), EINVAL),
    (dict(q_token_stride=516), EINVAL), (dict(k_out_head_stride=-64), EINVAL), (dict(pos=None), EINVAL),
    (dict(table_cos=None), EINVAL), (dict(table_sin=FAKE + 4), EINVAL), (dict(table_len=0), EINVAL)])
def test_norm_rope_rejects(over, status):
    assert _status(_norm_rope, **over) == status


@pytest.mark.parametrize("tokens,heads", [(2 ** 26 - 3, (1, 0)), (2 ** 26 - 3, (0, 1)), (2 ** 25 - 1, (1, 1))])
def test_norm_rope_takes_at_most_2_to_26_less_4_heads(tokens, heads):
    assert _status(_norm_rope, n_tokens=tokens, n_q_heads=heads[0], n_kv_heads=heads[1]) == EINVAL
    if NO_GPU:  # what fits passes every check
        assert _status(_norm_rope, n_tokens=tokens - 1, n_q_heads=heads[0], n_kv_heads=heads[1]) == kvb.KVB_EHIP


# ---- the 8-bit cache --------------------------------------------------------------

def _layout(**over):
    a = dict(n_blocks=8, n_kv_heads=2, head_dim=128, block_len=32, code=kvb.KVB_I8, max_blocks=4)
    a.update(over)
    return kvb.cache8_layout(**a)


ARRAYS = dict(table=FAKE, lens=FAKE, k_codes=FAKE, k_scale=FAKE, v_codes=FAKE, v_scale=FAKE, k_tail=FAKE, v_tail=FAKE)


def _append(**over):
    a = dict(ARRAYS, layout=_layout(), n_layers=1, n_seqs=1, cu_new=FAKE, max_new=1, k=FAKE, v=FAKE, layer_stride=0,
             token_stride=256, head_stride=128, stream=0)
    a.update(over)
    kvb.kvb_cache8_append(**a)


def _read(**over):
    a = dict(ARRAYS, layout=_layout(), n_layers=1, n_seqs=1, cu_out=FAKE, max_out=1, out_dtype=kvb.KVB_F32, k_out=FAKE,
             v_out=FAKE, layer_stride=0, token_stride=256, head_stride=128, stream=0)
    a.update(over)
    kvb.kvb_cache8_read(**a)


def _attn(**over):
    a = dict(ARRAYS, layout=_layout(), n_q_heads=16, n_seqs=1, cu_q=FAKE, n_queries=1, max_queries=1, max_len=100, q=FAKE,
             softmax_scale=0.1, out=FAKE, lse=None, weights_in=None, weights_out=None, workspace=FAKE,
             workspace_bytes=1 << 30, stream=0)
    a.update(over)
    kvb.kvb_cache8_attn(**a)


def _evict(**over):
    a = dict(layout=_layout(), n_layers=1, n_seqs=1, budget=2, n_first=1, n_recent=1, table=FAKE, lens=FAKE, weights=FAKE,
             table_out=2 * FAKE, lens_out=2 * FAKE, weights_out=2 * FAKE, stream=0)
    a.update(over)
    kvb.kvb_cache8_evict(**a)


BAD_LAYOUTS = [
    (dict(n_blocks=0), EINVAL), (dict(n_kv_heads=0), EINVAL), (dict(max_blocks=0), EINVAL), (dict(head_dim=96), EUNSUPPORTED),
    (dict(head_dim=-1), EINVAL), (dict(block_len=24), EUNSUPPORTED), (dict(block_len=256), EUNSUPPORTED),
    (dict(block_len=0), EINVAL), (dict(code=2), EINVAL), (dict(code=-1), EINVAL)]


@pytest.mark.parametrize("call", [_append, _read, _attn])
@pytest.mark.parametrize("over,status", BAD_LAYOUTS)
def test_layout_rejects(call, over, status):
    assert _status(call, layout=_layout(**over)) == status


COMMON = [(dict(n_seqs=0), EINVAL), (dict(n_seqs=2 ** 24), EINVAL), *((dict([(k, None)]), EINVAL) for k in ARRAYS),
          (dict(k_codes=FAKE + 8), EINVAL), (dict(v_scale=FAKE + 4), EINVAL), (dict(v_tail=FAKE + 2), EINVAL)]


@pytest.mark.parametrize("over,status", COMMON + [
    (dict(n_layers=0), EINVAL), (dict(n_layers=2 ** 21), EINVAL), (dict(cu_new=None), EINVAL), (dict(max_new=0), EINVAL),
    (dict(k=None), EINVAL), (dict(v=FAKE + 4), EINVAL), (dict(token_stride=4), EINVAL), (dict(head_stride=-8), EINVAL)])
def test_append_rejects(over, status):
    assert _status(_append, **over) == status


@pytest.mark.parametrize("over,status", COMMON + [
    (dict(cu_out=None), EINVAL), (dict(max_out=-1), EINVAL), (dict(k_out=None), EINVAL), (dict(v_out=FAKE + 4), EINVAL),
    (dict(out_dtype=kvb.KVB_F64), EINVAL), (dict(layer_stride=12), EINVAL)])
def test_read_rejects(over, status):
    assert _status(_read, **over) == status


@pytest.mark.parametrize("over,status", COMMON + [
    (dict(n_q_heads=15), EINVAL), (dict(n_q_heads=0), EINVAL), (dict(cu_q=None), EINVAL), (dict(n_queries=0), EINVAL),
    (dict(max_queries=0), EINVAL), (dict(max_queries=2 ** 20), EINVAL), (dict(max_len=0), EINVAL), (dict(q=None), EINVAL),
    (dict(out=FAKE + 2), EINVAL), (dict(weights_in=FAKE), EINVAL), (dict(softmax_scale=float("inf")), EINVAL),
    (dict(n_seqs=40000), EINVAL), (dict(max_len=1 << 20, workspace_bytes=16), EINVAL),
    (dict(max_len=1 << 20, workspace=None), EINVAL), (dict(weights_out=FAKE, workspace_bytes=0), EINVAL)])
def test_attn_rejects(over, status):
    assert _status(_attn, **over) == status


@pytest.mark.parametrize("over,status", [
    (dict(n_layers=0), EINVAL), (dict(n_seqs=0), EINVAL), (dict(budget=1), EINVAL), (dict(budget=-1, n_first=0, n_recent=0), EINVAL),
    (dict(n_first=-1), EINVAL), (dict(n_recent=-1), EINVAL), (dict(n_first=2 ** 31 - 1, n_recent=2 ** 31 - 1), EINVAL),
    (dict(table=None), EINVAL), (dict(lens=None), EINVAL), (dict(weights=None), EINVAL), (dict(table_out=None), EINVAL),
    (dict(lens_out=None), EINVAL), (dict(weights_out=None), EINVAL), (dict(table_out=FAKE), EINVAL),
    (dict(lens_out=FAKE), EINVAL), (dict(weights_out=FAKE), EINVAL), (dict(layout=_layout(max_blocks=0)), EINVAL),
    (dict(layout=_layout(block_len=0)), EINVAL), (dict(layout=_layout(n_kv_heads=-2)), EINVAL)])
def test_evict_rejects(over, status):
    assert _status(_evict, **over) == status


@pytest.mark.parametrize("out", ["table_out", "lens_out", "weights_out"])
@pytest.mark.parametrize("into", ["table", "lens", "weights"])
def test_evict_rejects_every_input_as_an_output(out, into):
    apart = dict(table=FAKE, lens=2 * FAKE, weights=3 * FAKE, table_out=4 * FAKE, lens_out=5 * FAKE, weights_out=6 * FAKE)
    assert _status(_evict, **{**apart, out: apart[into]}) == EINVAL


@pytest.mark.parametrize("what", [b"\0" * 16, "0123456789abcdef", bytearray(16), 1.0, [1, 2], object()],
                         ids=["bytes", "str", "bytearray", "float", "list", "object"])
def test_what_is_no_array_is_refused(what):
    """Neither the text's bytes nor the object's own memory become an address."""
    for call, name in ((_norm_rope, "q"), (_norm_rope, "pos"), (_append, "lens"), (_append, "k"), (_read, "k_out"),
                       (_attn, "workspace"), (_attn, "table"), (_evict, "weights")):
        with pytest.raises(AttributeError):
            call(**{name: what})
    with pytest.raises(AttributeError):  # an entry point of the prompt's path
        kvb.kvb_deviation(1, 1, 64, 1, what, FAKE, FAKE, FAKE, 0, FAKE, stream=0)


@pytest.mark.skipif(not NO_GPU, reason="would launch")
def test_addresses_and_host_arrays_are_taken():
    for what in (FAKE, True * FAKE, np.zeros(16, np.float32)):
        with pytest.raises(kvb.KvbError):
            _norm_rope(pos=what)


def test_attn_workspace_is_pure():
    lay = _layout(max_blocks=4096, n_blocks=100000)
    f = kvb.kvb_cache8_attn_workspace_bytes
    assert f(lay, 16, 1, 1, 1, 100000, 0) == f(lay, 16, 1, 1, 1, 100000, 0) > 0
    assert f(lay, 16, 1, 1, 1, 100000, 1) > f(lay, 16, 1, 1, 1, 100000, 0)
    assert f(lay, 15, 1, 1, 1, 100, 0) == 0 and f(_layout(head_dim=96), 16, 1, 1, 1, 100, 0) == 0


def test_without_a_device_the_status_says_so():
    if not NO_GPU:
        pytest.skip("would launch")
    for call in (_norm_rope, _append, _read, _attn, _evict):
        assert _status(call) == kvb.KVB_EHIP
