"""What the binding refuses before a kernel would read or write past a tensor, or an
address of another device: views of one call on several devices or on the host, an lse
or a workspace that is too small, of another type or not contiguous. Without a GPU: the
device of a view is what the binding knows of it, set here by hand."""
import ctypes

import pytest

from test_prompt_host import H, cfg_of  # noqa: F401 (H: fixture)

torch = pytest.importorskip("torch")


@pytest.fixture
def launched(H, monkeypatch):
    """Calls that reach the library, instead of the library."""
    calls, library = [], H.lib()

    class Fake:
        def __getattr__(self, name):
            if name == "hkv_status_str":
                return library.hkv_status_str

            def call(*args):
                calls.append(name)
                return 0
            return call
    monkeypatch.setattr(H, "_lib", Fake())
    return calls


def refused(H, f, *args, status, **kw):
    with pytest.raises(H.HkvError) as e:
        f(*args, **kw)
    assert e.value.status == status


def parts(H):
    x = torch.zeros(3, 5, 6, 64, dtype=torch.bfloat16)
    k = torch.zeros(3, 6, 9, 64, dtype=torch.bfloat16)
    pos, length = torch.zeros(1, 3, 5, dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    v = {"x": H.make_rows(x), "out": H.make_rows(x.clone()), "tokens": H.make_tokens(5, length, pos),
         "states": H.make_states(k, k.clone()), "norm": H.make_norm(H.HKV_NORM_RMS, 1e-5, x[0, 0, 0].clone())}
    for y in v.values():
        assert y.on == -1
        y.on = 0    # as if they lay on the first GPU
    return v


def calls(H, v, rope, **kw):
    cfg = cfg_of(H)
    return {
        "rotate": lambda: H.hkv_rope_rotate(cfg, rope, v["tokens"], v["x"], v["out"]),
        "prepare": lambda: H.hkv_qk_norm_rope(cfg, v["norm"], rope, v["tokens"], v["x"], None, v["x"], v["out"], None,
                                              v["out"]),
        "cross": lambda: H.hkv_cross_attention(cfg, v["states"], v["tokens"], v["x"], v["out"],
                                               kw.get("lse"), kw.get("ws", 256), kw.get("n", 0)),
    }


USES = {"rotate": ("x", "out", "tokens"), "prepare": ("x", "out", "tokens", "norm"),
        "cross": ("x", "out", "tokens", "states")}


@pytest.mark.parametrize("name", list(USES))
def test_views_of_several_devices_are_refused(H, launched, name):
    rope = H.hkv_rope(64, 64, H.HKV_ROPE_HALF, 1, (ctypes.c_int32 * 3)(32, 0, 0), 1.0)
    calls(H, parts(H), rope)[name]()
    assert len(launched) == 1
    for which in USES[name]:
        for other in (1, -1):
            v = parts(H)
            v[which].on = other
            refused(H, calls(H, v, rope)[name], status=H.HKV_ERR_INVALID_ARG)
    # all on the host
    v = parts(H)
    for y in v.values():
        y.on = -1
    refused(H, calls(H, v, rope)[name], status=H.HKV_ERR_INVALID_ARG)
    # what is given by address alone is not known
    for which in USES[name]:
        v = parts(H)
        for y in v.values():
            y.on = None
        v[which].on = 2
        calls(H, v, rope)[name]()
    assert len(launched) == 1 + len(USES[name])


def test_views_know_their_device(H):
    meta = torch.zeros(3, 5, 6, 64, device="meta", dtype=torch.bfloat16)
    host = torch.zeros(3, 5, 6, 64, dtype=torch.bfloat16)
    pos, length = torch.zeros(1, 3, 5, dtype=torch.int32), torch.zeros(3, dtype=torch.int32, device="meta")
    refused(H, H.make_tokens, 5, length, pos, status=H.HKV_ERR_INVALID_ARG)
    refused(H, H.make_tokens, 5, None, pos, length[:1], status=H.HKV_ERR_INVALID_ARG)   # an error word elsewhere
    refused(H, H.make_states, host, meta, status=H.HKV_ERR_INVALID_ARG)
    refused(H, H.make_states, host, host, None, length[:1], status=H.HKV_ERR_INVALID_ARG)
    refused(H, H.make_norm, 1, 1e-5, host[0, 0, 0], meta[0, 0, 0], status=H.HKV_ERR_INVALID_ARG)
    assert H.make_tokens(5).on is None and H.make_norm(1, 1e-5).on is None
    assert H.make_tokens(5, None, None, 4096).on is None      # an error word by its address
    assert H.make_tokens(5, None, pos).on == -1 and H.make_norm(1, 1e-5, host[0, 0, 0]).on == -1


def test_lse_and_workspace_of_another_size_or_type(H, launched):
    v = parts(H)
    S, T, heads = 3, 5, 6

    def run(**kw):
        calls(H, v, None, **kw)["cross"]()

    def at(x, device=0):
        """x as a tensor of that device, as far as the binding asks."""
        class On:
            def __getattr__(self, name):
                return getattr(x, name)

            def get_device(self):
                return device
        return On()
    whole = torch.zeros(S, heads, T)
    for lse in (None, 4096, at(whole), at(whole.view(-1)), at(torch.zeros(S * heads * T + 7))):
        run(lse=lse)
    assert len(launched) == 5
    for bad in (torch.zeros(S, heads, T - 1), torch.zeros(S, heads, T, dtype=torch.float64),
                torch.zeros(S, heads, T, dtype=torch.bfloat16), torch.zeros(S, heads, T, dtype=torch.int32),
                torch.zeros(S, T, heads).transpose(1, 2), torch.zeros(S, heads, 2 * T)[..., ::2]):
        refused(H, run, lse=at(bad), status=H.HKV_ERR_SHAPE)
    for device in (1, -1):
        refused(H, run, lse=at(whole, device), status=H.HKV_ERR_INVALID_ARG)
        refused(H, run, ws=at(torch.zeros(512), device), n=256, status=H.HKV_ERR_INVALID_ARG)
    run(ws=at(torch.zeros(64)), n=256)
    run(ws=at(torch.zeros(256, dtype=torch.uint8)), n=256)
    run(ws=4096, n=1 << 40)
    refused(H, run, ws=at(torch.zeros(63)), n=256, status=H.HKV_ERR_CAPACITY)
    refused(H, run, ws=at(torch.zeros(255, dtype=torch.uint8)), n=256, status=H.HKV_ERR_CAPACITY)
    assert len(launched) == 8
