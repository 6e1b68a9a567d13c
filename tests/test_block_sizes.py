"""CPU-only: sizes that a call takes as 32-bit numbers are refused by the binding if they do not fit, instead of losing their upper bits."""
import ctypes
from types import SimpleNamespace

import pytest
import torch

from paper_2002_06015_amd import kfac, workloads as wl

F32, I32, U8, E4M3 = torch.float32, torch.int32, torch.uint8, torch.float8_e4m3fn
BIG = (1 << 32) + 8                                                 # 8, if it lost them


def new(*shape, dtype=F32):
    return torch.empty(*shape, dtype=dtype, device="meta")          # sizes without memory; the address is 0


@pytest.fixture()
def ctx(monkeypatch):
    handle = ctypes.c_void_p()
    assert kfac.lib().kfac_create(ctypes.addressof(handle), None, ctypes.c_void_p(0x100000), 256) == kfac.KFAC_OK
    monkeypatch.setattr(kfac, "_device", lambda c: new(1).get_device())
    monkeypatch.setattr(kfac, "_ids", lambda t, what: 32)
    yield SimpleNamespace(handle=handle)
    kfac.lib().kfac_destroy(handle)


def _calls(ctx, n, dim, fan):
    """Every call with n rows, rows of dim elements, tokens of fan choices; the pointers are NULL, so that none of them gets to the GPU."""
    r, layer = kfac.router(1, 1), wl.fc_layer(1, 64, 32, 0)
    order, offsets, flat = new(n, dtype=I32), new(5, dtype=I32), new(n)
    wide, row = new(n, dim), new(dim)
    return {
        "route": lambda: kfac.kfac_route(ctx, r, new(n, 1), order, flat),
        "route_grad": lambda: kfac.kfac_route_grad(ctx, r, new(n, 1), order, flat, new(n, 1)),
        "combine": lambda: kfac.kfac_combine(ctx, wide, flat, wide),
        "combine_grad": lambda: kfac.kfac_combine_grad(ctx, wide, flat, wide, wide, flat),
        "combine_grad_gate": lambda: kfac.kfac_combine_grad(ctx, wide, None, wide, None, flat),
        "keep": lambda: kfac.kfac_keep(ctx, new(2, dim), new(2, dim, dtype=E4M3), new(2, (dim + 31) // 32, dtype=U8)),
        "restore": lambda: kfac.kfac_restore(ctx, new(2, dim, dtype=E4M3), new(2, (dim + 31) // 32, dtype=U8), new(2, dim)),
        "norm": lambda: kfac.kfac_rms_norm(ctx, wide, row, 1e-5, wide),
        "norm_grad": lambda: kfac.kfac_rms_norm_grad(ctx, wide, wide, row, 1e-5, wide),
        "weight": lambda: kfac.kfac_expert_grad_weight_kept(ctx, layer, order, offsets, new(n // fan, 64, dtype=E4M3), new(n // fan, 2, dtype=U8), new(n, 32),
                                                            new(4, 32, 64), fan=fan),
        "stats": lambda: kfac.kfac_stats_expert_kept(ctx, layer, order, offsets, new(n // fan, 64, dtype=E4M3), new(n // fan, 2, dtype=U8), new(n, 32), 0.0,
                                                     new(4, 64, 64), new(4, 32, 32), fan=fan),
    }


NAMES = ["route", "route_grad", "combine", "combine_grad", "combine_grad_gate", "keep", "restore", "norm", "norm_grad", "weight", "stats"]


@pytest.mark.parametrize("name", [n for n in NAMES if n not in ("keep", "restore")])
def test_rows(ctx, name):
    with pytest.raises(kfac.KfacError):                             # the call itself is one that only its NULL pointers spoil
        _calls(ctx, 8, 16, 1)[name]()
    with pytest.raises(ValueError):
        _calls(ctx, BIG, 16, 1)[name]()


@pytest.mark.parametrize("name", [n for n in NAMES if n not in ("route", "route_grad", "weight", "stats")])
def test_columns(ctx, name):
    with pytest.raises(kfac.KfacError):
        _calls(ctx, 8, 8, 1)[name]()
    with pytest.raises(ValueError):
        _calls(ctx, 8, BIG, 1)[name]()


@pytest.mark.parametrize("name", ["weight", "stats"])
def test_choices_of_a_token(ctx, name):
    with pytest.raises(kfac.KfacError):
        _calls(ctx, 8, 8, 2)[name]()
    with pytest.raises(ValueError):
        _calls(ctx, 8, 8, (1 << 32) + 2)[name]()
