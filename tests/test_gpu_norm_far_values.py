"""Group norm with an activation where a group's first value lies far from all others (a padded image's corner), over
sequences whose groups no workgroup holds; against 64 bits."""
import pytest
import torch

import encoder_ref as R

pytestmark = pytest.mark.gpu


# B, S, C, T, groups: several chunks; groups across blocks of columns, whole vectors and single elements
@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("B,S,C,T,G", [(1, 21000, 8, 2, 2), (2, 6000, 320, 4, 2), (1, 3000, 515, 1, 5), (3, 5003, 6, 4, 1)])
def test_first_value_far_from_the_others(B, S, C, T, G, dt):
    from paper_2607_21271_amd.norm import group_norm_act
    d = R.DT[dt]
    g = torch.Generator().manual_seed(71)
    far = 1000.0 if dt == "f32" else 30.0
    x = (torch.randn(B, S, C, T, generator=g) + far).to(d).cuda()
    x[:, 0, 0, 0] = 0.0
    w, b = ((torch.randn(C, generator=g) * 0.3 + s).to(d).cuda().requires_grad_() for s in (1.0, 0.0))
    dy = torch.randn(B, S, C, T, generator=g).to(d).cuda()
    x.requires_grad_()
    y = group_norm_act(x, w, b, G, "none", eps=1e-5)
    dx, dw, db = torch.autograd.grad(y, (x, w, b), dy)

    x6, w6, b6, g6 = (t.detach().double().cpu() for t in (x, w, b, dy))
    w6, b6 = w6[:, None], b6[:, None]
    grp = x6.view(B, S, G, -1)
    mean = grp.mean((1, 3), keepdim=True)
    rstd = 1.0 / torch.sqrt((grp - mean).pow(2).mean((1, 3), keepdim=True) + 1e-5)
    xh = ((grp - mean) * rstd).view_as(x6)
    z = xh * w6 + b6
    # E32: relative error of the variance's sums and of products; the mean is a few roundings (eight) off in fp32
    u, off = R.U[d], 2.0 ** -21 * (mean.abs() * rstd).expand_as(grp).reshape(x6.shape)
    exh = R.E32 * (1.0 + xh.abs()) + off
    R.within("y", y, z, u * z.abs() + exh * w6.abs() + R.E32 * z.abs() + R.TINY[d])
    gw = (g6 * w6)
    each = lambda t: t.view(B, S, G, -1).mean((1, 3), keepdim=True).expand_as(grp).reshape(x6.shape)
    rs = rstd.expand_as(grp).reshape(x6.shape)
    want = rs * (gw - each(gw) - xh * each(gw * xh))
    ex = rs * (R.E32 * gw.abs() + R.E32 * each(gw.abs()) + exh * each((gw * xh).abs()) + xh.abs() * each(gw.abs() * (exh + R.E32 * xh.abs())))
    R.within("dx", dx, want, u * want.abs() + ex + R.E32 * want.abs() + R.TINY[d])
    sums = lambda t: t.sum((0, 1, 3))
    R.within("dw", dw, sums(g6 * xh), u * sums(g6 * xh).abs() + sums(g6.abs() * (exh + R.E32 * xh.abs())) + R.TINY[d])
    R.within("db", db, sums(g6), u * sums(g6).abs() + R.E32 * sums(g6.abs()) + R.TINY[d])
