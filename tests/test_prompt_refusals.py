"""The entry points of prompts and drafted tokens refuse wrong arguments on the host, before anything
is launched (no GPU is needed), and the tensor helpers refuse wrong tensors."""
import math
import os

import pytest

import paper_2509_26436_amd as q

OK, ENULL, ESHAPE, EUNSUP, EALIGN, EWS = 0, 1, 2, 3, 4, 6
A = 4096      # a fake, 16-byte aligned address: never dereferenced on these paths


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not os.path.exists(q.library_path()):
        pytest.skip("libquartz.so not built")
    return q.load()


def test_head_norm_rotary():
    def call(x=A, xo=1 << 20, H=4, xt=512, xh=128, xot=512, xoh=128, xw=A, k=A, ko=1 << 21, KV=2, kt=256, kh=128, kot=256,
             koh=128, kw=A, T=4, d=128, rot=128, p=A, axes=1, step=4, axis=None, f=A, layout=0, norm=1, eps=1e-6, magnitude=1.0):
        return q.quartz_head_norm_rotary(x, xo, H, xt, xh, xot, xoh, xw, k, ko, KV, kt, kh, kot, koh, kw, T, d, rot, p, axes,
                                         step, axis, f, layout, norm, eps, magnitude, None)
    assert call(layout=2) == call(eps=-1.0) == call(eps=math.nan) == call(eps=math.inf) == call(magnitude=math.inf) == EUNSUP
    assert call(norm=0) == EUNSUP                               # weights without a norm
    assert call(T=-1) == call(H=-1) == call(KV=-1) == call(d=127) == call(d=514) == call(d=0, rot=0) == ESHAPE
    assert call(rot=130) == call(rot=3) == call(rot=-2) == call(axes=0) == call(T=1 << 24) == ESHAPE
    assert call(xt=1 << 41) == call(koh=-(1 << 41)) == call(step=1 << 41) == ESHAPE
    assert call(x=None) == call(xo=None) == call(k=None) == call(ko=None) == call(p=None) == call(f=None) == ENULL
    assert call(x=A + 1) == call(ko=(1 << 21) + 1) == call(xw=A + 1) == call(p=A + 2) == call(axis=A + 2) == call(f=A + 4) == EALIGN
    assert call(xo=A, xot=640) == call(k=A, ko=A, koh=64) == ESHAPE       # in place with other strides
    assert call(T=0, x=None) == call(H=0, KV=0, x=None, k=None) == OK


CACHE = dict(kc=A, vc=A, type=0, ks=1.0, vs=1.0, pages=4, page=16, stride=16 * 2 * 128, table=A)


def _sizes(T, S, H, kv, d, page, width):
    return q.quartz_paged_prompt_workspace_bytes(T, S, H, kv, d, page, width)


def _prompt(x=A, o=A, T=9, S=3, H=8, kv=2, d=128, qt=1024, qh=128, ot=1024, oh=128, starts=A, lengths=A, scale=0.1, window=0,
            cap=0.0, slopes=None, prefix=None, width=4, row=4, work=A, size=1 << 40, **over):
    c = dict(CACHE, **over)
    return q.quartz_paged_prompt_attention(x, o, T, S, H, kv, d, qt, qh, ot, oh, c["kc"], c["vc"], c["type"], c["ks"], c["vs"],
                                           c["pages"], c["page"], c["stride"], c["table"], width, row, starts, lengths, scale,
                                           window, cap, slopes, prefix, work, size, None)


def _tree(x=A, o=A, T=9, S=3, H=8, kv=2, d=128, qt=1024, qh=128, ot=1024, oh=128, starts=A, lengths=A, tree=A, words=1,
          step=1, scale=0.1, cap=0.0, width=4, row=4, work=A, size=1 << 40, **over):
    c = dict(CACHE, **over)
    return q.quartz_paged_tree_attention(x, o, T, S, H, kv, d, qt, qh, ot, oh, c["kc"], c["vc"], c["type"], c["ks"], c["vs"],
                                         c["pages"], c["page"], c["stride"], c["table"], width, row, starts, lengths, tree,
                                         words, step, scale, cap, work, size, None)


def _keep(first=A, kept=A, S=3, most=4, step=4, kv=2, d=128, width=4, row=4, **over):
    c = dict(CACHE, **over)
    return q.quartz_paged_keep(first, kept, S, most, step, c["kc"], c["vc"], c["type"], kv, d, c["pages"], c["page"],
                               c["stride"], c["table"], width, row, None)


@pytest.mark.parametrize("call", [_prompt, _tree, _keep])
def test_cache(call):
    assert call(type=2) == call(page=12) == call(page=4) == call(page=8192) == call(page=0) == call(page=1 << 62) == EUNSUP
    assert call(pages=0) == call(pages=1 << 31) == call(stride=16 * 2 * 128 - 8) == ESHAPE
    assert call(row=3) == call(width=-1) == call(width=1 << 27, row=1 << 27) == call(width=-(1 << 33)) == ESHAPE
    assert call(kc=None) == call(vc=None) == call(table=None) == ENULL
    assert call(kc=A + 8) == call(vc=A + 2) == call(table=A + 2) == call(stride=16 * 2 * 128 + 4) == EALIGN
    assert call(type=1, stride=16 * 2 * 128 + 8) == EALIGN
    assert call(d=96) == EUNSUP


@pytest.mark.parametrize("call", [_prompt, _tree])
def test_attention(call):
    assert call(ks=0.0) == call(vs=-1.0) == call(ks=math.nan) == call(vs=math.inf) == call(vs=1e-37) == EUNSUP
    assert call(scale=math.nan) == call(scale=math.inf) == call(scale=1e-38, ks=0.01) == call(scale=-3e38, ks=100.0) == EUNSUP
    assert call(cap=-1.0) == call(cap=math.nan) == call(cap=math.inf) == call(cap=2000.0) == call(cap=1e-4) == EUNSUP
    assert call(T=-1) == call(S=-1) == call(kv=3) == call(kv=0) == call(H=1) == call(T=1 << 28) == call(S=1 << 24) == ESHAPE
    assert call(qt=1 << 41) == call(oh=-(1 << 41)) == ESHAPE
    assert call(x=None) == call(o=None) == call(starts=None) == call(lengths=None) == ENULL
    assert call(x=A + 8) == call(o=A + 4) == call(starts=A + 2) == call(lengths=A + 2) == call(work=A + 8) == EALIGN
    assert call(qt=1028) == call(qh=132) == call(ot=1026) == call(oh=126) == EALIGN
    need = _sizes(9, 3, 8, 2, 128, 16, 4096)
    assert need > 0
    long = dict(width=4096, row=4096)
    assert call(**long, work=None) == call(**long, size=need - 1) == call(**long, size=0) == EWS
    assert call(T=0, x=None, o=None, kc=None) == call(S=0, x=None, o=None, kc=None) == OK
    for bad in ((9, 3, 8, 3, 128, 16, 4), (9, 3, 8, 2, 96, 16, 4), (9, 3, 8, 2, 128, 12, 4), (-1, 3, 8, 2, 128, 16, 4),
                (9, -3, 8, 2, 128, 16, 4), (9, 3, 8, 2, 128, 16, 1 << 40), (0, 3, 8, 2, 128, 16, 4096), (9, 0, 8, 2, 128, 16, 4096)):
        assert _sizes(*bad) == 0


def test_what_only_one_of_them_takes():
    assert _prompt(window=-1) == ESHAPE
    assert _prompt(slopes=A + 2) == _prompt(prefix=A + 2) == EALIGN
    assert _tree(words=0) == _tree(words=-1) == _tree(step=1 << 41) == ESHAPE
    assert _tree(tree=None) == ENULL
    assert _tree(tree=A + 4) == EALIGN
    assert _keep(S=-1) == _keep(most=-1) == _keep(step=3) == _keep(kv=0) == _keep(S=1 << 24) == _keep(most=1 << 31, step=1 << 31) == ESHAPE
    assert _keep(first=None) == _keep(kept=None) == ENULL
    assert _keep(first=A + 2) == _keep(kept=A + 1) == EALIGN
    assert _keep(S=0, kc=None) == _keep(most=0, step=0, kc=None) == _keep(width=0, row=0, table=None) == OK


def _tensors():
    import torch
    k = torch.zeros((3, 2, 16, 128), dtype=torch.bfloat16)
    cache = q.PagedCache(k, k.clone(), torch.zeros((2, 2), dtype=torch.int32))
    x = torch.zeros((5, 4, 128), dtype=torch.bfloat16)
    i32 = lambda n: torch.zeros(n, dtype=torch.int32)          # noqa: E731
    return torch, k, cache, x, i32


def test_helpers_refuse_tensors():
    torch, k, cache, x, i32 = _tensors()
    starts, lengths, tree, f = i32(3), i32(2), torch.zeros((5, 1), dtype=torch.int64), q.rotary_frequencies(128, device="cpu")
    w, p, kept = x[0, 0].clone(), i32(5), torch.zeros((2, 3), dtype=torch.int32)
    prompt = lambda **kw: q.paged_prompt_attention(**{**dict(q=x, cache=cache, starts=starts, lengths=lengths), **kw})     # noqa: E731
    trees = lambda **kw: q.paged_tree_attention(**{**dict(q=x, cache=cache, starts=starts, lengths=lengths, tree=tree), **kw})   # noqa: E731
    heads = lambda **kw: q.head_norm_rotary(**{**dict(q=x, k=x.clone(), positions=p, freqs=f, q_weight=w, k_weight=w), **kw})    # noqa: E731
    wrong = []
    for call in (prompt, trees):
        wrong += [lambda call=call, kw=kw: call(**kw) for kw in (
            dict(q=x.float()), dict(q=x[..., :64]), dict(q=x[:, :3]), dict(q=x[..., ::2]), dict(starts=i32(2)),
            dict(starts=starts.long()), dict(lengths=i32(3)), dict(lengths=lengths.float()), dict(out=x[:4]),
            dict(out=torch.zeros_like(x).float()), dict(workspace=torch.zeros(64, dtype=torch.uint8)[::2]), dict())]
    wrong += [lambda kw=kw: prompt(**kw) for kw in (dict(slopes=torch.zeros(3)), dict(slopes=torch.zeros(4).double()),
                                                    dict(prefix=i32(3)), dict(prefix=torch.zeros(2)))]
    wrong += [lambda kw=kw: trees(**kw) for kw in (dict(tree=tree[:4]), dict(tree=tree.int()), dict(tree=tree[:, :0]), dict(tree=tree[:, 0]), dict(tree=None))]
    wrong += [lambda kw=kw: heads(**kw) for kw in (
        dict(q=x.float()), dict(k=x[:4]), dict(k=x[..., :64]), dict(positions=p.long()), dict(positions=i32(4)),
        dict(positions=i32(10).view(5, 2)), dict(freqs=f.double()), dict(freqs=torch.cat([f, f])), dict(q_weight=w[:64]),
        dict(k_weight=w.float()), dict(axes=i32(63)), dict(axes=f), dict(layout="both"), dict(eps=None), dict(k=None),
        dict(out=(x[:4], None)), dict(positions=torch.zeros((0, 5), dtype=torch.int32)), dict())]
    wrong += [lambda: q.paged_keep(cache, i32(3), kept), lambda: q.paged_keep(cache, lengths, kept[:1]),
              lambda: q.paged_keep(cache, lengths, kept.long()), lambda: q.paged_keep(cache, lengths, kept[:, ::2]),
              lambda: q.paged_keep(q.PagedCache(k, k, cache.table), lengths, kept), lambda: q.paged_keep(cache, lengths, kept)]
    for i, call in enumerate(wrong):
        print("refused?", i)
        with pytest.raises(ValueError):
            call()


def test_helpers_refuse_shared_memory():
    torch, k, cache, x, i32 = _tensors()
    starts, lengths, f, p = i32(3), i32(2), q.rotary_frequencies(128, device="cpu"), i32(5)
    keys = k.view(-1)
    wrong = [
        (lambda: q.paged_prompt_attention(x, cache, starts, lengths, out=x), "share"),
        (lambda: q.paged_prompt_attention(x, cache, starts, lengths, out=keys[:5 * 512].view(5, 4, 128)), "share"),
        (lambda: q.paged_prompt_attention(x, cache, starts, lengths, out=x[:1].clone().expand(5, 4, 128)), "twice"),
        (lambda: q.paged_prompt_attention(x, cache, starts, lengths, workspace=keys.view(torch.uint8)), "share"),
        (lambda: q.paged_tree_attention(x, cache, starts, lengths, x.view(-1)[:20].view(torch.int64).view(5, 1), out=x), "share"),
        (lambda: q.head_norm_rotary(x, None, p, f, out=(x[:1].clone().expand(5, 4, 128), None)), "twice"),
        (lambda: q.head_norm_rotary(x, x.clone(), p, f, out=(None, x)), "share"),
        (lambda: q.head_norm_rotary(x, x.clone(), p, f, out=(x.view(-1)[8:8 + 4 * 512].view(4, 4, 128), None)), "share"),
        (lambda: q.head_norm_rotary(x.clone(), x.clone(), p, f, out=(x, x)), "share"),
        (lambda: q.paged_keep(q.PagedCache(k, k.clone(), keys[:8].view(torch.int32).view(2, 2)), lengths, torch.zeros((2, 3), dtype=torch.int32)), "share"),
        (lambda: q.paged_keep(cache, lengths, i32(3).expand(2, 3)), "overlap")]
    for i, (call, why) in enumerate(wrong):
        print("refused?", i)
        with pytest.raises(ValueError, match=why):
            call()
