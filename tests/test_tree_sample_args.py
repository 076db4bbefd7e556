"""Argument checks of the drafted-tree and sampling entry points that need no
GPU: each call fails on the host, before any work, with a message that names it."""
import pytest

import paper_2608_19147_gb300 as pkg
from paper_2608_19147_gb300 import build as libbuild

P = 4096  # never followed: every call here is refused for another argument


@pytest.fixture(scope="module", autouse=True)
def lib():
    libbuild.build()


def attention(**over):
    a = dict(q=P, q_type=pkg.SHARD_F16, k=P, v=P, kv_type=pkg.SHARD_F16, out=P, out_type=pkg.SHARD_F16, B=1, N=4, n_heads=8, n_kv_heads=2,
             head_dim=64, capacity=128, kv_strides=(2 * 128 * 64, 128 * 64, 64), tree_start=P, parents=P, lens=P, mask=P, mask_stride=128,
             work=P, work_bytes=1 << 40)
    return pkg.shard_tree_attention(**{**a, **over}, check=False)


@pytest.mark.parametrize("over", [{k: 0} for k in ("q", "k", "v", "out", "tree_start", "parents", "lens", "work", "B", "N", "capacity", "mask_stride")] +
                         [{"B": -1}, {"B": pkg.SHARD_MAX_TREES + 1}, {"N": -3}, {"work_bytes": 0}, {"q": P + 8}, {"k": P + 2}, {"work": P + 4},
                          {"q_stride": 8}, {"out_stride": 511}, {"q_stride": 516}, {"kv_strides": (0, 0, 32)}, {"kv_strides": (-8, 64, 64)}, {"kv_strides": (0, 4, 64)}])
def test_attention_refuses(over):
    assert attention(**over) == pkg.SHARD_EINVAL
    assert "shard_tree_attention" in pkg.shard_last_error()


@pytest.mark.parametrize("over", [{"head_dim": 80}, {"n_heads": 6}, {"n_heads": 7}, {"n_heads": 64}, {"q_type": 5}, {"q_type": pkg.SHARD_BF16},
                                  {"kv_type": pkg.SHARD_F32}, {"out_type": -1}, {"N": 1 << 28}, {"capacity": (1 << 30) + 1}, {"kv_strides": (1 << 40, 64, 64)},
                                  {"B": 256, "capacity": 1 << 30}])
def test_attention_does_not_support(over):
    assert attention(**over) == pkg.SHARD_EUNSUPPORTED
    assert "shard_tree_attention" in pkg.shard_last_error()


def test_arrays_that_are_not_aligned_to_their_values():
    for name in ("tree_start", "parents", "lens", "status"):
        assert attention(**{name: P + 2}) == pkg.SHARD_EINVAL and "shard_tree_attention: an int32" in pkg.shard_last_error()
    good = dict(B=1, N=4, tree_start=P, parents=P, drafts=P, targets=P, path_stride=4, path=P, tokens=P, count=P)
    for name in ("tree_start", "parents", "drafts", "targets", "path", "tokens", "count", "status"):
        assert pkg.shard_tree_accept(**{**good, name: P + 1}, check=False) == pkg.SHARD_EINVAL and "aligned" in pkg.shard_last_error()
    assert pkg.shard_tree_accept(**good, lens=P + 2, attention_mask=P + 1, mask_stride=9, check=False) == pkg.SHARD_EINVAL
    good = dict(logits=P, type=pkg.SHARD_F32, M=1, V=8, ld=8, u=P, token=P)
    for name in ("u", "token", "temperature", "top_k", "top_p", "min_p", "p", "n_kept"):
        assert pkg.head_sample_logits(**{**good, name: P + 2}, check=False) == pkg.SHARD_EINVAL and "aligned" in pkg.shard_last_error()


def test_work_refuses():
    for bad in ((0, 8, 2, 64), (4, 0, 2, 64), (4, 8, 0, 64), (4, 8, 3, 64), (4, 8, 2, 63)):
        with pytest.raises(pkg.ShardError) as e:
            pkg.shard_tree_attention_work(*bad)
        assert e.value.code == pkg.SHARD_EINVAL


def test_accept_refuses():
    good = dict(B=1, N=4, tree_start=P, parents=P, drafts=P, targets=P, path_stride=4, path=P, tokens=P, count=P)
    for over in ([{k: 0} for k in good] + [{"B": pkg.SHARD_MAX_TREES + 1}, {"lens": P}, {"attention_mask": P}, {"lens": P, "attention_mask": P}]):
        assert pkg.shard_tree_accept(**{**good, **over}, check=False) == pkg.SHARD_EINVAL, over
        assert "shard_tree_accept" in pkg.shard_last_error()


def test_sampling_refuses():
    good = dict(logits=P, type=pkg.SHARD_F32, M=1, V=8, ld=8, u=P, token=P)
    for over in ({"logits": 0}, {"u": 0}, {"token": 0}, {"M": 0}, {"V": 0}, {"ld": 7}, {"type": 3}, {"logits": P + 2},
                 {"logits": P + 1, "type": pkg.SHARD_BF16}):
        assert pkg.head_sample_logits(**{**good, **over}, check=False) == pkg.SHARD_EINVAL, over
        assert "head_sample_logits" in pkg.shard_last_error()
    assert pkg.head_sample_logits(**{**good, "V": pkg.HEAD_MAX_SAMPLE_VOCAB + 1, "ld": 1 << 30}, check=False) == pkg.SHARD_EUNSUPPORTED
    assert pkg.head_sample(0, P, 1, P, P, check=False) == pkg.SHARD_EINVAL


def test_step_tree_refuses():
    assert pkg.shard_step_tree(0, P, P, None, [1], P, P, P, 64, P, check=False) == pkg.SHARD_EINVAL
    assert "shard_step_tree" in pkg.shard_last_error()


def test_tree_depths():
    from paper_2608_19147_gb300.spec import tree_depths

    assert tree_depths([]) == [] and tree_depths([-1]) == [0] and tree_depths([-1, 0, 0, 1, 3, 2]) == [0, 1, 1, 2, 3, 2]
    for bad in ([0], [-1, 1], [-1, -1], [-1, 0, 5]):
        with pytest.raises(ValueError):
            tree_depths(bad)


def test_decoder_settings():
    from paper_2608_19147_gb300.spec import TreeDecoder

    for bad in (dict(temperature=-0.1), dict(temperature=float("inf")), dict(temperature=float("nan")), dict(top_k=-1), dict(top_p=0.0), dict(top_p=1.1),
                dict(top_p=1e-50), dict(min_p=-0.1), dict(min_p=1.1), dict(B=0), dict(B=pkg.SHARD_MAX_REQUESTS + 1)):
        with pytest.raises(ValueError):
            TreeDecoder([], 64, P, **{"B": 1, "capacity": 16, **bad})
