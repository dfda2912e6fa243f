"""CPU test: the package offers the operators' calls by name, those that sample among them."""
import paper_2602_24082_amd as pkg
from paper_2602_24082_amd import binding


def test_sampling_calls_are_the_packages():
    names = [n for n in binding.EXPORTED if n.startswith(("pp_cache_", "pp_tree_attn", "pp_verify_draft")) and not n.endswith("_size")]
    assert len(names) == 9
    for n in [*names, "Cache", "make_cache"]:
        assert getattr(pkg, n) is getattr(binding, n)
