"""README's example of the paged cache, as it stands there."""
import os

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def example() -> str:
    text = open(os.path.join(ROOT, "README.md")).read()
    at = text.index("cache = binding.PagedCache")
    return text[at:text.index("```", at)]
