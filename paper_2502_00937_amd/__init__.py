"""MI355X-native packed ViT image encoder: thin Python binding over libvitenc.so.

The binding marshals arguments only; every step of the encoder runs inside the HIP
library.  PyTorch supplies device memory and the stream.
"""
from .binding import (  # noqa: F401
    PRODUCT_EPILOGUES,
    PRODUCT_FORMS,
    TokenHandoff,
    VitEncoder,
    VitError,
    lib_path,
    load_library,
    preprocess_tiles,
    vit_encode_packed,
    vit_encode_packed_graph,
    vit_encode_packed_static,
    vit_encoder_create,
    vit_encoder_destroy,
    vit_encoder_query,
    vit_mfma_ceiling,
    vit_preprocess_tiles,
    vit_product_plan,
    vit_product_time,
    vit_weight_count,
)

_PAGES = ("PagePlan", "append_pages", "attend_pages", "plan_pages")


def __getattr__(name):  # the paged cache's calls are made of torch tensors: torch is imported with the first of them
    if name not in _PAGES:
        raise AttributeError(f"module {__name__!r} has no attribute {name!r}")
    from . import pages

    globals().update((n, getattr(pages, n)) for n in _PAGES)
    return globals()[name]
