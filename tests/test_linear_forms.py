"""Every form that the linear maps' kernels are built for has a shape that takes it, and no shape takes another (CPU)."""
import linear_forms


def test_every_form_has_a_shape():
    shapes = linear_forms.shapes()
    assert set(shapes) == set(linear_forms.expected())
    assert all(form in linear_forms.forms({"linear": "linear", "q8": "q8"}.get(form[0], "backward"), *shape)
               for form, found in shapes.items() for shape in found)
